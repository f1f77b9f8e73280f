// Attention of a stream of frames over a window and a few first frames (dsattn_sink_forward), and the
// upkeep of the cache that it reads.
//
// A query of frame a sees the frames [0, ns) and [lo, a], where lo = max(0, a - window + 1) is the first
// frame of its window and ns = min(sinks, lo): two runs that do not meet.
//
// Few queries of a head of K and V are a stream of the cache (sink_rows.h), more of them matrix products (sink_tile.h); head
// sizes that are neither have a wavefront a query.  us, and of a large copy's or library product's rate:
//   16 streams, a token of 32 heads on 8 x 128 over 16,388      225   93 %
//   a frame of 160 positions, 8 x 160, over 64                 12.8   82 %   (fp32 19.5)
//   128 frames of 640 positions, 8 x 80, window 32, cached      130   74 %   (fp32 311; on a full ring of 32, which a kernel
//                                                                     after it fills, 150 and 320)
//   2 prompts of 8,192, 16 heads on 4 x 128, window 2,048       276 to 295   53 to 57 %   (fp32 2,000)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dsattn.h"
#include "plan.h"

namespace dsattn {
namespace {

struct SinkArgs {
    const void *Q, *K, *V;
    void *Kc, *Vc, *O;
    const int32_t *start, *counts;  // or null
    int32_t B, T, P, h, hk, D, sinks, window, ring;
    float sc;  // softmax scale * log2(e)
    int32_t U, splits, fused;  // see sink_rows.h: units of a wavefront; parts of a row's frames; see puts_frames()
    float *parts;              // partial results of the splits
    int32_t per_xcd, row_tiles;  // see sink_tile.h: workgroups of an XCD, row tiles of a unit, tasks in all
    int64_t tasks;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// A stream's place: its first new frame, and how many there are.
struct Stream {
    int start, count;
};
__device__ __forceinline__ Stream stream_of(const SinkArgs &a, int b)
{
    Stream s;
    s.start = a.start ? min(max(a.start[b], 0), 0x7fffffff - a.T) : 0;
    s.count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
    return s;
}

// Whether the attention itself puts a stream's new frames into the cache, rather than a kernel after it: where none of them
// takes a slot whose frame a query of the call still reads.  `fused`: 1, the ring has room for both (or nothing is cached
// yet, for all streams); 2, where the stream has nothing cached yet; 0, never.
__device__ __forceinline__ bool puts_frames(const SinkArgs &a, const Stream &s) { return a.fused == 1 || (a.fused == 2 && s.start == 0); }
// Whether new frame f stays in the cache when the call is done: of several with one slot the last one does.
__device__ __forceinline__ bool stays(const SinkArgs &a, const Stream &s, int f)
{
    return f < a.sinks || s.start + s.count - 1 - f < a.ring;
}

// slot of a frame in the cache
__device__ __forceinline__ int slot_of(const SinkArgs &a, int f)
{
    return f < a.sinks ? f : a.sinks + (f - a.sinks) % a.ring;
}

// The frames that the queries of the new frames t0 .. t1 see between them: the first ns, and the frames from lo on; n in all, and
// frame(j) the j-th of them.
struct Frames {
    int ns, lo, n, base, base_slot;
    __device__ __forceinline__ int frame(int j) const { return j < ns ? j : j + (lo - ns); }
    // slot_of() for these frames: the ones behind the sinks are within one turn of the ring
    __device__ __forceinline__ int slot(const SinkArgs &a, int f) const
    {
        const int s = base_slot + (f - base);
        return f < a.sinks ? f : s >= a.sinks + a.ring ? s - a.ring : s;
    }
};
__device__ __forceinline__ Frames frames_of(const SinkArgs &a, const Stream &s, int t0, int t1)
{
    Frames f;
    f.lo = max(0, s.start + t0 - a.window + 1);
    f.ns = min(a.sinks, f.lo);
    f.n = f.ns + (s.start + t1 + 1 - f.lo);
    f.base = max(f.lo, a.sinks);
    f.base_slot = slot_of(a, f.base);
    return f;
}

// A split's partial result for row r of a unit: maximum, sum, two unused numbers, weighted sum.
constexpr int kPartHead = 4, kMaxSplits = 64;
__device__ __forceinline__ float *part_of(const SinkArgs &a, int b, int64_t unit, int r, int rows, int split)
{
    const int64_t row = (((int64_t)b * a.P * a.hk + unit) * rows + r) * a.splits + split;
    return a.parts + row * (a.D + kPartHead);
}

// Row of frame f of stream b in K or V, or in their caches.
template <typename T>
__device__ __forceinline__ const T *frame_row(const SinkArgs &a, const void *fresh, const void *cache, int b, const Stream &s, int f)
{
    const int64_t row = (int64_t)a.P * a.hk * a.D;
    if (f >= s.start) return (const T *)fresh + ((int64_t)b * a.T + (f - s.start)) * row;
    return (const T *)cache + ((int64_t)b * (a.sinks + a.ring) + slot_of(a, f)) * row;
}

__device__ __forceinline__ float wave_sum(float x)
{
    for (int w = 32; w > 0; w >>= 1) x += __shfl_xor(x, w);
    return x;
}

// One query and head on a wavefront's vector ALUs: lane l has channels l, l + 64, ...
constexpr int kMaxDim = 512;
template <typename T>
__device__ __forceinline__ void vector_row(const SinkArgs &a, int b, const Stream &s, int t, int p, int g, int lane)
{
    const int D = a.D;
    const int64_t id = (((int64_t)b * a.T + t) * a.P + p) * a.h + g;
    const T *q = (const T *)a.Q + id * D;
    const int64_t at = ((int64_t)p * a.hk + g / (a.h / a.hk)) * D;  // within a frame of K and V
    constexpr int R = kMaxDim / 64;
    float qv[R], o[R], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        qv[r] = lane + 64 * r < D ? (float)q[lane + 64 * r] * a.sc : 0.f;
        o[r] = 0.f;
    }
    const Frames fr = frames_of(a, s, t, t);
    for (int j = 0; j < fr.n; ++j) {
        const int f = fr.frame(j);
        const T *k = frame_row<T>(a, a.K, a.Kc, b, s, f) + at, *v = frame_row<T>(a, a.V, a.Vc, b, s, f) + at;
        float x = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (lane + 64 * r < D) x = fmaf(qv[r], (float)k[lane + 64 * r], x);
        x = wave_sum(x);
        const float mn = fmaxf(m, x), shift = mn == -INFINITY ? 0.f : mn;
        const float w = exp2f(x - shift), old = exp2f(m - shift);
        m = mn;
        l = fmaf(l, old, w);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (lane + 64 * r < D) o[r] = fmaf(w, (float)v[lane + 64 * r], o[r] * old);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *out = (T *)a.O + id * D;
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (lane + 64 * r < D) out[lane + 64 * r] = (T)(o[r] * inv);
}

// Plain vector kernel for every shape: a wavefront a query and head.
template <typename T>
__global__ __launch_bounds__(256) void sink_generic_kernel(const SinkArgs a)
{
    const int64_t tasks = (int64_t)a.B * a.T * a.P * a.h;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= tasks) return;
    const int g = (int)(id % a.h);
    const int64_t tok = id / a.h;  // (b T + t) P + p
    const int p = (int)(tok % a.P);
    const int t = (int)(tok / a.P % a.T), b = (int)(tok / a.P / a.T);
    const Stream s = stream_of(a, b);
    if (t < s.count) vector_row<T>(a, b, s, t, p, g, threadIdx.x & 63);
}

// New frames into the cache, in units that divide a frame's row: blockIdx.y is the new frame (and every
// gridDim.y-th after it), blockIdx.z the stream and K or V.
template <typename U>
__global__ __launch_bounds__(256) void sink_append_kernel(const SinkArgs a, int64_t units)
{
    const int b = (int)(blockIdx.z >> 1);
    const Stream s = stream_of(a, b);
    if (puts_frames(a, s)) return;
    const bool v = blockIdx.z & 1;
    for (int t = (int)blockIdx.y; t < s.count; t += (int)gridDim.y) {
        const int f = s.start + t;
        if (!stays(a, s, f)) continue;
        const U *from = (const U *)(v ? a.V : a.K) + ((int64_t)b * a.T + t) * units;
        U *to = (U *)(v ? a.Vc : a.Kc) + ((int64_t)b * (a.sinks + a.ring) + slot_of(a, f)) * units;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < units; i += (int64_t)gridDim.x * 256) to[i] = from[i];
    }
}

}  // namespace
}  // namespace dsattn

#include "sink_rows.h"
#include "sink_tile.h"

namespace dsattn {
namespace {

// Joins the splits of a row (64 at most): a workgroup a row, lane l of a wavefront has split l's maximum and sum, and then
// channels l, l + 64, ... of every fourth split, four of them in flight.
template <typename T>
__global__ __launch_bounds__(256) void sink_join_kernel(const SinkArgs a)
{
    constexpr int R = kMaxDim / 64, U = 4;
    __shared__ float sums[3][kMaxDim];
    const int g = a.h / a.hk, rows = a.T * g, D = a.D;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int64_t id = blockIdx.x, units = (int64_t)a.P * a.hk;
    const int r = (int)(id % rows), t = r / g;
    const int64_t unit = id / rows % units;
    const int b = (int)(id / rows / units);
    if (t >= stream_of(a, b).count) return;
    const float *parts = part_of(a, b, unit, r, rows, 0);
    const int stride = D + kPartHead;
    const bool mine = lane < a.splits;
    const float m = mine ? parts[lane * stride] : -INFINITY;
    float l = mine ? parts[lane * stride + 1] : 0.f, top = m;
    for (int w = 32; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
    l = wave_sum(l * f);
    float o[R] = {};
    for (int s0 = wv; s0 < a.splits; s0 += 4 * U) {
        float x[U][R];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int s = min(s0 + 4 * u, a.splits - 1);
                x[u][i] = lane + 64 * i < D ? parts[s * stride + kPartHead + lane + 64 * i] : 0.f;
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + 4 * u;
            const float fs = __shfl(f, min(s, a.splits - 1));
#pragma unroll
            for (int i = 0; i < R; ++i) o[i] = s < a.splits ? fmaf(x[u][i], fs, o[i]) : o[i];
        }
    }
    if (wv > 0)
#pragma unroll
        for (int i = 0; i < R; ++i) sums[wv - 1][lane + 64 * i] = o[i];
    __syncthreads();
    if (wv > 0) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        for (int w = 0; w < 3; ++w) o[i] += sums[w][lane + 64 * i];
        o[i] *= inv;
        nan = nan || o[i] != o[i];
    }
    const int p = (int)(unit / a.hk), head = (int)(unit % a.hk) * g + r % g;
    if (__any(nan)) {  // (a hidden frame's infinity times its weight of zero)
        vector_row<T>(a, b, stream_of(a, b), t, p, head, lane);
        return;
    }
    T *to = (T *)a.O + (((int64_t)b * a.T + t) * a.P + p) * a.h * D + (int64_t)head * D;
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (lane + 64 * i < D) to[lane + 64 * i] = (T)o[i];
}

bool overlap(const void *a, int64_t an, const void *b, int64_t bn)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + (uintptr_t)bn && y < x + (uintptr_t)an;
}

constexpr float kLog2e = 1.44269504f;

int sink_validate(const dsattn_sink_desc *d, const char *who)
{
    if (!d) return fail(DSATTN_EINVAL, "%s: null descriptor", who);
    if (d->streams < 1 || d->frames < 1 || d->spatial < 1 || d->heads < 1 || d->kv_heads < 1)
        return fail(DSATTN_EINVAL, "%s: sizes must be positive", who);
    if (d->head_dim < 1 || d->head_dim > kMaxDim)
        return fail(DSATTN_EINVAL, "%s: head_dim %d outside [1, %d]", who, d->head_dim, kMaxDim);
    if (d->heads % d->kv_heads != 0)
        return fail(DSATTN_EINVAL, "%s: kv_heads %d does not divide heads %d", who, d->kv_heads, d->heads);
    if (d->sinks < 0 || d->window < 0) return fail(DSATTN_EINVAL, "%s: sinks and window must be >= 0", who);
    if (d->ring < 1 || d->ring < d->window)
        return fail(DSATTN_EINVAL, "%s: a ring of %d frames does not hold a window of %d", who, d->ring, d->window);
    if (d->io_dtype != DSATTN_F32 && d->io_dtype != DSATTN_BF16)
        return fail(DSATTN_EINVAL, "%s: unknown dtype", who);
    if (!std::isfinite(d->scale) || std::isinf(std::max(d->scale, 0.f) * kLog2e))
        return fail(DSATTN_EINVAL, "%s: scale is not finite, or is not times log2(e)", who);
    if (d->flags & ~DSATTN_FLAG_FORCE_GENERIC)
        return fail(DSATTN_EINVAL, "%s: unknown flag bits 0x%x", who, d->flags);
    // 2^24 frames, 2^20 channels, 2^40 numbers a tensor at most
    const int64_t C = (int64_t)d->heads * d->head_dim, slots = (int64_t)d->sinks + d->ring;
    const int64_t most = (int64_t)1 << 40, frames = std::max<int64_t>(d->frames, slots);
    if (C > (1 << 20) || d->frames > (1 << 24) || slots > (1 << 24) || d->streams > 65535 / 2 ||
        (int64_t)d->streams * d->spatial > most / C || (int64_t)d->streams * d->spatial * C > most / frames)
        return fail(DSATTN_EINVAL, "%s: problem too large", who);
    return DSATTN_OK;
}

// How a shape runs: all of it follows from the descriptor, so that the workspace does too.
struct SinkLaunch {
    RowsLaunch rows;
    TileLaunch tile;
    int splits;
};
SinkLaunch sink_launch(const dsattn_sink_desc &d)
{
    SinkLaunch k{};
    k.splits = 1;
    if (d.flags & DSATTN_FLAG_FORCE_GENERIC) return k;
    k.rows = rows_launch(d);
    if (k.rows.fn) {
        k.splits = k.rows.splits;
        return k;
    }
    k.tile = tile_launch(d);
    if (k.tile.fn) k.splits = k.tile.splits;
    return k;
}
size_t sink_workspace_bytes(const dsattn_sink_desc &d)
{
    const SinkLaunch k = sink_launch(d);
    if (k.splits == 1) return 0;
    return (size_t)d.streams * d.spatial * d.heads * d.frames * k.splits * (d.head_dim + kPartHead) * sizeof(float);
}

}  // namespace
}  // namespace dsattn

using namespace dsattn;

extern "C" {

int dsattn_sink_workspace(const dsattn_sink_desc *desc, size_t *bytes)
{
    const int rc = sink_validate(desc, "dsattn_sink_workspace");
    if (rc != DSATTN_OK) return rc;
    if (!bytes) return fail(DSATTN_EINVAL, "dsattn_sink_workspace: null output");
    *bytes = sink_workspace_bytes(*desc);
    return DSATTN_OK;
}

int dsattn_sink_forward_info(const dsattn_sink_desc *desc, dsattn_sink_info *info)
{
    const int rc = sink_validate(desc, "dsattn_sink_forward_info");
    if (rc != DSATTN_OK) return rc;
    if (!info) return fail(DSATTN_EINVAL, "dsattn_sink_forward_info: null output");
    const dsattn_sink_desc &d = *desc;
    const SinkLaunch k = sink_launch(d);
    *info = dsattn_sink_info{};
    info->splits = k.splits;
    info->block_threads = 256;
    if (k.rows.fn) {
        info->kernel = 1;
        info->n_blocks = (int32_t)k.rows.blocks;
        info->lds_bytes = k.rows.lds;
    } else if (k.tile.fn) {
        info->kernel = k.tile.shared ? 3 : 2;
        info->tile_rows = k.tile.rows;
        info->tile_frames = k.tile.frames;
        info->n_blocks = (int32_t)((k.tile.workgroups + 7) / 8 * 8);
        info->block_threads = 64 * k.tile.waves;
        info->lds_bytes = k.tile.lds;
    } else {
        info->n_blocks = (int32_t)std::min<int64_t>(((int64_t)d.streams * d.frames * d.spatial * d.heads + 3) / 4, 0x7fffffff);
    }
    return DSATTN_OK;
}

int dsattn_sink_forward(const dsattn_sink_desc *desc, const int32_t *start, const int32_t *counts,
                        const void *Q, const void *K, const void *V, void *Kcache, void *Vcache, void *O,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "dsattn_sink_forward";
    const int rc = sink_validate(desc, who);
    if (rc != DSATTN_OK) return rc;
    const dsattn_sink_desc &d = *desc;
    if (!Q || !K || !V || !O) return fail(DSATTN_EINVAL, "%s: null pointer", who);
    if (!Kcache != !Vcache) return fail(DSATTN_EINVAL, "%s: one cache without the other", who);
    if (!Kcache && start) return fail(DSATTN_EINVAL, "%s: a start without caches", who);
    if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O | (uintptr_t)Kcache | (uintptr_t)Vcache |
         (uintptr_t)workspace) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    if (((uintptr_t)start | (uintptr_t)counts) & 3u)
        return fail(DSATTN_EINVAL, "%s: start and counts must be 4-byte aligned", who);
    const size_t need = sink_workspace_bytes(d);
    if (workspace_bytes < need || (need && !workspace))
        return fail(DSATTN_EINVAL, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, need);
    const int64_t es = d.io_dtype == DSATTN_BF16 ? 2 : 4;
    const int64_t per = (int64_t)d.streams * d.spatial * d.head_dim * es, row = d.spatial * (int64_t)d.kv_heads * d.head_dim;
    const int64_t qn = per * d.frames * d.heads, kn = per * d.frames * d.kv_heads;
    const int64_t cn = per * d.kv_heads * ((int64_t)d.sinks + d.ring), sn = 4 * (int64_t)d.streams;
    const struct { const void *p; int64_t n; } all[] = {
        {O, qn}, {Kcache, cn}, {Vcache, cn}, {workspace, (int64_t)need}, {Q, qn}, {K, kn}, {V, kn}, {start, sn}, {counts, sn}};
    for (int o = 0; o < 4; ++o)
        for (int i = o + 1; i < 9; ++i)
            if (overlap(all[o].p, all[o].n, all[i].p, all[i].n))
                return fail(DSATTN_EINVAL, "%s: an output, a cache or the workspace overlaps another tensor", who);
    SinkArgs a{};
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.Kc = Kcache;
    a.Vc = Vcache;
    a.O = O;
    a.start = start;
    a.counts = counts;
    a.B = d.streams;
    a.T = d.frames;
    a.P = d.spatial;
    a.h = d.heads;
    a.hk = d.kv_heads;
    a.D = d.head_dim;
    a.sinks = d.sinks;
    a.window = d.window;
    a.ring = d.ring;
    a.sc = (d.scale > 0.f ? d.scale : 1.f / sqrtf((float)d.head_dim)) * kLog2e;
    const hipStream_t st = (hipStream_t)stream;
    const SinkLaunch k = sink_launch(d);
    const bool f32 = d.io_dtype == DSATTN_F32;
    a.splits = k.splits;
    a.parts = (float *)workspace;
    hipError_t e = hipSuccess;
    if ((k.rows.fn || k.tile.fn) && Kcache && d.window >= 1)  // (without a window a query does not see its own frame)
        a.fused = !start || d.ring >= (int64_t)d.window + d.frames - 1 ? 1 : 2;
    if (k.rows.fn) {
        a.U = k.rows.U;
        void *params[] = {&a};
        e = hipLaunchKernel(k.rows.fn, dim3((unsigned)k.rows.blocks), dim3(256), params, (size_t)k.rows.lds, st);
    } else if (k.tile.fn) {
        a.row_tiles = k.tile.row_tiles;
        a.tasks = k.tile.tasks;
        a.per_xcd = (int)((k.tile.workgroups + 7) / 8);
        void *params[] = {&a};
        // the default cap on dynamic LDS is 64 KB
        if (k.tile.lds > 64 << 10) e = hipFuncSetAttribute(k.tile.fn, hipFuncAttributeMaxDynamicSharedMemorySize, k.tile.lds);
        if (e == hipSuccess)
            e = hipLaunchKernel(k.tile.fn, dim3((unsigned)a.per_xcd * 8u), dim3(64u * k.tile.waves), params, (size_t)k.tile.lds, st);
    } else {
        // (a launch has less than 2^32 threads)
        const int64_t blocks = ((int64_t)a.B * a.T * a.P * a.h + 3) / 4;
        if (blocks > 0xffffff) return fail(DSATTN_EUNSUPPORTED, "%s: too large for the generic kernel", who);
        if (f32)
            hipLaunchKernelGGL((sink_generic_kernel<float>), dim3((unsigned)blocks), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((sink_generic_kernel<__bf16>), dim3((unsigned)blocks), dim3(256), 0, st, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && k.splits > 1) {
        const unsigned blocks = (unsigned)((int64_t)a.B * a.T * a.P * a.h);
        if (f32)
            hipLaunchKernelGGL((sink_join_kernel<float>), dim3(blocks), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((sink_join_kernel<__bf16>), dim3(blocks), dim3(256), 0, st, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && Kcache && a.fused != 1) {
        // in units that divide a frame's row
        const bool wide = row * es % 16 == 0;
        const int64_t units = wide ? row * es / 16 : row;
        // some 4,096 workgroups, of which those of streams that have theirs already end at once
        const int64_t per = std::max<int64_t>(1, 4096 / (2 * a.B)), x = std::min<int64_t>((units + 255) / 256, per);
        const dim3 grid((unsigned)x, (unsigned)std::min<int64_t>(a.T, std::max<int64_t>(1, per / x)), 2u * a.B);
        if (wide)
            hipLaunchKernelGGL((sink_append_kernel<uint4>), grid, dim3(256), 0, st, a, units);
        else if (es == 4)
            hipLaunchKernelGGL((sink_append_kernel<uint32_t>), grid, dim3(256), 0, st, a, units);
        else
            hipLaunchKernelGGL((sink_append_kernel<uint16_t>), grid, dim3(256), 0, st, a, units);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
}

}  // extern "C"
