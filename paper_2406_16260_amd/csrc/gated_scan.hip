// Gated linear recurrence over frames and its backward pass (dsattn_gated_scan, dsattn_gated_scan_backward).
//
//   a_t = sigmoid(g_t),  h_t = a_t h_(t-1) + w(a_t) x_t            w = 1, 1 - a or sqrt(1 - a^2)
//   D_t = dy_t + a_(t+1) D_(t+1),  dx_t = w D_t,  dg_t = D_t (a (1 - a) h_(t-1) + x_t dw/dg)
//
// Bound by memory.  Positions and channels are independent and lie next to each other: a lane has four bytes of a frame (two
// bf16 or one fp32 channel) and walks the frames, those ahead already on their way.  Where that makes too few wavefronts the
// frames are cut into chunks: a first pass finds what each chunk does to a state (its product of gates A and its result H
// from 0), one kernel joins these, and the chunks run again from their states.  The backward pass does the same from the end; it
// needs the states h, which it runs again, in 32 bits, from those that the forward pass left every 16 frames.
// us and TB/s (a large copy 5.1):
//   384 frames x 640 x 640, bf16, forward           197     4.8
//   384 frames x 160 x 1,280, bf16, backward        172     4.7
//   2 x 16,384 frames x 1, x 1,280, bf16, forward   98      2.6, 4.3 of what is read twice
//   1 frame x 160 x 1,280, bf16                     7.4     of which 4.8 are the host's marshalling and 2.6 its launch
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "dsattn.h"
#include "plan.h"
#include "rows.h"

namespace dsattn {
namespace {

constexpr int kStep = DSATTN_SCAN_FRAMES;

struct ScanArgs {
    const void *X, *G, *dY;
    const float *states_in;   // backward: [B][steps][n]
    const float *carry_in;    // start state, or the end state's gradient; null: 0
    const int32_t *counts;    // or null
    void *Y;                  // Y, or dX
    void *dG;
    float *carry_out;         // end state, or the start state's gradient; null: not wanted
    float *states_out;        // forward: [B][steps][n] or null
    float *A, *H;             // of chunks: [B][chunks][n]; after the join H is what each chunk starts from
    int64_t n;                // P * channels
    int32_t B, T, steps;      // steps: ceil(T / kStep)
    int32_t chunk, chunks;    // frames of a chunk (a multiple of kStep), chunks of a stream
};

// e^x, within two ulps: 2^(x log2(e)), and what the product's rounding has left of x
__device__ __forceinline__ float exp_of(float x)
{
    const float p = x * 1.44269504f;
    const float left = fmaf(p, 1.90465430e-9f, fmaf(p, -0.693147182f, x));  // x - p ln 2, ln 2 in two parts
    const float e = __builtin_amdgcn_exp2f(p);
    return fmaf(e, left, e);
}

// What a gate keeps, a = sigmoid(g), what it leaves, 1 - a, and what it lets in, w(a): each with a small relative error.  (The
// instructions for quotients and roots, an ulp off at most, not the sequences that round them, which took twice the time.)
// With e = e^-g, a = 1 / (1 + e), 1 - a = e a, and 1 - a^2 = e a (1 + a), whose root is taken with e^(-g / 2) outside, so that it
// does not underflow before w does.  Below -87, where e would soon be infinite, e is that of -87, and what a gate of -87 keeps,
// 2^-125.5, is taken off what every gate does: it is 0 there, so that a frame that begins anew is free of the state before it, of
// whatever size that is, and unchanged from 2^-100 up.  (One instruction; with a comparison and a choice 384 frames x 640 x 640 197 us
// and 2,304 x 160 x 320 226, instead of 194.6 and 215.)  Beyond 210, where even e^(-g / 2) is 0 in fp32, a gate is one of 210: infinite
// logits are gates of 0 and of 1.
struct Gate {
    float keep, leave, let;
};
constexpr float kFar = 87.f;
template <int MODE>
__device__ __forceinline__ Gate gate_at(float x)  // x: -g
{
    Gate q;
    if constexpr (MODE == DSATTN_SCAN_NORM) {
        const float h = exp_of(0.5f * x), e = h * h;
        q.keep = __builtin_amdgcn_rcpf(1.f + e);
        q.leave = e * q.keep;
        q.let = h * __builtin_amdgcn_sqrtf(fmaf(q.keep, q.keep, q.keep));
    } else {
        const float e = exp_of(x);
        q.keep = __builtin_amdgcn_rcpf(1.f + e);
        q.leave = e * q.keep;
        q.let = MODE == DSATTN_SCAN_MEAN ? q.leave : 1.f;
    }
    return q;
}
// What a gate of -87 keeps, by the instructions that gates come from.
template <int MODE>
__device__ __forceinline__ float least_kept()
{
    float x = kFar;
    asm volatile("" : "+v"(x));  // (or the compiler works it out by arithmetic of its own)
    return gate_at<MODE>(x).keep;
}
template <int MODE>
__device__ __forceinline__ Gate gate_of(float g, float least)
{
    Gate q = gate_at<MODE>(__builtin_elementwise_minimum(__builtin_elementwise_maximum(-g, -210.f), kFar));  // (a NaN stays)
    q.keep -= least;
    return q;
}
// dw / dg
template <int MODE>
__device__ __forceinline__ float slope_of(const Gate &q)
{
    if constexpr (MODE == DSATTN_SCAN_MEAN) return -q.keep * q.leave;
    if constexpr (MODE == DSATTN_SCAN_NORM) return -q.keep * q.keep * q.let * __builtin_amdgcn_rcpf(1.f + q.keep);
    return 0.f;
}

template <typename T, int V>
struct Lane {
    typedef T Piece __attribute__((ext_vector_type(V)));
};

// This lane's first channel, stream and frames.  (Grid: channels, chunks, streams.)  An address is the workgroup's, which the
// scalar unit moves from frame to frame, and the lane's offset.
template <int V>
struct Place {
    int64_t c0, c;  // the workgroup's first channel, the lane's
    uint32_t lane;
    int b, j, t0, t1;  // frames [t0, t1): none where the stream is over
    __device__ __forceinline__ Place(const ScanArgs &a)
    {
        c0 = (int64_t)blockIdx.x * (256 * V);
        lane = threadIdx.x * V;
        c = c0 + lane;
        j = (int)blockIdx.y;
        b = (int)blockIdx.z;
        const int count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
        t0 = (int)min((int64_t)j * a.chunk, (int64_t)count);
        t1 = (int)min((int64_t)(j + 1) * a.chunk, (int64_t)count);
    }
};

// Steps of kStep frames, the next one's on their way meanwhile.  With STORE the states and Y are written, else A and H of the chunk.
template <typename T, int V, int MODE, bool STORE>
__global__ __launch_bounds__(256) void scan_kernel(const ScanArgs a)
{
    using Piece = typename Lane<T, V>::Piece;
    const Place<V> p(a);
    if (p.c >= a.n) return;
    const int64_t base = (int64_t)p.b * a.T * a.n + p.c0, part = ((int64_t)p.b * a.chunks + p.j) * a.n + p.c;
    const T *X = (const T *)a.X + base, *G = (const T *)a.G + base;
    const float least = least_kept<MODE>();
    float h[V], prod[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        prod[v] = 1.f;
        h[v] = 0.f;
        if constexpr (STORE) h[v] = a.chunks > 1 ? a.H[part + v] : a.carry_in ? a.carry_in[(int64_t)p.b * a.n + p.c + v] : 0.f;
    }
    Piece x[kStep], g[kStep];
    auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            const int64_t at = (int64_t)min(t + i, p.t1 - 1) * a.n;  // (past the end: the last one again, not used)
            x[i] = *(const Piece *)(X + at + p.lane);
            g[i] = *(const Piece *)(G + at + p.lane);
        }
    };
    if (p.t1 > p.t0) fetch(p.t0);
    // (whole steps in a loop of their own, where no branch keeps the gates of different frames apart: 2,304 frames x 160 x 320
    // 280 -> 241 us)
    auto step = [&](int t, auto whole) __attribute__((always_inline)) {
        Piece xc[kStep], gc[kStep];
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            xc[i] = x[i];
            gc[i] = g[i];
        }
        if (t + kStep < p.t1) fetch(t + kStep);
        if constexpr (STORE) {
            if (a.states_out) {
                float *to = a.states_out + ((int64_t)p.b * a.steps + t / kStep) * a.n + p.c;
#pragma unroll
                for (int v = 0; v < V; ++v) to[v] = h[v];
            }
        }
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            if (!decltype(whole)::value && t + i >= p.t1) break;
            Piece y;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate q = gate_of<MODE>((float)gc[i][v], least);
                h[v] = fmaf(q.keep, h[v], q.let * (float)xc[i][v]);
                if constexpr (STORE)
                    y[v] = (T)h[v];
                else
                    prod[v] *= q.keep;
            }
            if constexpr (STORE) *(Piece *)((T *)a.Y + base + (int64_t)(t + i) * a.n + p.lane) = y;
        }
    };
    int t = p.t0;
    for (; t + kStep <= p.t1; t += kStep) step(t, std::true_type{});
    if (t < p.t1) step(t, std::false_type{});
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if constexpr (!STORE) {
            a.A[part + v] = prod[v];
            a.H[part + v] = h[v];
        } else if (a.chunks == 1 && a.carry_out) {
            a.carry_out[(int64_t)p.b * a.n + p.c + v] = h[v];
        }
    }
}

// The same from the end: c is a_(t+1) D_(t+1), what frame t gets of the later ones.
template <typename T, int V>
__global__ __launch_bounds__(256) void scan_back_parts_kernel(const ScanArgs a)
{
    using Piece = typename Lane<T, V>::Piece;
    const Place<V> p(a);
    if (p.c >= a.n) return;
    const int64_t base = (int64_t)p.b * a.T * a.n + p.c0, part = ((int64_t)p.b * a.chunks + p.j) * a.n + p.c;
    const T *G = (const T *)a.G + base, *dY = (const T *)a.dY + base;
    const float least = least_kept<DSATTN_SCAN_SUM>();
    float c[V], prod[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        prod[v] = 1.f;
        c[v] = 0.f;
    }
    auto step = [&](int t, auto whole) __attribute__((always_inline)) {
        Piece g[kStep], dy[kStep];
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            const int64_t at = (int64_t)min(t + i, p.t1 - 1) * a.n;  // (past the end: the last one again, not used)
            g[i] = *(const Piece *)(G + at + p.lane);
            dy[i] = *(const Piece *)(dY + at + p.lane);
        }
#pragma unroll
        for (int i = kStep - 1; i >= 0; --i) {
            if (!decltype(whole)::value && t + i >= p.t1) continue;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float keep = gate_of<DSATTN_SCAN_SUM>((float)g[i][v], least).keep;
                c[v] = keep * (c[v] + (float)dy[i][v]);
                prod[v] *= keep;
            }
        }
    };
    const int whole = p.t0 + (p.t1 - p.t0) / kStep * kStep;  // the end of the whole steps
    if (whole < p.t1) step(whole, std::false_type{});
    for (int t = whole - kStep; t >= p.t0; t -= kStep) step(t, std::true_type{});
#pragma unroll
    for (int v = 0; v < V; ++v) {
        a.A[part + v] = prod[v];
        a.H[part + v] = c[v];
    }
}

template <typename T, int V, int MODE>
__global__ __launch_bounds__(256) void scan_back_kernel(const ScanArgs a)
{
    using Piece = typename Lane<T, V>::Piece;
    const Place<V> p(a);
    if (p.c >= a.n) return;
    const int64_t base = (int64_t)p.b * a.T * a.n + p.c0, part = ((int64_t)p.b * a.chunks + p.j) * a.n + p.c;
    const T *X = (const T *)a.X + base, *G = (const T *)a.G + base, *dY = (const T *)a.dY + base;
    const float *S = a.states_in + (int64_t)p.b * a.steps * a.n + p.c;
    const float least = least_kept<MODE>();
    float c[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        c[v] = a.chunks > 1 ? a.H[part + v] : a.carry_in ? a.carry_in[(int64_t)p.b * a.n + p.c + v] : 0.f;
    Piece x[kStep], g[kStep], dy[kStep];
    float s[V];
    auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = S[(int64_t)(t / kStep) * a.n + v];
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            const int64_t at = (int64_t)min(t + i, p.t1 - 1) * a.n;  // (past the end: the last one again, not used)
            x[i] = *(const Piece *)(X + at + p.lane);
            g[i] = *(const Piece *)(G + at + p.lane);
            dy[i] = *(const Piece *)(dY + at + p.lane);
        }
    };
    auto step = [&](int t, auto whole) __attribute__((always_inline)) {
        Piece xc[kStep], gc[kStep], dc[kStep];
        float h[kStep][V];  // the state in front of each frame
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            xc[i] = x[i];
            gc[i] = g[i];
            dc[i] = dy[i];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) h[0][v] = s[v];
        if (t - kStep >= p.t0) fetch(t - kStep);
#pragma unroll
        for (int i = 0; i + 1 < kStep; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate q = gate_of<MODE>((float)gc[i][v], least);
                h[i + 1][v] = fmaf(q.keep, h[i][v], q.let * (float)xc[i][v]);  // (past the end: not used)
            }
#pragma unroll
        for (int i = kStep - 1; i >= 0; --i) {
            if (!decltype(whole)::value && t + i >= p.t1) continue;
            Piece dx, dg;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate q = gate_of<MODE>((float)gc[i][v], least);
                const float d = c[v] + (float)dc[i][v];
                dx[v] = (T)(d * q.let);
                if constexpr (MODE == DSATTN_SCAN_MEAN)  // the two slopes differ in sign only
                    dg[v] = (T)(d * (q.keep * q.leave) * (h[i][v] - (float)xc[i][v]));
                else
                    dg[v] = (T)(d * fmaf(q.keep * q.leave, h[i][v], slope_of<MODE>(q) * (float)xc[i][v]));
                c[v] = q.keep * d;
            }
            *(Piece *)((T *)a.Y + base + (int64_t)(t + i) * a.n + p.lane) = dx;
            *(Piece *)((T *)a.dG + base + (int64_t)(t + i) * a.n + p.lane) = dg;
        }
    };
    const int whole = p.t0 + (p.t1 - p.t0) / kStep * kStep;  // the end of the whole steps
    if (p.t1 > p.t0) fetch(whole < p.t1 ? whole : whole - kStep);
    if (whole < p.t1) step(whole, std::false_type{});
    for (int t = whole - kStep; t >= p.t0; t -= kStep) step(t, std::true_type{});
    if (a.chunks == 1 && a.carry_out) {
#pragma unroll
        for (int v = 0; v < V; ++v) a.carry_out[(int64_t)p.b * a.n + p.c + v] = c[v];
    }
}

// What each chunk starts from: 16 channels a workgroup, 64 threads to each, which have runs of chunks.  BACK: from the last on.
template <bool BACK>
__global__ __launch_bounds__(1024) void scan_join_kernel(const ScanArgs a)
{
    __shared__ float As[64][17], Hs[64][17];
    const int l = threadIdx.x & 15, w = threadIdx.x >> 4, b = (int)blockIdx.y;
    const int64_t c = (int64_t)blockIdx.x * 16 + l;
    const bool there = c < a.n;
    const int per = (a.chunks + 63) / 64, first = min(w * per, a.chunks), end = min(first + per, a.chunks);
    auto at = [&](int j) __attribute__((always_inline)) {
        return ((int64_t)b * a.chunks + (BACK ? a.chunks - 1 - j : j)) * a.n + c;
    };
    // (read before anything is written: the state that there is may be where the last one goes)
    const float start = there && a.carry_in ? a.carry_in[(int64_t)b * a.n + c] : 0.f;
    float A = 1.f, H = 0.f;
    if (there)
        for (int j = first; j < end; ++j) {
            const float aj = a.A[at(j)];
            H = fmaf(aj, H, a.H[at(j)]);
            A *= aj;
        }
    if (w == 0) {  // the first run begins with the state that there is
        if (a.carry_in) H = fmaf(A, start, H);
        A = 0.f;
    }
    for (int span = 1; span < 64; span *= 2) {
        As[w][l] = A;
        Hs[w][l] = H;
        __syncthreads();
        if (w >= span) {
            H = fmaf(A, Hs[w - span][l], H);
            A *= As[w - span][l];
        }
        __syncthreads();
    }
    Hs[w][l] = H;
    __syncthreads();
    if (!there) return;
    H = w ? Hs[w - 1][l] : start;
    for (int j = first; j < end; ++j) {
        const float hj = a.H[at(j)], aj = a.A[at(j)];
        a.H[at(j)] = H;
        H = fmaf(aj, H, hj);
    }
    if (a.carry_out && w == 63) a.carry_out[(int64_t)b * a.n + c] = Hs[63][l];
}

int scan_validate(const dsattn_scan_desc *desc, const char *who)
{
    if (!desc) return fail(DSATTN_EINVAL, "%s: null descriptor", who);
    const dsattn_scan_desc &d = *desc;
    if (d.streams < 1 || d.frames < 1 || d.spatial < 1 || d.channels < 1)
        return fail(DSATTN_EINVAL, "%s: sizes must be positive", who);
    if (d.frames > 0x7fffffff - 2 * kStep) return fail(DSATTN_EINVAL, "%s: too many frames", who);
    const int64_t most = (int64_t)1 << 46, n = (int64_t)d.spatial * d.channels;
    if (n > most / d.streams || n * d.streams > most / d.frames) return fail(DSATTN_EINVAL, "%s: problem too large", who);
    if (d.mode < DSATTN_SCAN_SUM || d.mode > DSATTN_SCAN_NORM) return fail(DSATTN_EINVAL, "%s: unknown mode", who);
    if (d.io_dtype != DSATTN_F32 && d.io_dtype != DSATTN_BF16) return fail(DSATTN_EINVAL, "%s: unknown dtype", who);
    return DSATTN_OK;
}

// Channels of a lane: four bytes, or one 16-bit one where a frame is an odd number of them or two a lane would make less than
// 512 wavefronts (a lane's steps take twice the time then: 384 frames x 100 x 640 69 us, by ones 42).
int scan_lane(const dsattn_scan_desc &d)
{
    const int64_t n = (int64_t)d.spatial * d.channels;
    return d.io_dtype == DSATTN_BF16 && n % 2 == 0 && n * d.streams >= 512 * 128 ? 2 : 1;
}

// Chunks of a stream.  From 512 wavefronts on one pass keeps enough loads on their way; below, chunks read their inputs twice,
// but as many as make 4,096 wavefronts (2 x 16,384 x 1,280: 127 us with 2,048, 104, 101 with 8,192, 275 before), of 32 frames
// or more (1 x 255 x 640, bf16: 37 us in one chunk, 18.5).
void scan_chunks(const dsattn_scan_desc &d, int32_t &chunk, int32_t &chunks)
{
    const int64_t n = (int64_t)d.spatial * d.channels, lanes = (n + scan_lane(d) - 1) / scan_lane(d);
    const int64_t waves = std::max<int64_t>(1, (lanes + 63) / 64 * d.streams);
    const int64_t want = waves >= 512 ? 1 : std::min<int64_t>(4096 / waves, d.frames / 32);
    chunk = d.frames;
    chunks = 1;
    if (want >= 4) {
        chunk = (int32_t)(((d.frames + want - 1) / want + kStep - 1) / kStep * kStep);
        chunks = (int32_t)(((int64_t)d.frames + chunk - 1) / chunk);
    }
}

size_t scan_bytes(const dsattn_scan_desc &d)
{
    int32_t chunk, chunks;
    scan_chunks(d, chunk, chunks);
    return chunks == 1 ? 0 : (size_t)d.streams * chunks * d.spatial * d.channels * 2 * sizeof(float);
}

enum { kPartsPass, kRunPass, kBackPartsPass, kBackPass };

// (two channels a lane are 512 wavefronts or more, which are in one chunk)
template <typename T, int V, int MODE>
const void *scan_kernel_of(int pass)
{
    if (pass == kRunPass) return (const void *)&scan_kernel<T, V, MODE, true>;
    if (pass == kBackPass) return (const void *)&scan_back_kernel<T, V, MODE>;
    if constexpr (V == 1) {
        if (pass == kPartsPass) return (const void *)&scan_kernel<T, V, MODE, false>;
        if (pass == kBackPartsPass) return (const void *)&scan_back_parts_kernel<T, V>;
    }
    return nullptr;
}
// One pass over many channels: eight bytes a lane (384 frames x 640 x 640, bf16, 4.7 TB/s instead of 4.45).
const void *scan_wide_of(const dsattn_scan_desc &d)
{
    if (d.io_dtype == DSATTN_F32) {
        switch (d.mode) {
        case DSATTN_SCAN_MEAN: return (const void *)&scan_kernel<float, 2, DSATTN_SCAN_MEAN, true>;
        case DSATTN_SCAN_NORM: return (const void *)&scan_kernel<float, 2, DSATTN_SCAN_NORM, true>;
        default: return (const void *)&scan_kernel<float, 2, DSATTN_SCAN_SUM, true>;
        }
    }
    switch (d.mode) {
    case DSATTN_SCAN_MEAN: return (const void *)&scan_kernel<__bf16, 4, DSATTN_SCAN_MEAN, true>;
    case DSATTN_SCAN_NORM: return (const void *)&scan_kernel<__bf16, 4, DSATTN_SCAN_NORM, true>;
    default: return (const void *)&scan_kernel<__bf16, 4, DSATTN_SCAN_SUM, true>;
    }
}
template <typename T, int V>
const void *scan_kernel_of(int mode, int pass)
{
    switch (mode) {
    case DSATTN_SCAN_MEAN: return scan_kernel_of<T, V, DSATTN_SCAN_MEAN>(pass);
    case DSATTN_SCAN_NORM: return scan_kernel_of<T, V, DSATTN_SCAN_NORM>(pass);
    default: return scan_kernel_of<T, V, DSATTN_SCAN_SUM>(pass);
    }
}

// Checks what both directions share and fills a; then the launches.
int scan_setup(const dsattn_scan_desc &d, const char *who, ScanArgs &a, void *workspace, size_t workspace_bytes)
{
    a.n = (int64_t)d.spatial * d.channels;
    a.B = d.streams;
    a.T = d.frames;
    a.steps = (d.frames + kStep - 1) / kStep;
    scan_chunks(d, a.chunk, a.chunks);
    const size_t need = scan_bytes(d);
    if (need && (!workspace || workspace_bytes < need)) return fail(DSATTN_EINVAL, "%s: workspace of %zu bytes needed", who, need);
    if ((uintptr_t)workspace & 15u) return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    a.A = need ? (float *)workspace : nullptr;
    a.H = need ? a.A + (int64_t)a.B * a.chunks * a.n : nullptr;
    const int64_t lanes = (a.n + scan_lane(d) - 1) / scan_lane(d);
    // (a launch has less than 2^32 threads, and less than 2^16 in the grid's other dimensions)
    if (a.B > 65535 || a.chunks > 65535 || (lanes + 255) / 256 * a.chunks * a.B > 0xffffff ||
        (a.chunks > 1 && (a.n + 15) / 16 * a.B > 0x3fffff))
        return fail(DSATTN_EUNSUPPORTED, "%s: too large for one launch", who);
    return DSATTN_OK;
}

int scan_launch(const dsattn_scan_desc &d, const char *who, ScanArgs &a, bool back, hipStream_t st)
{
    int V = scan_lane(d);
    const int parts = back ? kBackPartsPass : kPartsPass, run = back ? kBackPass : kRunPass;
    auto fn = [&](int pass) {
        return d.io_dtype == DSATTN_F32 ? scan_kernel_of<float, 1>(d.mode, pass)
               : V == 2                 ? scan_kernel_of<__bf16, 2>(d.mode, pass)
                                        : scan_kernel_of<__bf16, 1>(d.mode, pass);
    };
    const void *runner = fn(run);
    const int wide = 2 * (d.io_dtype == DSATTN_F32 ? 1 : 2);
    if (!back && a.chunks == 1 && a.n % wide == 0 && a.n / wide * a.B >= 64 * 1024) {
        V = wide;
        runner = scan_wide_of(d);
    }
    const dim3 grid((unsigned)(((a.n + V - 1) / V + 255) / 256), (unsigned)a.chunks, (unsigned)a.B);
    void *params[] = {&a};
    hipError_t e = hipSuccess;
    if (a.chunks > 1) {
        e = hipLaunchKernel(fn(parts), grid, dim3(256), params, 0, st);
        const void *join = back ? (const void *)&scan_join_kernel<true> : (const void *)&scan_join_kernel<false>;
        if (e == hipSuccess) e = hipLaunchKernel(join, dim3((unsigned)((a.n + 15) / 16), (unsigned)a.B), dim3(1024), params, 0, st);
    }
    if (e == hipSuccess) e = hipLaunchKernel(runner, grid, dim3(256), params, 0, st);
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
}

struct Span {
    const void *p;
    int64_t n;
};

// Outputs (the first `n_in_place` of which may be one of the first `n_taken` inputs) against inputs and each other.
int scan_overlaps(const char *who, const Span *in, int n_in, int n_taken, const Span *out, int n_out, int n_in_place, bool carry_in_place)
{
    for (int o = 0; o < n_out; ++o) {
        for (int i = 0; i < n_in; ++i) {
            const bool same = in[i].p == out[o].p && in[i].n == out[o].n &&
                              ((o < n_in_place && i < n_taken) || (carry_in_place && o == n_in_place && i == n_taken));
            if (!same && overlap(out[o].p, out[o].n, in[i].p, in[i].n)) return fail(DSATTN_EINVAL, "%s: an output overlaps an input", who);
        }
        for (int q = 0; q < o; ++q)
            if (overlap(out[o].p, out[o].n, out[q].p, out[q].n)) return fail(DSATTN_EINVAL, "%s: two outputs overlap", who);
    }
    return DSATTN_OK;
}

}  // namespace
}  // namespace dsattn

using namespace dsattn;

extern "C" {

int dsattn_gated_scan_workspace(const dsattn_scan_desc *desc, size_t *bytes)
{
    const int rc = scan_validate(desc, "dsattn_gated_scan_workspace");
    if (rc != DSATTN_OK) return rc;
    if (!bytes) return fail(DSATTN_EINVAL, "dsattn_gated_scan_workspace: null output");
    *bytes = scan_bytes(*desc);
    return DSATTN_OK;
}

int dsattn_gated_scan(const dsattn_scan_desc *desc, const int32_t *counts, const void *X, const void *G,
                      const float *start_state, void *Y, float *end_state, float *states, void *workspace,
                      size_t workspace_bytes, void *stream)
{
    const char *who = "dsattn_gated_scan";
    int rc = scan_validate(desc, who);
    if (rc != DSATTN_OK) return rc;
    const dsattn_scan_desc &d = *desc;
    if (!X || !G || !Y) return fail(DSATTN_EINVAL, "%s: null pointer", who);
    if (((uintptr_t)X | (uintptr_t)G | (uintptr_t)Y | (uintptr_t)start_state | (uintptr_t)end_state | (uintptr_t)states) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    if ((uintptr_t)counts & 3u) return fail(DSATTN_EINVAL, "%s: counts must be 4-byte aligned", who);
    ScanArgs a{};
    rc = scan_setup(d, who, a, workspace, workspace_bytes);
    if (rc != DSATTN_OK) return rc;
    const int64_t rows = (int64_t)d.streams * d.frames * a.n * (d.io_dtype == DSATTN_F32 ? 4 : 2), state = 4 * d.streams * a.n;
    const Span in[] = {{X, rows}, {G, rows}, {start_state, state}, {counts, 4 * (int64_t)d.streams}},
               out[] = {{Y, rows}, {end_state, state}, {states, state * a.steps}, {a.A, (int64_t)scan_bytes(d)}};
    rc = scan_overlaps(who, in, 4, 2, out, 4, 1, true);
    if (rc != DSATTN_OK) return rc;
    a.X = X;
    a.G = G;
    a.counts = counts;
    a.carry_in = start_state;
    a.carry_out = end_state;
    a.states_out = states;
    a.Y = Y;
    return scan_launch(d, who, a, false, (hipStream_t)stream);
}

int dsattn_gated_scan_backward(const dsattn_scan_desc *desc, const int32_t *counts, const void *X, const void *G,
                               const float *states, const void *dY, const float *dend_state, void *dX, void *dG,
                               float *dstart_state, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "dsattn_gated_scan_backward";
    int rc = scan_validate(desc, who);
    if (rc != DSATTN_OK) return rc;
    const dsattn_scan_desc &d = *desc;
    if (!X || !G || !states || !dY || !dX || !dG) return fail(DSATTN_EINVAL, "%s: null pointer", who);
    if (((uintptr_t)X | (uintptr_t)G | (uintptr_t)dY | (uintptr_t)dX | (uintptr_t)dG | (uintptr_t)states | (uintptr_t)dend_state |
         (uintptr_t)dstart_state) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    if ((uintptr_t)counts & 3u) return fail(DSATTN_EINVAL, "%s: counts must be 4-byte aligned", who);
    ScanArgs a{};
    rc = scan_setup(d, who, a, workspace, workspace_bytes);
    if (rc != DSATTN_OK) return rc;
    const int64_t rows = (int64_t)d.streams * d.frames * a.n * (d.io_dtype == DSATTN_F32 ? 4 : 2), state = 4 * d.streams * a.n;
    const Span in[] = {{X, rows}, {G, rows}, {dY, rows}, {dend_state, state}, {states, state * a.steps}, {counts, 4 * (int64_t)d.streams}},
               out[] = {{dX, rows}, {dG, rows}, {dstart_state, state}, {a.A, (int64_t)scan_bytes(d)}};
    rc = scan_overlaps(who, in, 6, 3, out, 4, 2, true);
    if (rc != DSATTN_OK) return rc;
    a.X = X;
    a.G = G;
    a.dY = dY;
    a.counts = counts;
    a.states_in = states;
    a.carry_in = dend_state;
    a.carry_out = dstart_state;
    a.Y = dX;
    a.dG = dG;
    return scan_launch(d, who, a, true, (hipStream_t)stream);
}

}  // extern "C"
