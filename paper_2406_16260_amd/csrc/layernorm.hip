// Layer norm with the residual's addition and its backward pass (dsattn_layernorm, dsattn_layernorm_backward).
//
//   s = x + r,  n = (s - mean s) * rsqrt(var s + eps),  y = n * gamma + beta,  optionally y / scale in 8 bits
//   e = dy * gamma,  dx = rsqrt(var s + eps) * (e - mean e - n * mean(e n)) + dsum,  dgamma = sum dy n,  dbeta = sum dy
//
// Bound by memory: a row stays in registers from its only read to its output, in L lanes with NV pieces of V numbers each.
// The mean is taken off twice, the second time that of the differences: what the first left of it by rounding (a row whose
// mean is 1,000 times its spread would lose ten bits of the spread to that) is gone, and the variance comes with it.
// us and TB/s (a large copy 5.1):
//   368,640 x 1,280, bf16, residual and sum         656-670 5.75
//   40,960 x 640, bf16, residual, all gradients     59.6    4.4, of which the joining kernel is 4.3 us
//   368,640 x 1,280, the same                       968     4.9
//   24,591 x 1,863, bf16, residual, then all gradients   75.5 and 105, the floors 72 and 90 (pieces of one number: 225 and 307)
//   40 x 1,280                                      6.9, of which 4.3 are the host's marshalling and 2.6 its launch
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "dsattn.h"
#include "plan.h"
#include "rows.h"

namespace dsattn {
namespace {

struct LnArgs {
    const void *X, *R;
    const float *gamma, *beta;
    void *S, *Y;
    float *scales;
    int64_t rows;
    int32_t C;
    float eps;
};

struct LnBackArgs {
    const void *X, *R, *dY, *dS;
    const float *gamma;
    void *dX;
    float *dgamma, *dbeta;  // a workgroup's sums of dy n and of dy go to these and `part` on from those of the one before, or null
    int64_t part;
    struct RowStats *stats;  // long rows only
    int64_t rows;
    int32_t C;
    float eps;
};

// n = ((s * unit - mean) * gain - rest) * rstd, and 1 / sqrt(var + eps) = unit * gain * rstd.  unit is 1, or 2^-75 for a row
// whose squares are beyond fp32's numbers (2^20 numbers of up to 2^53 stay within them then); gain is 1, or 2^100 for one whose
// differences have squares below 2^-100 (and eps far less): both exact, so that rows of every size are normalised alike.
struct RowStats {
    float unit, gain, mean, rest, rstd;
    __device__ __forceinline__ float norm(float s) const
    {
#pragma clang fp contract(off)
        return ((s * unit - mean) * gain - rest) * rstd;
    }
    // (one after the other: their product may be infinite where d is 0)
    __device__ __forceinline__ float slope(float d) const { return d * rstd * gain * unit; }
};

// Sums of N numbers over the L lanes of a row; part: LDS of a workgroup, for rows of several wavefronts.
template <int L, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*part)[N])
{
#pragma unroll
    for (int w = 1; w < (L < 64 ? L : 64); w *= 2)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], w);
    if constexpr (L > 64) {
        __syncthreads();  // the sums before have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) part[threadIdx.x >> 6][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = part[0][k];
#pragma unroll
            for (int w = 1; w < L / 64; ++w) v[k] += part[w][k];
        }
    }
}

constexpr float kLargest = 0x1.fffffep127f;

// each(f) calls f(s) for the lane's numbers of the row, sums(v) adds v over the row's lanes: whether another turn is needed
// depends on sums only, which all lanes of a row have.
// Means are those of numbers times 2^-21, whose sums are within fp32's range (what that takes of the mean of numbers below 2^-105 is
// part of the rest; differences as small as that have a gain, or an eps that is far more).  Where what the mean is off by, the rest,
// is more than a quarter of the spread, it is put right by that and the turn taken again: the mean of a row of equal numbers is then
// that number itself, its variance 0, and that of numbers which differ in their last bits loses no more to the rest's square
// than it has.  Only then are the squares asked whether they are within range: eps is lost beside a variance in `unit`s
// (1e-6 * 2^-150), which has to be that of numbers that do differ.
template <typename Each, typename Sums>
__device__ __forceinline__ RowStats row_stats(int C, float eps, Each each, Sums sums)
{
    // (mean and rest are rounded before they are used: one product and difference without that in some lanes only, and rows of
    // equal numbers would not come to 0)
#pragma clang fp contract(off)
    RowStats t{1.f, 1.f, 0.f, 0.f, 0.f};
    const float inv = 1.f / (float)C;
    float v[2] = {0.f, 0.f}, var;
    each([&](float s) __attribute__((always_inline)) { v[0] = fmaf(s, 0x1p-21f, v[0]); });
    sums(v);
    t.mean = fminf(fmaxf(v[0] * inv * 0x1p21f, -kLargest), kLargest);
    for (int better = 0;;) {
        v[0] = v[1] = 0.f;
        each([&](float s) __attribute__((always_inline)) {
            const float d = (s * t.unit - t.mean) * t.gain;
            v[0] = fmaf(d, 0x1p-21f, v[0]);
            v[1] = fmaf(d, d, v[1]);
        });
        sums(v);
        t.rest = v[0] * inv * 0x1p21f;
        const float square = v[1] * inv;
        var = fmaf(-t.rest, t.rest, square);
        const bool beyond = !(v[1] < INFINITY), off = var < 0.9375f * square;
        if (__builtin_expect(v[1] >= 0x1p-100f && !beyond && !off, 1)) break;
        if (better < 3 && (beyond || off)) {
            const float mean = t.mean + t.rest * (t.gain == 1.f ? 1.f : 0x1p-100f);
            if (mean != t.mean && fabsf(mean) < INFINITY) {
                t.mean = mean;
                ++better;
                continue;
            }
        }
        if (t.unit != 1.f || t.gain != 1.f) break;
        if (beyond) {
            t.unit = 0x1p-75f;
            t.mean *= t.unit;
        } else if (eps < 0x1p-80f && v[1] < 0x1p-100f) {
            t.gain = 0x1p100f;
        } else {
            break;
        }
        better = 0;
    }
    // (var is not below 0 but by rounding; a NaN stays)
    const float g = t.unit * t.gain;
    t.rstd = 1.f / sqrtf((var < 0.f ? 0.f : var) + eps * g * g);
    return t;
}

// A row is pieces of V numbers; a lane has every L-th of them, NV at most, of which all but the last are there in every lane.
// ODD: V does not divide the row, whose last piece then begins where it ends with the row, V - 1 numbers at most of the one before
// in it (`skip`, which sums leave out, and which both lanes write alike), and no piece is aligned but to a number: memory takes
// 16 bytes from there all the same.  (Pieces of the 4, 2 or 1 numbers that divide the row instead: 30,000 x 1,284 in bf16 65 us
// against 56, 50,000 x 250 20 against 17, 20,001 x 2,049 202 against 84, its gradients 408 against 116.)
template <typename T, int V, int L, int NV, bool ODD>
struct Row {
    typedef T Piece __attribute__((ext_vector_type(V), aligned(ODD ? sizeof(T) : sizeof(T) * V)));
    typedef float Floats __attribute__((ext_vector_type(V)));
    typedef float FloatsThere __attribute__((ext_vector_type(V), aligned(ODD ? sizeof(float) : sizeof(float) * V)));
    int c[NV], skip;
    bool in;  // the last piece
    __device__ __forceinline__ Row(int lane, int C)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) c[i] = (lane + i * L) * V;
        in = c[NV - 1] < C;
        skip = 0;
        if constexpr (ODD) {
            const int from = min(c[NV - 1], C - V);
            skip = c[NV - 1] - from;
            c[NV - 1] = from;
        }
    }
    __device__ __forceinline__ bool has(int i) const { return i < NV - 1 || in; }
    // f(piece, element) for each number that is the lane's own
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (has(i))
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (!ODD || i < NV - 1 || e >= skip) f(i, e);
    }
    __device__ __forceinline__ void load(const T *row, Piece (&x)[NV]) const
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (has(i)) x[i] = *(const Piece *)(row + c[i]);
    }
    __device__ __forceinline__ void load_floats(const float *row, Floats (&x)[NV]) const
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (has(i)) x[i] = *(const FloatsThere *)(row + c[i]);
    }
    // x + r in fp32; 0 behind the row's end
    __device__ __forceinline__ void load_sum(const void *X, const void *R, int64_t base, Floats (&s)[NV]) const
    {
        Piece x[NV], r[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            x[i] = Piece{};
            r[i] = -Piece{};  // (-0, which leaves every x as it is)
            if (!has(i)) continue;
            x[i] = *(const Piece *)((const T *)X + base + c[i]);
            if (R) r[i] = *(const Piece *)((const T *)R + base + c[i]);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) s[i][e] = (float)x[i][e] + (float)r[i][e];
    }
};

template <typename T, int V, int L, int NV, bool E8, bool ODD>
__global__ __launch_bounds__(L <= 256 ? 256 : L) void ln_vec_kernel(const LnArgs a)
{
    using Pieces = Row<T, V, L, NV, ODD>;
    using Piece = typename Pieces::Piece;
    using Floats = typename Pieces::Floats;
    constexpr int THREADS = L <= 256 ? 256 : L, NW = L > 64 ? L / 64 : 1;
    __shared__ float part[NW][2];
    const int64_t row = (int64_t)blockIdx.x * (THREADS / L) + threadIdx.x / L;
    const int C = a.C, lane = threadIdx.x % L;
    const Pieces mine(lane, C);
    const bool there = row < a.rows;
    const int64_t base = (there ? row : a.rows - 1) * C;
    Floats s[NV];
    mine.load_sum(a.X, a.R, base, s);
    Floats g[NV], b[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        g[i] = Floats{} + 1.f;
        b[i] = Floats{};
    }
    if (a.gamma) mine.load_floats(a.gamma, g);
    if (a.beta) mine.load_floats(a.beta, b);
    const RowStats t = row_stats(
        C, a.eps,
        [&](auto f) __attribute__((always_inline)) { mine.each([&](int i, int e) __attribute__((always_inline)) { f(s[i][e]); }); },
        [&](float (&v)[2]) __attribute__((always_inline)) { row_sums<L, 2>(v, part); });
    Floats y[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) y[i][e] = fmaf(t.norm(s[i][e]), g[i][e], b[i][e]);
    float inv = 1.f;
    if constexpr (E8) {
        float top = 0.f;
        mine.each([&](int i, int e) __attribute__((always_inline)) { top = max_or_nan(top, fabsf(y[i][e])); });
#pragma unroll
        for (int w = 1; w < (L < 64 ? L : 64); w *= 2) top = max_or_nan(top, __shfl_xor(top, w));
        if constexpr (L > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][0] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NW; ++w) top = max_or_nan(top, part[w][0]);
        }
        float scale = top / 448.f;
        scale = scale < 0x1p-126f ? 0x1p-126f : scale;  // (a NaN stays)
        if (there && lane == 0) a.scales[row] = scale;
        inv = 1.f / scale;
    }
    if (!there) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (!mine.has(i)) continue;
        const int64_t at = base + mine.c[i];
        if (a.S) {
            Piece p;
#pragma unroll
            for (int e = 0; e < V; ++e) p[e] = (T)s[i][e];
            *(Piece *)((T *)a.S + at) = p;
        }
        if constexpr (E8) {
            typedef int Words __attribute__((ext_vector_type(V / 4 ? V / 4 : 1), aligned(ODD ? 1 : V)));
            uint8_t *to = (uint8_t *)a.Y + at;
            if constexpr (V % 4 == 0) {
                Words w;
#pragma unroll
                for (int q = 0; q < V / 4; ++q) {
                    w[q] = __builtin_amdgcn_cvt_pk_fp8_f32(y[i][4 * q] * inv, y[i][4 * q + 1] * inv, 0, false);
                    w[q] = __builtin_amdgcn_cvt_pk_fp8_f32(y[i][4 * q + 2] * inv, y[i][4 * q + 3] * inv, w[q], true);
                }
                *(Words *)to = w;
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) to[e] = to_e4m3(y[i][e] * inv);
            }
        } else {
            Piece p;
#pragma unroll
            for (int e = 0; e < V; ++e) p[e] = (T)y[i][e];
            *(Piece *)((T *)a.Y + at) = p;
        }
    }
}

// A workgroup's loop over a row that is longer than its registers: f(column, x + r).
template <typename T, typename F>
__device__ __forceinline__ void long_row(const T *x, const T *r, int C, F f)
{
    for (int c = threadIdx.x; c < C; c += 256) f(c, (float)x[c] + (r ? (float)r[c] : -0.f));
}

template <typename T>
__device__ __forceinline__ RowStats long_row_stats(const T *x, const T *r, int C, float eps, float (*part)[2])
{
    return row_stats(
        C, eps,
        [&](auto f) __attribute__((always_inline)) { long_row(x, r, C, [&](int, float s) __attribute__((always_inline)) { f(s); }); },
        [&](float (&v)[2]) __attribute__((always_inline)) { row_sums<256, 2>(v, part); });
}

template <typename T, bool E8>
__global__ __launch_bounds__(256) void ln_row_kernel(const LnArgs a)
{
    __shared__ float part[4][2];
    const int64_t row = blockIdx.x;
    const int C = a.C;
    const T *x = (const T *)a.X + row * C, *r = a.R ? (const T *)a.R + row * C : nullptr;
    const RowStats t = long_row_stats(x, r, C, a.eps, part);
    auto y_of = [&](int c, float s) __attribute__((always_inline)) {
        return fmaf(t.norm(s), a.gamma ? a.gamma[c] : 1.f, a.beta ? a.beta[c] : 0.f);
    };
    float inv = 1.f;
    if constexpr (E8) {
        float top = 0.f;
        long_row(x, r, C, [&](int c, float s) __attribute__((always_inline)) { top = max_or_nan(top, fabsf(y_of(c, s))); });
        for (int w = 32; w > 0; w >>= 1) top = max_or_nan(top, __shfl_xor(top, w));
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][0] = top;
        __syncthreads();
        top = max_or_nan(max_or_nan(part[0][0], part[1][0]), max_or_nan(part[2][0], part[3][0]));
        float scale = top / 448.f;
        scale = scale < 0x1p-126f ? 0x1p-126f : scale;
        if (threadIdx.x == 0) a.scales[row] = scale;
        inv = 1.f / scale;
    }
    // (each number is read before its place is written, by the same thread: outputs may be the inputs)
    long_row(x, r, C, [&](int c, float s) __attribute__((always_inline)) {
        const float y = y_of(c, s) * inv;
        if (a.S) ((T *)a.S)[row * C + c] = (T)s;
        if constexpr (E8)
            ((uint8_t *)a.Y)[row * C + c] = to_e4m3(y);
        else
            ((T *)a.Y)[row * C + c] = (T)y;
    });
}

// A workgroup takes rows blockIdx.x, + gridDim.x, .. (times the rows that it has at once); a lane has the same channels of all of
// them, adds up their dgamma and dbeta in registers, and the workgroup's sums go to memory for
// ln_join_kernel, or to the result where there is one workgroup only: no atomics, one order.
template <typename T, int V, int L, int NV, bool ODD>
__global__ __launch_bounds__(L <= 256 ? 256 : L) void ln_back_vec_kernel(const LnBackArgs a)
{
    using Pieces = Row<T, V, L, NV, ODD>;
    using Piece = typename Pieces::Piece;
    using Floats = typename Pieces::Floats;
    constexpr int THREADS = L <= 256 ? 256 : L, NW = L > 64 ? L / 64 : 1, PER = THREADS / L;
    __shared__ float part[NW][2];
    const int C = a.C, turn = threadIdx.x / L;
    const Pieces mine(threadIdx.x % L, C);
    const float inv = 1.f / (float)C;
    Floats g[NV], dg[NV], db[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        g[i] = Floats{} + 1.f;
        dg[i] = db[i] = Floats{};
    }
    if (a.gamma) mine.load_floats(a.gamma, g);
    for (int64_t first = (int64_t)blockIdx.x * PER; first < a.rows; first += (int64_t)gridDim.x * PER) {
        const bool there = first + turn < a.rows;
        const int64_t base = (there ? first + turn : a.rows - 1) * C;
        Piece dyp[NV], dsp[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) dyp[i] = dsp[i] = Piece{};
        mine.load((const T *)a.dY + base, dyp);
        if (a.dS) mine.load((const T *)a.dS + base, dsp);
        Floats s[NV];
        mine.load_sum(a.X, a.R, base, s);
        const RowStats t = row_stats(
            C, a.eps,
            [&](auto f) __attribute__((always_inline)) { mine.each([&](int i, int e) __attribute__((always_inline)) { f(s[i][e]); }); },
            [&](float (&v)[2]) __attribute__((always_inline)) { row_sums<L, 2>(v, part); });
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) s[i][e] = t.norm(s[i][e]);
        mine.each([&](int i, int e) __attribute__((always_inline)) {  // (behind the row's end dy is 0, but n may be infinite)
            const float de = (float)dyp[i][e] * g[i][e];
            v[0] += de;
            v[1] = fmaf(de, s[i][e], v[1]);
        });
        row_sums<L, 2>(v, part);
        if (!there) continue;  // (rows of several wavefronts: PER is 1, and all of the workgroup are there)
        const float m0 = v[0] * inv, m1 = v[1] * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!mine.has(i)) continue;
            Piece p;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float dy = (float)dyp[i][e], n = s[i][e];
                dg[i][e] = fmaf(dy, n, dg[i][e]);
                db[i][e] += dy;
                const float dx = t.slope(fmaf(dy, g[i][e], -m0) - n * m1);
                p[e] = (T)(a.dS ? dx + (float)dsp[i][e] : dx);
            }
            *(Piece *)((T *)a.dX + base + mine.c[i]) = p;
        }
    }
    if (!a.dgamma && !a.dbeta) return;
    typedef float Loose __attribute__((ext_vector_type(V), aligned(sizeof(float))));  // (as much as the caller's are aligned)
    const int64_t part_at = (int64_t)blockIdx.x * a.part;
    if constexpr (PER > 1) {
        __shared__ Floats sums[256];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                __syncthreads();
                sums[threadIdx.x] = k ? db[i] : dg[i];
                __syncthreads();
                float *to = k ? a.dbeta : a.dgamma;
                if (to && turn == 0 && mine.has(i)) {
                    Floats v = sums[threadIdx.x];
#pragma unroll
                    for (int w = 1; w < PER; ++w) v += sums[threadIdx.x + w * L];
                    *(Loose *)(to + part_at + mine.c[i]) = v;
                }
            }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!mine.has(i)) continue;
            if (a.dgamma) *(Loose *)(a.dgamma + part_at + mine.c[i]) = dg[i];
            if (a.dbeta) *(Loose *)(a.dbeta + part_at + mine.c[i]) = db[i];
        }
    }
}

// Longer rows: a workgroup a row for dX, which leaves the row's mean and deviation, and a thread a column of every 64 rows
// for the sums.
template <typename T>
__global__ __launch_bounds__(256) void ln_back_row_kernel(const LnBackArgs a)
{
    __shared__ float part[4][2];
    const int64_t row = blockIdx.x;
    const int C = a.C;
    const T *x = (const T *)a.X + row * C, *r = a.R ? (const T *)a.R + row * C : nullptr;
    const T *dy = (const T *)a.dY + row * C, *ds = a.dS ? (const T *)a.dS + row * C : nullptr;
    const RowStats t = long_row_stats(x, r, C, a.eps, part);
    float v[2] = {0.f, 0.f};
    long_row(x, r, C, [&](int c, float s) __attribute__((always_inline)) {
        const float e = (float)dy[c] * (a.gamma ? a.gamma[c] : 1.f);
        v[0] += e;
        v[1] = fmaf(e, t.norm(s), v[1]);
    });
    row_sums<256, 2>(v, part);
    const float inv = 1.f / (float)C, m0 = v[0] * inv, m1 = v[1] * inv;
    if (threadIdx.x == 0 && a.stats) a.stats[row] = t;
    long_row(x, r, C, [&](int c, float s) __attribute__((always_inline)) {
        const float e = (float)dy[c] * (a.gamma ? a.gamma[c] : 1.f);
        const float dx = t.slope(e - m0 - t.norm(s) * m1);
        ((T *)a.dX)[row * C + c] = (T)(ds ? dx + (float)ds[c] : dx);
    });
}

constexpr int kLongRows = 64;  // rows of a partial sum
template <typename T>
__global__ __launch_bounds__(256) void ln_back_col_kernel(const LnBackArgs a)
{
    const int C = a.C, c = (int)blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    const int64_t first = (int64_t)blockIdx.y * kLongRows, end = min(first + kLongRows, a.rows);
    float dg = 0.f, db = 0.f;
    for (int64_t row = first; row < end; ++row) {
        const int64_t i = row * C + c;
        const float s = (float)((const T *)a.X)[i] + (a.R ? (float)((const T *)a.R)[i] : -0.f), dy = (float)((const T *)a.dY)[i];
        dg = fmaf(dy, a.stats[row].norm(s), dg);
        db += dy;
    }
    a.dgamma[blockIdx.y * a.part + c] = dg;
    a.dbeta[blockIdx.y * a.part + c] = db;
}

// The partial sums of `groups` workgroups added up: 16 columns a workgroup, 64 threads to each.
__global__ __launch_bounds__(1024) void ln_join_kernel(const float *partial, int groups, int C, float *dgamma, float *dbeta)
{
    __shared__ float sums[64][17];
    const int c = (int)blockIdx.x * 16 + (threadIdx.x & 15), g0 = threadIdx.x >> 4, which = blockIdx.y;
    float *to = which ? dbeta : dgamma;
    if (!to) return;
    float v = 0.f;
    if (c < C) {
        const float *from = partial + (int64_t)which * C + c;
#pragma unroll 4
        for (int g = g0; g < groups; g += 64) v += from[(int64_t)g * 2 * C];
    }
    sums[g0][threadIdx.x & 15] = v;
    __syncthreads();
    for (int w = 32; w > 0; w >>= 1) {
        if (g0 < w) sums[g0][threadIdx.x & 15] += sums[g0 + w][threadIdx.x & 15];
        __syncthreads();
    }
    if (g0 == 0 && c < C) to[c] = sums[0][threadIdx.x & 15];
}

// The kernel of a shape: pieces of 16 bytes (of one number for rows shorter than that), and the fewest lanes that hold the row in
// four pieces each (1,024 lanes: in two), so that only the last piece of a lane may be missing; null: longer.  The backward pass
// holds a row four times, which leaves 1,024 lanes too few registers.
struct LnKernel {
    const void *fn;
    int lanes;
};
template <typename K, int L>
const void *ln_of(int nv)
{
    if constexpr (L == 64)
        if (nv == 1) return K::template of<L, 1>();
    if constexpr (L != 512)  // (what 512 lanes have begins where 256 end, at three pieces each)
        if (nv <= 2) return K::template of<L, 2>();
    if constexpr (L < 1024) {
        if (nv == 3) return K::template of<L, 3>();
        if (nv == 4) return K::template of<L, 4>();
    }
    return nullptr;
}
template <typename K>
LnKernel ln_pick_of(int C)
{
    const int pieces = (C + K::V - 1) / K::V;
    if (pieces <= 8) return {K::template of<8, 1>(), 8};
    if (pieces <= 16) return {K::template of<16, 1>(), 16};
    if (pieces <= 32) return {K::template of<32, 1>(), 32};
    if (pieces <= 256) return {ln_of<K, 64>((pieces + 63) / 64), 64};
    if (pieces <= 1024) return {ln_of<K, 256>((pieces + 255) / 256), 256};
    if (pieces <= 2048) return {ln_of<K, K::WIDE>((pieces + K::WIDE - 1) / K::WIDE), K::WIDE};
    return {nullptr, 0};
}
template <typename T, int VV, bool E8, bool ODD>
struct LnForward {
    static constexpr int V = VV, WIDE = 1024;
    template <int L, int NV>
    static const void *of() { return (const void *)&ln_vec_kernel<T, V, L, NV, E8, ODD>; }
};
template <typename T, int VV, bool ODD>
struct LnBackward {
    static constexpr int V = VV, WIDE = 512;
    template <int L, int NV>
    static const void *of() { return (const void *)&ln_back_vec_kernel<T, V, L, NV, ODD>; }
};
template <typename T, bool E8>
LnKernel ln_pick(int C)
{
    constexpr int V = 16 / (int)sizeof(T);
    if (C < V) return {LnForward<T, 1, E8, false>::template of<8, 1>(), 8};
    return C % V == 0 ? ln_pick_of<LnForward<T, V, E8, false>>(C) : ln_pick_of<LnForward<T, V, E8, true>>(C);
}
template <typename T>
LnKernel ln_back_pick(int C)
{
    constexpr int V = 16 / (int)sizeof(T);
    if (C < V) return {LnBackward<T, 1, false>::template of<8, 1>(), 8};
    return C % V == 0 ? ln_pick_of<LnBackward<T, V, false>>(C) : ln_pick_of<LnBackward<T, V, true>>(C);
}

int ln_validate(const dsattn_ln_desc *desc, const char *who)
{
    if (!desc) return fail(DSATTN_EINVAL, "%s: null descriptor", who);
    const dsattn_ln_desc &d = *desc;
    if (d.rows < 1 || d.rows > 0x7fffffffLL || d.channels < 1 || d.channels > (1 << 20))
        return fail(DSATTN_EINVAL, "%s: rows outside [1, 2^31 - 1] or channels outside [1, 2^20]", who);
    if (d.io_dtype != DSATTN_F32 && d.io_dtype != DSATTN_BF16)
        return fail(DSATTN_EINVAL, "%s: unknown input dtype", who);
    if (d.out_dtype != d.io_dtype && d.out_dtype != DSATTN_E4M3)
        return fail(DSATTN_EINVAL, "%s: the output is of the input's dtype or in 8 bits", who);
    if (!(d.eps >= 0.f) || std::isinf(d.eps)) return fail(DSATTN_EINVAL, "%s: eps must be finite and >= 0", who);
    return DSATTN_OK;
}

// How a backward pass runs: workgroups of the sums, and whether its rows are long ones.
struct LnBackLaunch {
    const void *fn;
    int threads, groups;
    size_t bytes;
};
LnBackLaunch ln_back_launch(const dsattn_ln_desc &d)
{
    const LnKernel k = d.io_dtype == DSATTN_F32 ? ln_back_pick<float>(d.channels) : ln_back_pick<__bf16>(d.channels);
    LnBackLaunch l{k.fn, 256, 0, 0};
    if (k.fn) {
        const int per = k.lanes <= 256 ? 256 / k.lanes : 1;
        l.threads = k.lanes <= 256 ? 256 : k.lanes;
        // Few rows take turns in one workgroup, which needs no join after it.  us of a call with and without, bf16:
        // 8 x 320 (two turns) 10.2 7.3, 16 x 320 (four) 10.2 7.7, 8 x 1,280 (two) 10.1 7.8, 16 x 1,280 (four) 10.1 12.1,
        // 4 x 2,560 (four) 9.9 10.9.  (Turns are short where rows are.)
        const int turns = d.channels * (d.io_dtype == DSATTN_F32 ? 4 : 2) <= 1024 ? 4 : 2;
        // Else 1,024 workgroups (40,960 x 640 41 us, of 512 50), but 512 where those have four turns or less: what they leave for
        // the join is more than what they read (4,484 x 824 16.0 us with 1,024, 14.6, 2,000 x 4,096 29.8 and 25.6).
        const int64_t all = (d.rows + per - 1) / per;
        l.groups = d.rows <= turns * per ? 1 : (int)std::min<int64_t>(all, k.lanes <= 256 && all > 4 * 512 ? 1024 : 512);
    } else {
        l.groups = (int)((d.rows + kLongRows - 1) / kLongRows);
    }
    l.bytes = (size_t)l.groups * 2 * (size_t)d.channels * sizeof(float);
    if (!k.fn) l.bytes += (size_t)d.rows * sizeof(RowStats);
    return l;
}

}  // namespace
}  // namespace dsattn

using namespace dsattn;

extern "C" {

int dsattn_layernorm(const dsattn_ln_desc *desc, const void *X, const void *residual, const float *gamma,
                     const float *beta, void *sum, void *Y, float *scales, void *stream)
{
    const char *who = "dsattn_layernorm";
    const int rc = ln_validate(desc, who);
    if (rc != DSATTN_OK) return rc;
    const dsattn_ln_desc &d = *desc;
    const bool e8 = d.out_dtype == DSATTN_E4M3;
    if (!X || !Y || (e8 && !scales)) return fail(DSATTN_EINVAL, "%s: null pointer", who);
    if (!e8 && scales) return fail(DSATTN_EINVAL, "%s: scales without an output in 8 bits", who);
    if (((uintptr_t)X | (uintptr_t)residual | (uintptr_t)gamma | (uintptr_t)beta | (uintptr_t)sum | (uintptr_t)Y) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    if ((uintptr_t)scales & 3u) return fail(DSATTN_EINVAL, "%s: scales must be 4-byte aligned", who);
    const int64_t n = d.rows * d.channels, in = n * (d.io_dtype == DSATTN_BF16 ? 2 : 4), cn = 4 * (int64_t)d.channels;
    const int64_t out = e8 ? n : in;
    const struct { const void *p; int64_t n; } inputs[] = {{X, in}, {residual, in}, {gamma, cn}, {beta, cn}},
                                               outputs[] = {{sum, in}, {Y, out}, {scales, 4 * d.rows}};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 4; ++i) {
            const bool same = i < 2 && outputs[o].p == inputs[i].p && (o == 0 || (o == 1 && !e8));
            if (!same && overlap(outputs[o].p, outputs[o].n, inputs[i].p, inputs[i].n))
                return fail(DSATTN_EINVAL, "%s: an output overlaps an input", who);
        }
        for (int q = 0; q < o; ++q)
            if (overlap(outputs[o].p, outputs[o].n, outputs[q].p, outputs[q].n))
                return fail(DSATTN_EINVAL, "%s: two outputs overlap", who);
    }
    const LnArgs a{X, residual, gamma, beta, sum, Y, scales, d.rows, d.channels, d.eps};
    const bool f32 = d.io_dtype == DSATTN_F32;
    const LnKernel k = f32 ? (e8 ? ln_pick<float, true>(d.channels) : ln_pick<float, false>(d.channels))
                           : (e8 ? ln_pick<__bf16, true>(d.channels) : ln_pick<__bf16, false>(d.channels));
    const void *fn = k.fn;
    unsigned groups = (unsigned)d.rows, threads = 256;
    if (fn) {
        const int per = k.lanes <= 256 ? 256 / k.lanes : 1;  // rows of a workgroup
        groups = (unsigned)((d.rows + per - 1) / per);
        threads = k.lanes <= 256 ? 256u : (unsigned)k.lanes;
    } else {
        fn = f32 ? (e8 ? (const void *)&ln_row_kernel<float, true> : (const void *)&ln_row_kernel<float, false>)
                 : (e8 ? (const void *)&ln_row_kernel<__bf16, true> : (const void *)&ln_row_kernel<__bf16, false>);
    }
    // (a launch has less than 2^32 threads)
    if ((uint64_t)groups * threads > 0xffffffffull)
        return fail(DSATTN_EUNSUPPORTED, "%s: too many rows for one launch", who);
    void *params[] = {(void *)&a};
    const hipError_t e = hipLaunchKernel(fn, dim3(groups), dim3(threads), params, 0, (hipStream_t)stream);
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
}

int dsattn_layernorm_backward_workspace(const dsattn_ln_desc *desc, size_t *bytes)
{
    const int rc = ln_validate(desc, "dsattn_layernorm_backward_workspace");
    if (rc != DSATTN_OK) return rc;
    if (!bytes) return fail(DSATTN_EINVAL, "dsattn_layernorm_backward_workspace: null output");
    *bytes = ln_back_launch(*desc).bytes;
    return DSATTN_OK;
}

int dsattn_layernorm_backward(const dsattn_ln_desc *desc, const void *X, const void *residual, const float *gamma,
                              const void *dY, const void *dsum, void *dX, float *dgamma, float *dbeta, void *workspace,
                              size_t workspace_bytes, void *stream)
{
    const char *who = "dsattn_layernorm_backward";
    const int rc = ln_validate(desc, who);
    if (rc != DSATTN_OK) return rc;
    const dsattn_ln_desc &d = *desc;
    if (d.out_dtype != d.io_dtype) return fail(DSATTN_EINVAL, "%s: gradients are of the input's dtype", who);
    if (!X || !dY || !dX) return fail(DSATTN_EINVAL, "%s: null pointer", who);
    if (((uintptr_t)X | (uintptr_t)residual | (uintptr_t)gamma | (uintptr_t)dY | (uintptr_t)dsum | (uintptr_t)dX |
         (uintptr_t)workspace) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    if (((uintptr_t)dgamma | (uintptr_t)dbeta) & 3u) return fail(DSATTN_EINVAL, "%s: gradients of weights must be 4-byte aligned", who);
    const LnBackLaunch l = ln_back_launch(d);
    const bool sums = dgamma || dbeta;
    if (sums && (!workspace || workspace_bytes < l.bytes)) return fail(DSATTN_EINVAL, "%s: workspace of %zu bytes needed", who, l.bytes);
    const int64_t n = d.rows * d.channels * (d.io_dtype == DSATTN_BF16 ? 2 : 4), cn = 4 * (int64_t)d.channels;
    const struct { const void *p; int64_t n; }
        inputs[] = {{X, n}, {residual, n}, {dY, n}, {dsum, n}, {gamma, cn}},
        outputs[] = {{dX, n}, {dgamma, cn}, {dbeta, cn}, {sums ? workspace : nullptr, (int64_t)l.bytes}};
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 5; ++i) {
            // (dX in the place of an input: not where rows are long and their columns are read again for the sums)
            const bool same = o == 0 && i < 4 && outputs[o].p == inputs[i].p && (l.fn || !sums || i == 3);
            if (!same && overlap(outputs[o].p, outputs[o].n, inputs[i].p, inputs[i].n))
                return fail(DSATTN_EINVAL, "%s: an output overlaps an input", who);
        }
        for (int q = 0; q < o; ++q)
            if (overlap(outputs[o].p, outputs[o].n, outputs[q].p, outputs[q].n))
                return fail(DSATTN_EINVAL, "%s: two outputs overlap", who);
    }
    const bool join = sums && (!l.fn || l.groups > 1);
    float *partial = (float *)workspace;
    LnBackArgs a{X, residual, dY, dsum, gamma, dX, join ? partial : dgamma, join ? partial + d.channels : dbeta,
                 2 * (int64_t)d.channels, nullptr, d.rows, d.channels, d.eps};
    const bool f32 = d.io_dtype == DSATTN_F32;
    const hipStream_t st = (hipStream_t)stream;
    void *params[] = {&a};
    hipError_t e;
    if (l.fn) {
        e = hipLaunchKernel(l.fn, dim3((unsigned)l.groups), dim3((unsigned)l.threads), params, 0, st);
    } else {
        if ((uint64_t)d.rows * 256 > 0xffffffffull || l.groups > 65535)
            return fail(DSATTN_EUNSUPPORTED, "%s: too many rows of this length", who);
        if (sums) a.stats = (RowStats *)((char *)workspace + (size_t)l.groups * 2 * (size_t)d.channels * sizeof(float));
        const void *fn = f32 ? (const void *)&ln_back_row_kernel<float> : (const void *)&ln_back_row_kernel<__bf16>;
        e = hipLaunchKernel(fn, dim3((unsigned)d.rows), dim3(256), params, 0, st);
        fn = f32 ? (const void *)&ln_back_col_kernel<float> : (const void *)&ln_back_col_kernel<__bf16>;
        if (e == hipSuccess && sums)
            e = hipLaunchKernel(fn, dim3((unsigned)(d.channels + 255) / 256, (unsigned)l.groups), dim3(256), params, 0, st);
    }
    if (e == hipSuccess && join) {
        int groups = l.groups, C = d.channels;
        void *args[] = {&partial, &groups, &C, &dgamma, &dbeta};
        e = hipLaunchKernel((const void *)&ln_join_kernel, dim3((unsigned)(C + 15) / 16, 2), dim3(1024), args, 0, st);
    }
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
}

}  // extern "C"
