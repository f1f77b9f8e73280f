// Root-mean-square normalisation with the residual's addition (dsattn_rmsnorm).
//
//   s = x + r,  y = s * rsqrt(mean(s^2) + eps) * gamma,  optionally y / scale in 8 bits
//
// Bound by memory: each number of x and r is read once, each of the sum and of y written once.  A row stays in
// registers between the sum of its squares and its output: L lanes have it, NV pieces of V numbers each, and a
// wavefront has 64 / L rows (L <= 64) or a workgroup one (L = 256 or 1,024).  The largest |y|, which a scale is
// made of, is max|s gamma| times the row's factor, and so comes with the sum of squares.
// 368,640 x 1,280 bf16 with residual and sum into 8 bits, 3.3 GB: 567 to 577 us, 5.8 TB/s (a large copy 5.1; a workgroup a row
// in two passes 1,755 us).  40 x 1,280: 7.0 us, of which 6 are the host's.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "dsattn.h"
#include "plan.h"
#include "rows.h"

namespace dsattn {
namespace {

struct RmsArgs {
    const void *X, *R;
    const float *gamma;
    void *S, *Y;
    float *scales;
    int64_t rows;
    int32_t C;
    float eps;
};

// A power of two that brings a row's squares into fp32's range, 1 where they are there (a row of ordinary size, and every one
// where eps is far above the squares that are lost).  Sums of squares below 2^-100 are of numbers below 2^-50 and times 2^100
// at least 2^-49 and below 2^50; one of 2^128 or more has a number beyond 2^54, and 2^20 squares of numbers below 2^53 fit.  The
// factor is exact, so that a row's result has the same error at every size, but for what it pushes below 2^-126: numbers
// below 2^-51 in a row of a norm of 2^64 or more.  (A sum that is infinite for an infinity stays so.)
__device__ __forceinline__ float row_unit(float ss, float eps)
{
    if (ss < 0x1p-100f && eps < 0x1p-80f) return 0x1p100f;
    return ss == INFINITY ? 0x1p-75f : 1.f;
}

// The scale of a row whose largest |s gamma| is top.
__device__ __forceinline__ float row_scale(float top, float rstd)
{
    const float s = top * rstd / 448.f;
    return s < 0x1p-126f ? 0x1p-126f : s;  // (a NaN stays)
}

// L lanes a row, NV pieces of V numbers a lane.
template <typename T, int V, int L, int NV, bool E8>
__global__ __launch_bounds__(L <= 256 ? 256 : L) void rms_vec_kernel(const RmsArgs a)
{
    typedef T Piece __attribute__((ext_vector_type(V)));
    typedef float Floats __attribute__((ext_vector_type(V)));
    constexpr int THREADS = L <= 256 ? 256 : L, NW = L / 64;  // wavefronts of a row
    const int64_t row = (int64_t)blockIdx.x * (THREADS / L) + threadIdx.x / L;
    const int C = a.C, at = (int)(threadIdx.x % L) * V;
    const bool there = row < a.rows;
    const int64_t base = (there ? row : a.rows - 1) * C;
    Piece x[NV], r[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = at + i * (L * V);
        x[i] = Piece{};
        r[i] = -Piece{};  // (-0, which leaves every x as it is)
        if (c < C) {
            x[i] = *(const Piece *)((const T *)a.X + base + c);
            if (a.R) r[i] = *(const Piece *)((const T *)a.R + base + c);
        }
    }
    Floats s[NV], g[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = at + i * (L * V);
        g[i] = Floats{} + 1.f;
        if (a.gamma && c < C) g[i] = *(const Floats *)(a.gamma + c);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) s[i][e] = (float)x[i][e] + (float)r[i][e];
    float ss, top;
    auto moments = [&](float unit) __attribute__((always_inline)) {
        ss = top = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float su = s[i][e] * unit;
                ss = fmaf(su, su, ss);
                if constexpr (E8) top = max_or_nan(top, fabsf(su * g[i][e]));
            }
#pragma unroll
        for (int w = 1; w < (L < 64 ? L : 64); w *= 2) {
            ss += __shfl_xor(ss, w);
            if constexpr (E8) top = max_or_nan(top, __shfl_xor(top, w));
        }
        if constexpr (L > 64) {
            __shared__ float part[2][NW];
            if ((threadIdx.x & 63) == 0) {
                part[0][threadIdx.x >> 6] = ss;
                part[1][threadIdx.x >> 6] = top;
            }
            __syncthreads();
            ss = part[0][0];
            top = part[1][0];
#pragma unroll
            for (int w = 1; w < NW; ++w) {
                ss += part[0][w];
                top = max_or_nan(top, part[1][w]);
            }
        }
    };
    moments(1.f);
    const float unit = row_unit(ss, a.eps);
    if (unit != 1.f) {  // (the same for all lanes of a row, which a workgroup's barrier is for)
        if constexpr (L > 64) __syncthreads();
        moments(unit);
    }
    const float rstd = 1.f / sqrtf(ss / (float)C + a.eps * unit * unit);
    const float scale = E8 ? row_scale(top, rstd) : 1.f, inv = 1.f / scale;  // (its product with rstd may overflow)
    if (!there) return;
    if (E8 && at == 0) a.scales[row] = scale;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = at + i * (L * V);
        if (c >= C) continue;
        if (a.S) {
            Piece t;
#pragma unroll
            for (int e = 0; e < V; ++e) t[e] = (T)s[i][e];
            *(Piece *)((T *)a.S + base + c) = t;
        }
        Floats y;
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = s[i][e] * unit * g[i][e] * rstd;
        if constexpr (E8) {
            uint8_t *to = (uint8_t *)a.Y + base + c;
            if constexpr (V % 4 == 0) {
                typedef int Words __attribute__((ext_vector_type(V / 4)));
                Words w;
#pragma unroll
                for (int q = 0; q < V / 4; ++q) {
                    w[q] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * q] * inv, y[4 * q + 1] * inv, 0, false);
                    w[q] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * q + 2] * inv, y[4 * q + 3] * inv, w[q], true);
                }
                *(Words *)to = w;
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) to[e] = to_e4m3(y[e] * inv);
            }
        } else {
            Piece t;
#pragma unroll
            for (int e = 0; e < V; ++e) t[e] = (T)y[e];
            *(Piece *)((T *)a.Y + base + c) = t;
        }
    }
}

// The kernel of a shape: pieces of as many numbers as divide the row, up to 16 bytes, and the fewest lanes that hold the row in
// four pieces each (eight of one or two numbers); null: longer than 1,024 lanes hold.
struct RmsKernel {
    const void *fn;
    int lanes;
};
template <typename T, int V, bool E8, int L>
const void *rms_kernel_of(int nv)
{
    if constexpr (L == 64)  // (with more lanes a row is longer than one piece each)
        if (nv == 1) return (const void *)&rms_vec_kernel<T, V, L, 1, E8>;
    switch (nv) {
    case 2: return (const void *)&rms_vec_kernel<T, V, L, 2, E8>;
    case 3: return (const void *)&rms_vec_kernel<T, V, L, 3, E8>;
    case 4: return (const void *)&rms_vec_kernel<T, V, L, 4, E8>;
    default: return nullptr;
    }
}
template <typename T, int V, bool E8>
RmsKernel rms_pick_of(int C)
{
    const int pieces = (C + V - 1) / V;
    if (pieces <= 8) return {(const void *)&rms_vec_kernel<T, V, 8, 1, E8>, 8};
    if (pieces <= 16) return {(const void *)&rms_vec_kernel<T, V, 16, 1, E8>, 16};
    if (pieces <= 32) return {(const void *)&rms_vec_kernel<T, V, 32, 1, E8>, 32};
    if (pieces <= 256) return {rms_kernel_of<T, V, E8, 64>((pieces + 63) / 64), 64};
    if (V <= 2 && pieces <= 512) return {(const void *)&rms_vec_kernel<T, V, 64, 8, E8>, 64};
    if (pieces <= 1024) return {rms_kernel_of<T, V, E8, 256>((pieces + 255) / 256), 256};
    if (V <= 2 && pieces <= 2048) return {(const void *)&rms_vec_kernel<T, V, 256, 8, E8>, 256};
    if (pieces <= 4096) return {rms_kernel_of<T, V, E8, 1024>((pieces + 1023) / 1024), 1024};
    return {nullptr, 0};
}
template <typename T, bool E8>
RmsKernel rms_pick(int C)
{
    if (sizeof(T) == 2 && C % 8 == 0) return rms_pick_of<T, 16 / (int)sizeof(T), E8>(C);
    return C % 4 == 0 ? rms_pick_of<T, 4, E8>(C) : C % 2 == 0 ? rms_pick_of<T, 2, E8>(C) : rms_pick_of<T, 1, E8>(C);
}

// Rows longer than that: a workgroup a row, two passes over it.
template <typename T, bool E8>
__global__ __launch_bounds__(256) void rms_row_kernel(const RmsArgs a)
{
    __shared__ float part[2][4];
    const int64_t row = blockIdx.x;
    const int C = a.C;
    const T *x = (const T *)a.X + row * C, *r = a.R ? (const T *)a.R + row * C : nullptr;
    float ss, unit = 1.f;
    for (;;) {
        float top = 0.f;
        ss = 0.f;
        for (int c = threadIdx.x; c < C; c += 256) {
            const float s = ((float)x[c] + (r ? (float)r[c] : 0.f)) * unit;
            ss = fmaf(s, s, ss);
            top = max_or_nan(top, fabsf(a.gamma ? s * a.gamma[c] : s));
        }
        for (int w = 32; w > 0; w >>= 1) {
            ss += __shfl_xor(ss, w);
            top = max_or_nan(top, __shfl_xor(top, w));
        }
        if ((threadIdx.x & 63) == 0) {
            part[0][threadIdx.x >> 6] = ss;
            part[1][threadIdx.x >> 6] = top;
        }
        __syncthreads();
        ss = part[0][0] + part[0][1] + part[0][2] + part[0][3];
        if (unit != 1.f) break;
        unit = row_unit(ss, a.eps);
        if (unit == 1.f) break;
        __syncthreads();  // (the second turn, at most, is the last)
    }
    const float rstd = 1.f / sqrtf(ss / (float)C + a.eps * unit * unit);
    float scale = 1.f;
    if constexpr (E8) {
        const float top = max_or_nan(max_or_nan(part[1][0], part[1][1]), max_or_nan(part[1][2], part[1][3]));
        scale = row_scale(top, rstd);
        if (threadIdx.x == 0) a.scales[row] = scale;
    }
    const float inv = 1.f / scale;  // (its product with rstd may overflow)
    for (int c = threadIdx.x; c < C; c += 256) {
        const float s = (float)x[c] + (r ? (float)r[c] : 0.f), su = s * unit;
        const float y = (a.gamma ? su * a.gamma[c] : su) * rstd * inv;
        if (a.S) ((T *)a.S)[row * C + c] = (T)s;
        if constexpr (E8)
            ((uint8_t *)a.Y)[row * C + c] = to_e4m3(y);
        else
            ((T *)a.Y)[row * C + c] = (T)y;
    }
}

}  // namespace
}  // namespace dsattn

using namespace dsattn;

extern "C" int dsattn_rmsnorm(const dsattn_rms_desc *desc, const void *X, const void *residual,
                              const float *gamma, void *sum, void *Y, float *scales, void *stream)
{
    const char *who = "dsattn_rmsnorm";
    if (!desc) return fail(DSATTN_EINVAL, "%s: null descriptor", who);
    const dsattn_rms_desc &d = *desc;
    if (d.rows < 1 || d.rows > 0x7fffffffLL || d.channels < 1 || d.channels > (1 << 20))
        return fail(DSATTN_EINVAL, "%s: rows outside [1, 2^31 - 1] or channels outside [1, 2^20]", who);
    if (d.io_dtype != DSATTN_F32 && d.io_dtype != DSATTN_BF16)
        return fail(DSATTN_EINVAL, "%s: unknown input dtype", who);
    if (d.out_dtype != d.io_dtype && d.out_dtype != DSATTN_E4M3)
        return fail(DSATTN_EINVAL, "%s: the output is of the input's dtype or in 8 bits", who);
    if (!(d.eps >= 0.f) || std::isinf(d.eps)) return fail(DSATTN_EINVAL, "%s: eps must be finite and >= 0", who);
    const bool e8 = d.out_dtype == DSATTN_E4M3;
    if (!X || !Y || (e8 && !scales)) return fail(DSATTN_EINVAL, "%s: null pointer", who);
    if (!e8 && scales) return fail(DSATTN_EINVAL, "%s: scales without an output in 8 bits", who);
    if (((uintptr_t)X | (uintptr_t)residual | (uintptr_t)gamma | (uintptr_t)sum | (uintptr_t)Y) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    if ((uintptr_t)scales & 3u) return fail(DSATTN_EINVAL, "%s: scales must be 4-byte aligned", who);
    const int64_t n = d.rows * d.channels, in = n * (d.io_dtype == DSATTN_BF16 ? 2 : 4);
    const int64_t out = e8 ? n : in;
    const struct { const void *p; int64_t n; } inputs[] = {{X, in}, {residual, in}, {gamma, 4 * (int64_t)d.channels}},
                                               outputs[] = {{sum, in}, {Y, out}, {scales, 4 * d.rows}};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 3; ++i) {
            const bool same = i < 2 && outputs[o].p == inputs[i].p && (o == 0 || (o == 1 && !e8));
            if (!same && overlap(outputs[o].p, outputs[o].n, inputs[i].p, inputs[i].n))
                return fail(DSATTN_EINVAL, "%s: an output overlaps an input", who);
        }
        for (int q = 0; q < o; ++q)
            if (overlap(outputs[o].p, outputs[o].n, outputs[q].p, outputs[q].n))
                return fail(DSATTN_EINVAL, "%s: two outputs overlap", who);
    }
    const RmsArgs a{X, residual, gamma, sum, Y, scales, d.rows, d.channels, d.eps};
    const bool f32 = d.io_dtype == DSATTN_F32;
    const RmsKernel k = f32 ? (e8 ? rms_pick<float, true>(d.channels) : rms_pick<float, false>(d.channels))
                            : (e8 ? rms_pick<__bf16, true>(d.channels) : rms_pick<__bf16, false>(d.channels));
    const void *fn = k.fn;
    unsigned groups = (unsigned)d.rows, threads = 256;
    if (fn) {
        const int per = k.lanes <= 256 ? 256 / k.lanes : 1;  // rows of a workgroup
        groups = (unsigned)((d.rows + per - 1) / per);
        threads = k.lanes <= 256 ? 256u : (unsigned)k.lanes;
    } else {
        fn = f32 ? (e8 ? (const void *)&rms_row_kernel<float, true> : (const void *)&rms_row_kernel<float, false>)
                 : (e8 ? (const void *)&rms_row_kernel<__bf16, true> : (const void *)&rms_row_kernel<__bf16, false>);
    }
    // (a launch has less than 2^32 threads)
    if ((uint64_t)groups * threads > 0xffffffffull)
        return fail(DSATTN_EUNSUPPORTED, "%s: too many rows for one launch", who);
    void *params[] = {(void *)&a};
    const hipError_t e = hipLaunchKernel(fn, dim3(groups), dim3(threads), params, 0, (hipStream_t)stream);
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
}
