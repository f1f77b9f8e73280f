// Root-mean-square normalisation with the residual's addition (dsattn_rmsnorm).
//
//   s = x + r,  y = s * rsqrt(mean(s^2) + eps) * gamma,  optionally y / scale in 8 bits
//
// One workgroup a row: a pass for the sum of squares and for max|s gamma| (the largest |y| is that
// times the row's factor, so a scale needs no pass of its own), a second one that writes.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "dsattn.h"
#include "plan.h"

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

// y in 8 bits, to nearest, ties to even
__device__ __forceinline__ uint8_t to_e4m3(float y)
{
    return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 255);
}

// The maximum of two numbers, NaN if one is: what fmaxf() would drop.
__device__ __forceinline__ float max_or_nan(float a, float b) { return a > b || a != a ? a : b; }

// The scale of a row whose largest |s gamma| is top.
__device__ __forceinline__ float row_scale(float top, float rstd)
{
    const float s = top * rstd / 448.f;
    return s < 0x1p-126f ? 0x1p-126f : s;  // (a NaN stays)
}

template <typename T, bool E8>
__global__ __launch_bounds__(256) void rms_row_kernel(const RmsArgs a)
{
    __shared__ float part[2][4];
    const int64_t row = blockIdx.x;
    const int C = a.C;
    const T *x = (const T *)a.X + row * C, *r = a.R ? (const T *)a.R + row * C : nullptr;
    float ss = 0.f, top = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) {
        const float s = (float)x[c] + (r ? (float)r[c] : 0.f);
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
    const float rstd = 1.f / sqrtf(ss / (float)C + a.eps);
    float scale = 1.f;
    if constexpr (E8) {
        top = max_or_nan(max_or_nan(part[1][0], part[1][1]), max_or_nan(part[1][2], part[1][3]));
        scale = row_scale(top, rstd);
        if (threadIdx.x == 0) a.scales[row] = scale;
    }
    const float inv = 1.f / scale;  // (its product with rstd may overflow)
    for (int c = threadIdx.x; c < C; c += 256) {
        const float s = (float)x[c] + (r ? (float)r[c] : 0.f);
        const float y = (a.gamma ? s * a.gamma[c] : s) * rstd * inv;
        if (a.S) ((T *)a.S)[row * C + c] = (T)s;
        if constexpr (E8)
            ((uint8_t *)a.Y)[row * C + c] = to_e4m3(y);
        else
            ((T *)a.Y)[row * C + c] = (T)y;
    }
}

bool overlap(const void *a, int64_t an, const void *b, int64_t bn)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + (uintptr_t)bn && y < x + (uintptr_t)an;
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
    const void *fn = f32 ? (e8 ? (const void *)&rms_row_kernel<float, true> : (const void *)&rms_row_kernel<float, false>)
                         : (e8 ? (const void *)&rms_row_kernel<__bf16, true> : (const void *)&rms_row_kernel<__bf16, false>);
    void *params[] = {(void *)&a};
    const hipError_t e = hipLaunchKernel(fn, dim3((unsigned)d.rows), dim3(256), params, 0, (hipStream_t)stream);
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
}
