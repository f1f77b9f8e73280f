// Gradients of a product with bias, activation and gate (dsattn_linear_act_backward).
//
//   z_k = X W_k^T + b_k again,  dz_0 = dy [* z_1] act'(z_0),  dz_1 = dy * act(z_0)
//   dX = sum dz_k W_k,  dW_k = dz_k^T X,  db_k = column sums of dz_k
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "dsattn.h"
#include "plan.h"
#include "rows.h"

namespace dsattn {
namespace {

struct GradArgs {
    const void *X, *dY;
    const void *W[2];
    const float *bias[2];
    void *dX;
    void *dW[2];
    float *db[2];
    void *dz;          // [M][n_w * Cout]
    int64_t M;
    int32_t Cin, Cout, n_w, act;
};

// The activation and its derivative.
__device__ __forceinline__ void act_and_slope(float x, int act, float &y, float &d)
{
    switch (act) {
    case DSATTN_ACT_RELU:
        y = x > 0.f || x != x ? x : 0.f;
        d = x > 0.f ? 1.f : x != x ? x : 0.f;
        break;
    case DSATTN_ACT_GELU: {
        const float p = 0.5f * erfcf(x * -0.70710678f);
        y = x * p;
        d = fmaf(x * 0.39894228f, expf(-0.5f * x * x), p);
        break;
    }
    case DSATTN_ACT_GELU_TANH: {
        // p = (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)), dp/dx = 2 p (1 - p) du/dx
        const float x2 = x * x, u = 0.79788456f * x * fmaf(0.044715f, x2, 1.f);
        const float p = 1.f / (1.f + expf(-2.f * u)), q = 1.f / (1.f + expf(2.f * u));
        y = x * p;
        d = fmaf(2.f * x * p * q, 0.79788456f * fmaf(0.134145f, x2, 1.f), p);
        break;
    }
    case DSATTN_ACT_SILU: {
        const float p = 1.f / (1.f + expf(-x)), q = 1.f / (1.f + expf(x));
        y = x * p;
        d = fmaf(x * p, q, p);
        break;
    }
    default:
        y = x;
        d = 1.f;
    }
}

// Plain vector kernels: one thread per number of dz (fp32), dX and dW.  TZ: float, or T where dz is dY itself.
template <typename T>
__global__ __launch_bounds__(256) void grad_dz_kernel(const GradArgs a)
{
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= a.M * a.Cout) return;
    const int64_t m = idx / a.Cout;
    const int co = (int)(idx - m * a.Cout);
    const T *x = (const T *)a.X + m * a.Cin;
    float z[2] = {0.f, 0.f};
    for (int k = 0; k < a.n_w; ++k) {
        const T *w = (const T *)a.W[k] + (int64_t)co * a.Cin;
        float acc = 0.f;
        for (int c = 0; c < a.Cin; ++c) acc = fmaf((float)w[c], (float)x[c], acc);
        z[k] = acc + (a.bias[k] ? a.bias[k][co] : 0.f);
    }
    float y, d;
    act_and_slope(z[0], a.act, y, d);
    const float dy = (float)((const T *)a.dY)[idx];
    float *to = (float *)a.dz + m * a.n_w * a.Cout + co;
    to[0] = dy * (a.n_w == 2 ? z[1] * d : d);
    if (a.n_w == 2) to[a.Cout] = dy * y;
}

template <typename T, typename TZ>
__global__ __launch_bounds__(256) void grad_dx_kernel(const GradArgs a)
{
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= a.M * a.Cin) return;
    const int64_t m = idx / a.Cin;
    const int ci = (int)(idx - m * a.Cin);
    float acc = 0.f;
    for (int k = 0; k < a.n_w; ++k) {
        const TZ *dz = (const TZ *)a.dz + (m * a.n_w + k) * a.Cout;
        const T *w = (const T *)a.W[k] + ci;
        for (int c = 0; c < a.Cout; ++c) acc = fmaf((float)dz[c], (float)w[(int64_t)c * a.Cin], acc);
    }
    ((T *)a.dX)[idx] = (T)acc;
}

template <typename T, typename TZ>
__global__ __launch_bounds__(256) void grad_dw_kernel(const GradArgs a)
{
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int k = blockIdx.y;
    if (idx >= (int64_t)a.Cout * a.Cin || !a.dW[k]) return;
    const int co = (int)(idx / a.Cin), ci = (int)(idx - (int64_t)co * a.Cin);
    const TZ *dz = (const TZ *)a.dz + (int64_t)k * a.Cout + co;
    const T *x = (const T *)a.X + ci;
    float acc = 0.f;
    for (int64_t m = 0; m < a.M; ++m) acc = fmaf((float)dz[m * a.n_w * a.Cout], (float)x[m * a.Cin], acc);
    ((T *)a.dW[k])[idx] = (T)acc;
}

// Column sums of dz: 16 columns a workgroup, 64 threads to each.
template <typename TZ>
__global__ __launch_bounds__(1024) void grad_db_kernel(const GradArgs a)
{
    __shared__ float sums[64][17];
    const int l = threadIdx.x & 15, w = threadIdx.x >> 4, k = blockIdx.y;
    const int c = (int)blockIdx.x * 16 + l;
    if (!a.db[k]) return;
    float v = 0.f;
    if (c < a.Cout)
        for (int64_t m = w; m < a.M; m += 64) v += (float)((const TZ *)a.dz)[(m * a.n_w + k) * a.Cout + c];
    sums[w][l] = v;
    __syncthreads();
    for (int h = 32; h > 0; h >>= 1) {
        if (w < h) sums[w][l] += sums[w + h][l];
        __syncthreads();
    }
    if (w == 0 && c < a.Cout) a.db[k][c] = sums[0][l];
}

int grad_validate(const dsattn_linear_act_desc *desc, const char *who)
{
    if (!desc) return fail(DSATTN_EINVAL, "%s: null descriptor", who);
    const dsattn_linear_act_desc &d = *desc;
    if (d.rows < 1 || d.rows > 0x7fffffffLL || d.c_in < 1 || d.c_out < 1)
        return fail(DSATTN_EINVAL, "%s: sizes must be positive (rows at most 2^31 - 1)", who);
    // (2^45 numbers a tensor, so that the bytes of both sets are counted in 64 bits)
    const int64_t most = (int64_t)1 << 45, widest = std::max(d.c_in, d.c_out);
    if (d.rows > most / widest || (int64_t)d.c_in > most / d.c_out) return fail(DSATTN_EINVAL, "%s: problem too large", who);
    if (d.n_w < 1 || d.n_w > 2) return fail(DSATTN_EINVAL, "%s: n_w %d is neither 1 nor 2", who, d.n_w);
    if (d.act < DSATTN_ACT_NONE || d.act > DSATTN_ACT_SILU) return fail(DSATTN_EINVAL, "%s: unknown activation", who);
    if (d.io_dtype != DSATTN_F32 && d.io_dtype != DSATTN_BF16)
        return fail(DSATTN_EINVAL, "%s: tensors are fp32 or bf16", who);
    if (d.out_dtype != d.io_dtype) return fail(DSATTN_EINVAL, "%s: the output's dtype must be the input's", who);
    if (d.flags & ~DSATTN_FLAG_FORCE_GENERIC) return fail(DSATTN_EINVAL, "%s: unknown flag bits 0x%x", who, d.flags);
    return DSATTN_OK;
}

// Where the derivative is 1 everywhere dz is dY itself.
bool grad_is_dy(const dsattn_linear_act_desc &d) { return d.act == DSATTN_ACT_NONE && d.n_w == 1; }

size_t grad_bytes(const dsattn_linear_act_desc &d)
{
    if (grad_is_dy(d)) return 0;
    return (size_t)d.rows * d.n_w * d.c_out * sizeof(float);
}

}  // namespace
}  // namespace dsattn

using namespace dsattn;

extern "C" {

int dsattn_linear_act_backward_workspace(const dsattn_linear_act_desc *desc, size_t *bytes)
{
    const int rc = grad_validate(desc, "dsattn_linear_act_backward_workspace");
    if (rc != DSATTN_OK) return rc;
    if (!bytes) return fail(DSATTN_EINVAL, "dsattn_linear_act_backward_workspace: null output");
    *bytes = grad_bytes(*desc);
    return DSATTN_OK;
}

int dsattn_linear_act_backward(const dsattn_linear_act_desc *desc, const void *X, const void *const *W,
                               const float *const *bias, const void *dY, void *dX, void *const *dW, float *const *dbias,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "dsattn_linear_act_backward";
    const int rc = grad_validate(desc, who);
    if (rc != DSATTN_OK) return rc;
    const dsattn_linear_act_desc &d = *desc;
    if (!X || !W || !dY) return fail(DSATTN_EINVAL, "%s: null pointer", who);
    const int64_t es = d.io_dtype == DSATTN_F32 ? 4 : 2;
    const int64_t xn = d.rows * d.c_in * es, yn = d.rows * d.c_out * es, wn = (int64_t)d.c_out * d.c_in * es, bn = 4 * (int64_t)d.c_out;
    const size_t need = grad_bytes(d);
    if (need && (!workspace || workspace_bytes < need)) return fail(DSATTN_EINVAL, "%s: workspace of %zu bytes needed", who, need);
    if (((uintptr_t)X | (uintptr_t)dY | (uintptr_t)dX | (uintptr_t)workspace) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    GradArgs a{};
    a.X = X;
    a.dY = dY;
    a.dX = dX;
    a.dz = need ? workspace : (void *)dY;
    a.M = d.rows;
    a.Cin = d.c_in;
    a.Cout = d.c_out;
    a.n_w = d.n_w;
    a.act = d.act;
    for (int k = 0; k < d.n_w; ++k) {
        a.W[k] = W[k];
        a.bias[k] = bias ? bias[k] : nullptr;
        a.dW[k] = dW ? dW[k] : nullptr;
        a.db[k] = dbias ? dbias[k] : nullptr;
        if (!W[k]) return fail(DSATTN_EINVAL, "%s: null pointer in set %d", who, k);
        if (((uintptr_t)W[k] | (uintptr_t)a.dW[k]) & 15u) return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
        if (((uintptr_t)a.bias[k] | (uintptr_t)a.db[k]) & 3u) return fail(DSATTN_EINVAL, "%s: biases must be 4-byte aligned", who);
    }
    const struct { const void *p; int64_t n; }
        in[] = {{X, xn}, {dY, yn}, {a.W[0], wn}, {a.W[1], wn}, {a.bias[0], bn}, {a.bias[1], bn}},
        out[] = {{dX, xn}, {a.dW[0], wn}, {a.dW[1], wn}, {a.db[0], bn}, {a.db[1], bn}, {need ? workspace : nullptr, (int64_t)need}};
    for (int o = 0; o < 6; ++o) {
        for (const auto &i : in)
            if (overlap(out[o].p, out[o].n, i.p, i.n)) return fail(DSATTN_EINVAL, "%s: an output overlaps an input", who);
        for (int q = 0; q < o; ++q)
            if (overlap(out[o].p, out[o].n, out[q].p, out[q].n)) return fail(DSATTN_EINVAL, "%s: two outputs overlap", who);
    }
    const bool f32 = d.io_dtype == DSATTN_F32;
    const hipStream_t st = (hipStream_t)stream;
    void *params[] = {&a};
    hipError_t e = hipSuccess;
    // (a launch has less than 2^32 threads)
    auto blocks = [](int64_t n) { return (n + 255) / 256; };
    if (blocks(d.rows * std::max(d.c_out, d.c_in)) > 0xffffff || blocks((int64_t)d.c_out * d.c_in) > 0x7fffff)
        return fail(DSATTN_EUNSUPPORTED, "%s: too large for the generic kernel", who);
    if (need)
        e = hipLaunchKernel(f32 ? (const void *)&grad_dz_kernel<float> : (const void *)&grad_dz_kernel<__bf16>,
                            dim3((unsigned)blocks(d.rows * d.c_out)), dim3(256), params, 0, st);
    const bool wide = f32 || need;  // dz in fp32
    if (e == hipSuccess && dX)
        e = hipLaunchKernel(f32    ? (const void *)&grad_dx_kernel<float, float>
                            : wide ? (const void *)&grad_dx_kernel<__bf16, float>
                                   : (const void *)&grad_dx_kernel<__bf16, __bf16>,
                            dim3((unsigned)blocks(d.rows * d.c_in)), dim3(256), params, 0, st);
    if (e == hipSuccess && (a.dW[0] || a.dW[1]))
        e = hipLaunchKernel(f32    ? (const void *)&grad_dw_kernel<float, float>
                            : wide ? (const void *)&grad_dw_kernel<__bf16, float>
                                   : (const void *)&grad_dw_kernel<__bf16, __bf16>,
                            dim3((unsigned)blocks((int64_t)d.c_out * d.c_in), (unsigned)d.n_w), dim3(256), params, 0, st);
    if (e == hipSuccess && (a.db[0] || a.db[1]))
        e = hipLaunchKernel(wide ? (const void *)&grad_db_kernel<float> : (const void *)&grad_db_kernel<__bf16>,
                            dim3((unsigned)(d.c_out + 15) / 16, (unsigned)d.n_w), dim3(1024), params, 0, st);
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
}

}  // extern "C"
