// Token-wise product with bias, activation, gate and residual in its epilogue (dsattn_linear_act).
//
//   z_k = (X W_k^T) x_scale w_scale_k + b_k,   Y = act(z_0) [* z_1] + R
//
// Bound by the matrix cores where there are many rows, by latency where there are few.  Four kernels on the matrix cores and a
// vector kernel for rows that are not whole 16-byte pieces; estimates of their times choose (act_pick()).  us and TFLOP/s:
//   25,920 x 5,120 x 1,280, residual, bf16             270 to 283   1,200 to 1,260   (elementary fp32 operations 2,560; a
//                                                                     library product without bias and residual 251)
//   40,960 x 640 x 5,120, bias, bf16                   232   1,157   (library product 308 to 348)
//   40,960 x 640 x 2 x 2,560, GELU gate, bf16          249 to 272   990 to 1,080
//   61,440 x 1,280 x 2 x 5,120, GELU gate, 8 bits      783 to 831   1,940 to 2,060   (16,384 x 5,120 x 16,384: 2,440 to 2,860)
//       the same with fp32 sums                        1,682 to 1,833   880 to 960   (16,384 x 5,120 x 16,384: 1,010 to 1,090)
//   8,192 x 4,096 x 4,096, bias, fp32                  1,917 to 1,931   143
//   160 x 1,280 x 1,280, bf16                          4.1           in a captured graph
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "dsattn.h"
#include "plan.h"

namespace dsattn {
namespace {

struct ActArgs {
    const void *X;
    const void *W[2];
    const float *bias[2];      // [c_out] or null
    const float *xs, *ws[2];   // scales of rows and channels, or null
    const void *R;             // [M][c_out] or null
    void *Y;
    int64_t M;
    int32_t Cin, Cout, n_w, act;
    int32_t tiles_n, tiles, per_xcd;  // column tiles; all of them; ceil(tiles / 8)
    int32_t panel;                    // persistent kernels: column tiles that are numbered together
};

struct e4m3 { uint8_t bits; };
struct e4m3w { uint8_t bits; };  // the same, to be multiplied in 16 bits

template <typename T>
__device__ __forceinline__ float to_float(T x)
{
    if constexpr (std::is_same_v<T, e4m3>)
        return __builtin_amdgcn_cvt_f32_fp8((int)x.bits, 0);
    else
        return (float)x;
}

__device__ __forceinline__ float activate(float x, int act)
{
    switch (act) {
    case DSATTN_ACT_RELU: return x > 0.f || x != x ? x : 0.f;
    case DSATTN_ACT_GELU: return 0.5f * x * (1.f + erff(x * 0.70710678f));
    case DSATTN_ACT_GELU_TANH: {
        // 1 + tanh(u) = 2 / (1 + exp(-2 u))
        const float u = 0.79788456f * (x + 0.044715f * x * x * x);
        return x / (1.f + expf(-2.f * u));
    }
    case DSATTN_ACT_SILU: return x / (1.f + expf(-x));
    default: return x;
    }
}

// Plain vector kernel: one thread per output element, output channel fastest.
template <typename Tin, typename Tout>
__global__ __launch_bounds__(256) void act_generic_kernel(const ActArgs a)
{
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= a.M * a.Cout) return;
    const int64_t m = idx / a.Cout;
    const int co = (int)(idx - m * a.Cout);
    const Tin *x = (const Tin *)a.X + m * a.Cin;
    float z[2] = {0.f, 0.f};
    for (int k = 0; k < a.n_w; ++k) {
        const Tin *w = (const Tin *)a.W[k] + (int64_t)co * a.Cin;
        float acc = 0.f;
        for (int c = 0; c < a.Cin; ++c) acc = fmaf(to_float(w[c]), to_float(x[c]), acc);
        if (a.xs) acc *= a.xs[m];
        if (a.ws[k]) acc *= a.ws[k][co];
        z[k] = acc + (a.bias[k] ? a.bias[k][co] : 0.f);
    }
    float y = activate(z[0], a.act);
    if (a.n_w == 2) y *= z[1];
    if (a.R) y += (float)((const Tout *)a.R)[idx];
    ((Tout *)a.Y)[idx] = (Tout)y;
}

}  // namespace
}  // namespace dsattn

#include "act_tile.h"

namespace dsattn {
namespace {

// Kernels of one tile shape, by operands, gate and output.
struct ActVariant {
    int rows, cols, waves, lds;  // tile (rows of X, rows of W of both sets), wavefronts, bytes of dynamic LDS
    const void *fn[2][2];        // gated, fp32 output
};

// The persistent kernels, by gate, output and activation.
constexpr int kActs = DSATTN_ACT_SILU + 1;
struct StreamVariant {
    const void *fn[2][2][kActs];
};
#define DSATTN_ACT_TILE(T, MB, NB, WVM, WVN)                                                                        \
    {Mul<T>::BS * MB * WVM, Mul<T>::BS * NB * WVN, WVM * WVN,                                                       \
     2 * (Mul<T>::BS * MB * WVM + Mul<T>::BS * NB * WVN) * kRow,                                                    \
     {{(const void *)&act_tile_kernel<T, MB, NB, WVM, WVN, false, __bf16>,                                          \
       (const void *)&act_tile_kernel<T, MB, NB, WVM, WVN, false, float>},                                          \
      {(const void *)&act_tile_kernel<T, MB, NB, WVM, WVN, true, __bf16>,                                           \
       (const void *)&act_tile_kernel<T, MB, NB, WVM, WVN, true, float>}}}
// (8 bits: bf16 outputs only)
#define DSATTN_ACT_TILE_E4M3(MB, NB, WVM, WVN)                                                                      \
    {32 * MB * WVM, 32 * NB * WVN, WVM * WVN, 2 * (32 * MB * WVM + 32 * NB * WVN) * kRow,                           \
     {{(const void *)&act_tile_kernel<e4m3, MB, NB, WVM, WVN, false, __bf16>, nullptr},                             \
      {(const void *)&act_tile_kernel<e4m3, MB, NB, WVM, WVN, true, __bf16>, nullptr}}}
#define DSATTN_ACT_TILE_F32(MB, NB, WVM, WVN)                                                                       \
    {16 * MB * WVM, 16 * NB * WVN, WVM * WVN, 2 * (16 * MB * WVM + 16 * NB * WVN) * kRow,                           \
     {{nullptr, (const void *)&act_tile_kernel<float, MB, NB, WVM, WVN, false, float>},                             \
      {nullptr, (const void *)&act_tile_kernel<float, MB, NB, WVM, WVN, true, float>}}}
const ActVariant kBf16Variants[] = {DSATTN_ACT_TILE(__bf16, 2, 4, 4, 2), DSATTN_ACT_TILE(__bf16, 2, 2, 2, 2)};
const ActVariant kF32Variants[] = {DSATTN_ACT_TILE_F32(2, 4, 4, 2), DSATTN_ACT_TILE_F32(2, 2, 2, 2)};
const ActVariant kE4m3Variants[] = {DSATTN_ACT_TILE_E4M3(1, 2, 4, 2), DSATTN_ACT_TILE_E4M3(1, 2, 2, 1)};
const ActVariant kE4m3WideVariants[] = {DSATTN_ACT_TILE(e4m3w, 2, 4, 4, 2), DSATTN_ACT_TILE(e4m3w, 2, 4, 2, 1)};

// The kernels of small products: gated, fp32 output.
#define DSATTN_ACT_SMALL(T, F32)                                                                  \
    {F32 ? (const void *)&act_small_kernel<T, false, float> : (const void *)&act_small_kernel<T, false, __bf16>, \
     F32 ? (const void *)&act_small_kernel<T, true, float> : (const void *)&act_small_kernel<T, true, __bf16>}
const void *const kSmall[3][2][2] = {  // by type of the operands, fp32 output, gate
    {{nullptr, nullptr}, DSATTN_ACT_SMALL(float, true)},
    {DSATTN_ACT_SMALL(__bf16, false), DSATTN_ACT_SMALL(__bf16, true)},
    {DSATTN_ACT_SMALL(e4m3w, false), DSATTN_ACT_SMALL(e4m3w, true)}};

#define DSATTN_ACT_STREAM(T, MB, NB, G, TO)                                                       \
    {                                                                                             \
        (const void *)&act_stream_kernel<T, MB, NB, G, TO, DSATTN_ACT_NONE>,                      \
            (const void *)&act_stream_kernel<T, MB, NB, G, TO, DSATTN_ACT_RELU>,                  \
            (const void *)&act_stream_kernel<T, MB, NB, G, TO, DSATTN_ACT_GELU>,                  \
            (const void *)&act_stream_kernel<T, MB, NB, G, TO, DSATTN_ACT_GELU_TANH>,             \
            (const void *)&act_stream_kernel<T, MB, NB, G, TO, DSATTN_ACT_SILU>                   \
    }
const StreamVariant kBf16Stream = {{{DSATTN_ACT_STREAM(__bf16, 4, 8, false, __bf16), DSATTN_ACT_STREAM(__bf16, 4, 8, false, float)},
                                    {DSATTN_ACT_STREAM(__bf16, 4, 8, true, __bf16), DSATTN_ACT_STREAM(__bf16, 4, 8, true, float)}}};
const StreamVariant kE4m3Stream = {{{DSATTN_ACT_STREAM(e4m3, 2, 4, false, __bf16), {}}, {DSATTN_ACT_STREAM(e4m3, 2, 4, true, __bf16), {}}}};

// Whether the small kernel is faster than 64 x 64 tiles, by estimates in us: rounds of workgroups on a whole card's 256 compute
// units (on a part of one the choice is the same, and the result), and the time of a stage (of all of a row's in the tile
// kernel, of its eighth in the small one).  Measured us in a captured graph, small and 64 x 64, rows x c_in x c_out:
//                                       bf16            fp32            e4m3
//       1 x   320 x 1,280            2.9   3.5       4.2   8.0       3.0   3.4
//       1 x 5,120 x 1,280            7.1  21.7      23.8  96.6       6.1  13.7
//     160 x 1,280 x 1,280            4.1   7.5       8.8  26.7       4.0   5.9
//     320 x 1,280 x 1,280            6.7   7.7      15.5  27.5       6.4   6.0
//     640 x   640 x   640            5.5   5.1      10.0  14.9       5.4   4.5
//     100 x 4,096 x 4,096           17.0  32.0      46.5  79.5      12.3  17.6
//     640 x 1,280 x 1,280           12.3   8.8      30.0  28.0      11.6   6.3
bool small_is_faster(int32_t type, int64_t small_tiles, int64_t stages)
{
    static const double small_stage[] = {0.17, 0.07, 0.1}, tile_stage[] = {0.6, 0.27, 0.35};  // by dsattn_dtype
    const double rounds = (double)((small_tiles + 255) / 256);
    return 1.5 + rounds * (1.2 + small_stage[type] * (double)stages) < 2.0 + tile_stage[type] * (double)stages;
}

// Estimated us of `tiles` tiles of 256 x 256 (persistent), 128 x 128 or 64 x 64 and `stages` stages, bf16 or 8 bits: a start,
// and per round on the compute units the stages of a tile and what its start and end cost (two workgroups of the 128 x 128
// kernel share a unit, so that a round of it is 512 tiles).  Measured us in a captured graph, bf16 and e4m3, rows x c_in x c_out:
//                                  64 x 64       128 x 128     256 x 256
//      2,560 x 1,280 x 1,280     17.8  10.3     18.1   9.7    27.9  17.0
//      5,120 x 1,280 x 1,280     29.8  18.6     23.8  15.5    30.0  19.1
//     10,240 x 1,280 x 1,280     55.8  30.8     43.1  26.7    34.0  21.4
//     16,000 x 1,280 x 1,280     79.8  46.1     60.5  35.1    57.6  35.2
//     20,000 x 1,280 x   320     29.0  18.9     23.3  15.8    28.9  19.4
//     40,960 x   320 x   320     19.2  17.4     17.6  14.4    22.4  19.7
//      8,000 x   640 x   640     13.5  10.8     13.1  10.1    17.9  12.8
double tile_estimate(int size, int64_t tiles, int64_t stages)
{
    const double st = (double)stages, n = (double)tiles;
    const int64_t full = tiles / 512, rest = tiles - 512 * full, rounds = (tiles + 255) / 256;
    if (size == 256) return 3.0 + (double)rounds * (1.22 * st + 5.0);
    if (size == 128)
        return 3.0 + (double)full * (0.95 * st + 2.0) + (rest > 256 ? 0.82 * st + 2.6 : rest > 0 ? 0.61 * st + 2.9 : 0.0);
    static const double stage[] = {0.25, 0.3, 0.41, 0.61};
    return 4.0 + 1.3e-3 * n + st * (rounds > 4 ? std::max(1.0, 8.2e-4 * n) : stage[rounds - 1]);
}

// How a product runs; fn null: the vector kernel.
struct ActLaunch {
    const void *fn = nullptr;
    int rows, cols, waves, lds;
    bool stream, small;
};
ActLaunch act_pick(const dsattn_linear_act_desc &d, int64_t es)
{
    const int64_t rowbytes = d.c_in * es;
    // rows are whole 16-byte chunks, and a tile's are addressed with 32-bit offsets
    if (rowbytes % 16 != 0 || rowbytes * 256 >= ((int64_t)1 << 31) || d.c_out >= 1 << 22 || (d.flags & DSATTN_FLAG_FORCE_GENERIC))
        return {};
    const bool f32 = d.out_dtype == DSATTN_F32, gated = d.n_w == 2;
    const int64_t n = (int64_t)d.c_out * d.n_w;
    auto tiles = [&](int rows, int cols) { return (d.rows + rows - 1) / rows * ((n + cols - 1) / cols); };
    const int64_t stages = (rowbytes + kRow - 1) / kRow, large = tiles(256, 256);
    if (small_is_faster(d.io_dtype, tiles(32, 32), stages))
        return {kSmall[d.io_dtype][f32][gated], 32, 32, 8, kSmallLds, false, true};
    // sums of 8-bit operands in fp32: for an fp32 output, and where the caller wants them
    const bool wide = d.io_dtype == DSATTN_E4M3 && (f32 || (d.flags & DSATTN_FLAG_FP32_SUMS));
    const ActVariant *v = d.io_dtype == DSATTN_F32    ? kF32Variants
                          : d.io_dtype == DSATTN_BF16 ? kBf16Variants
                          : wide                      ? kE4m3WideVariants
                                                      : kE4m3Variants;
    if (d.io_dtype == DSATTN_F32) {
        if (tiles(128, 128) < 384) ++v;
    } else {
        const double us128 = tile_estimate(128, tiles(128, 128), stages), us64 = tile_estimate(64, tiles(64, 64), stages);
        const StreamVariant *sv = d.io_dtype == DSATTN_BF16 ? &kBf16Stream : &kE4m3Stream;
        // (tiles are numbered with 32 bits)
        if (!wide && large < (1 << 30) && tile_estimate(256, large, stages) < std::min(us128, us64))
            return {sv->fn[gated][f32][d.act], 256, 256, 8, kStreamLds, true, false};
        if (us64 < us128) ++v;
    }
    // (a launch has less than 2^32 threads)
    if (tiles(v->rows, v->cols) >= ((int64_t)1 << 32) / (64 * v->waves) - kXcds) return {};
    return {v->fn[gated][f32], v->rows, v->cols, v->waves, v->lds, false, false};
}

// Column tiles that are numbered together.  An XCD's 32 tiles in flight are this many wide and 32 / width row tiles high,
// and read as many rows of X and of W as the sum of the two: the width for which that is least, in panels of one size.
int act_panel(int tiles_n)
{
    int best = 1, least = 1 << 30;
    for (int width = 1; width <= std::min(tiles_n, 32); ++width) {
        const int rows = width + (32 + width - 1) / width;
        if (tiles_n % width == 0 && rows < least) {
            least = rows;
            best = width;
        }
    }
    return best;
}

int compute_units(int dev)
{
    static std::atomic<int> cached[64];
    int n = dev < 64 ? cached[dev].load(std::memory_order_relaxed) : 0;
    if (n > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    if (dev < 64) cached[dev].store(n, std::memory_order_relaxed);
    return n;
}

bool overlap(const void *a, int64_t an, const void *b, int64_t bn)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + (uintptr_t)bn && y < x + (uintptr_t)an;
}

int64_t dtype_bytes(int32_t t) { return t == DSATTN_F32 ? 4 : t == DSATTN_BF16 ? 2 : 1; }

int act_validate(const dsattn_linear_act_desc *desc, const char *who)
{
    if (!desc) return fail(DSATTN_EINVAL, "%s: null descriptor", who);
    const dsattn_linear_act_desc &d = *desc;
    if (d.rows < 1 || d.rows > 0x7fffffffLL || d.c_in < 1 || d.c_out < 1)
        return fail(DSATTN_EINVAL, "%s: sizes must be positive (rows at most 2^31 - 1)", who);
    // (2^46 numbers a tensor, so that their bytes are counted in 64 bits)
    const int64_t most = (int64_t)1 << 46, widest = std::max(d.c_in, d.c_out);
    if (d.rows > most / widest || (int64_t)d.c_in > most / d.c_out) return fail(DSATTN_EINVAL, "%s: problem too large", who);
    if (d.n_w < 1 || d.n_w > 2) return fail(DSATTN_EINVAL, "%s: n_w %d is neither 1 nor 2", who, d.n_w);
    if (d.act < DSATTN_ACT_NONE || d.act > DSATTN_ACT_SILU)
        return fail(DSATTN_EINVAL, "%s: unknown activation", who);
    if (d.io_dtype != DSATTN_F32 && d.io_dtype != DSATTN_BF16 && d.io_dtype != DSATTN_E4M3)
        return fail(DSATTN_EINVAL, "%s: unknown input dtype", who);
    if (d.out_dtype != DSATTN_F32 && (d.out_dtype != DSATTN_BF16 || d.io_dtype == DSATTN_F32))
        return fail(DSATTN_EINVAL, "%s: the output is fp32, or bf16 of inputs of 16 or 8 bits", who);
    if (d.flags & ~(DSATTN_FLAG_FORCE_GENERIC | DSATTN_FLAG_FP32_SUMS))
        return fail(DSATTN_EINVAL, "%s: unknown flag bits 0x%x", who, d.flags);
    return DSATTN_OK;
}

}  // namespace
}  // namespace dsattn

using namespace dsattn;

extern "C" {

int dsattn_linear_act_info(const dsattn_linear_act_desc *desc, dsattn_conv_info *info)
{
    const int rc = act_validate(desc, "dsattn_linear_act_info");
    if (rc != DSATTN_OK) return rc;
    if (!info) return fail(DSATTN_EINVAL, "dsattn_linear_act_info: null output");
    const dsattn_linear_act_desc &d = *desc;
    const int64_t es = dtype_bytes(d.io_dtype), os = dtype_bytes(d.out_dtype), n = (int64_t)d.c_out * d.n_w;
    *info = dsattn_conv_info{};
    const ActLaunch v = act_pick(d, es);
    if (v.fn) {
        info->kernel = 1;
        info->tile_m = v.rows;
        info->tile_n = v.cols;
        info->tile_k = (int32_t)(kRow / es);
        info->n_blocks = (int32_t)((d.rows + v.rows - 1) / v.rows * ((n + v.cols - 1) / v.cols));
        info->block_threads = 64 * v.waves;
        info->lds_bytes = v.lds;
    } else {
        info->tile_n = 1;
        info->tile_k = 1;
        info->n_blocks = (int32_t)std::min<int64_t>((d.rows * d.c_out + 255) / 256, 0x7fffffff);
        info->block_threads = 256;
    }
    info->useful_flops = (int64_t)std::min(2.0 * (double)(d.rows * d.c_in) * (double)n, 0x1p62);
    info->algorithmic_bytes = (d.rows + n) * d.c_in * es + d.rows * d.c_out * os;
    return DSATTN_OK;
}

int dsattn_linear_act(const dsattn_linear_act_desc *desc, const void *X, const float *x_scales,
                      const void *const *W, const float *const *w_scales, const float *const *bias,
                      const void *residual, void *Y, void *stream)
{
    const char *who = "dsattn_linear_act";
    const int rc = act_validate(desc, who);
    if (rc != DSATTN_OK) return rc;
    const dsattn_linear_act_desc &d = *desc;
    if (!X || !W || !Y) return fail(DSATTN_EINVAL, "%s: null pointer", who);
    const int64_t es = dtype_bytes(d.io_dtype), os = dtype_bytes(d.out_dtype);
    const int64_t xn = d.rows * d.c_in * es, wn = (int64_t)d.c_out * d.c_in * es, yn = d.rows * d.c_out * os;
    if (((uintptr_t)X | (uintptr_t)Y | (uintptr_t)residual) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    if (d.io_dtype != DSATTN_E4M3 && (x_scales || w_scales))
        return fail(DSATTN_EINVAL, "%s: scales belong to operands in 8 bits", who);
    if ((uintptr_t)x_scales & 3u) return fail(DSATTN_EINVAL, "%s: scales must be 4-byte aligned", who);
    ActArgs a{};
    a.X = X;
    a.xs = x_scales;
    a.R = residual;
    a.Y = Y;
    a.M = d.rows;
    a.Cin = d.c_in;
    a.Cout = d.c_out;
    a.n_w = d.n_w;
    a.act = d.act;
    for (int k = 0; k < d.n_w; ++k) {
        a.W[k] = W[k];
        a.bias[k] = bias ? bias[k] : nullptr;
        a.ws[k] = w_scales ? w_scales[k] : nullptr;
        if (!W[k]) return fail(DSATTN_EINVAL, "%s: null pointer in set %d", who, k);
        if ((uintptr_t)W[k] & 15u) return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
        if (((uintptr_t)a.bias[k] | (uintptr_t)a.ws[k]) & 3u)
            return fail(DSATTN_EINVAL, "%s: biases and scales must be 4-byte aligned", who);
        if (overlap(Y, yn, W[k], wn)) return fail(DSATTN_EINVAL, "%s: Y overlaps W", who);
        if (overlap(Y, yn, a.bias[k], 4 * (int64_t)d.c_out) || overlap(Y, yn, a.ws[k], 4 * (int64_t)d.c_out))
            return fail(DSATTN_EINVAL, "%s: Y overlaps a bias or a scale", who);
    }
    if (overlap(Y, yn, X, xn) || overlap(Y, yn, x_scales, 4 * d.rows))
        return fail(DSATTN_EINVAL, "%s: Y overlaps X or its scales", who);
    if (residual != Y && overlap(Y, yn, residual, yn))
        return fail(DSATTN_EINVAL, "%s: Y overlaps the residual without being it", who);
    const bool f32 = d.out_dtype == DSATTN_F32;
    const ActLaunch v = act_pick(d, es);
    if (v.fn) {
        const int cols = v.cols / d.n_w;
        a.tiles_n = (d.c_out + cols - 1) / cols;
        a.tiles = (int32_t)((d.rows + v.rows - 1) / v.rows) * a.tiles_n;
        a.per_xcd = (a.tiles + kXcds - 1) / kXcds;
        a.panel = act_panel(a.tiles_n);
        int dev = 0, per_xcd = a.per_xcd;
        hipError_t e = v.stream ? hipGetDevice(&dev) : hipSuccess;
        if (v.stream) per_xcd = std::min(per_xcd, (compute_units(dev) + kXcds - 1) / kXcds);
        // the default cap on dynamic LDS is 64 KB
        if (e == hipSuccess && v.lds > 64 << 10) e = hipFuncSetAttribute(v.fn, hipFuncAttributeMaxDynamicSharedMemorySize, v.lds);
        void *params[] = {&a};
        if (e == hipSuccess)
            e = hipLaunchKernel(v.fn, dim3(v.small ? (unsigned)a.tiles : (unsigned)per_xcd * kXcds), dim3(64 * v.waves), params, (size_t)v.lds, (hipStream_t)stream);
        if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
        return DSATTN_OK;
    }
    // (a launch has less than 2^32 threads)
    const int64_t blocks = (d.rows * d.c_out + 255) / 256;
    if (blocks > 0xffffff) return fail(DSATTN_EUNSUPPORTED, "%s: too large for the generic kernel", who);
    const void *fn = d.io_dtype == DSATTN_F32 ? (const void *)&act_generic_kernel<float, float>
                     : d.io_dtype == DSATTN_BF16
                         ? (f32 ? (const void *)&act_generic_kernel<__bf16, float> : (const void *)&act_generic_kernel<__bf16, __bf16>)
                         : (f32 ? (const void *)&act_generic_kernel<e4m3, float> : (const void *)&act_generic_kernel<e4m3, __bf16>);
    void *params[] = {&a};
    const hipError_t e = hipLaunchKernel(fn, dim3((unsigned)blocks), dim3(256), params, 0, (hipStream_t)stream);
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
}

}  // extern "C"
