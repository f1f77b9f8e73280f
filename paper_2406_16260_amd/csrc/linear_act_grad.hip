// Gradients of a product with bias, activation and gate (dsattn_linear_act_backward).
//
//   z_k = X W_k^T + b_k again,  dz_0 = dy [* z_1] act'(z_0),  dz_1 = dy * act(z_0)
//   dX = sum dz_k W_k,  dW_k = dz_k^T X,  db_k = column sums of dz_k
//
// Three products of the forward pass's size.  z is computed again: nothing is kept between the passes but X (z of 40,960 x 2 x
// 2,560 would be 420 MB, written and read in 165 us, a product 206 us at 1,300 TFLOP/s).
// dz goes through memory in the operands' type, to the other two: in bf16 that is its only rounding to fewer bits than fp32, and all
// that dX and dW are less exact by than an fp32 dz's would be (of the 2-norm, 2.35 * 10^-3 against 1.66 for the outputs' own
// rounding).  Two bf16 parts of dz would take twice the multiplies of both products and twice the traffic of dz.
// dX is the product of dz with W turned (X W^T kernels then do it); dW contracts over rows, which grad_tile.h reads transposed, its
// rows split over the card where W has few tiles.
// No atomics: splits and parts are joined in an order that the shape alone decides.  us, of which dz, dX, dW with its join:
//   40,960 x 640 x 2 x 2,560, GELU gate, bf16   876    363  241  262    (920 TFLOP/s; a large library product 1,300)
//   25,920 x 5,120 x 1,280, bias, bf16          614     20  263  331    (1,110 TFLOP/s)
//   160 x 1,280 x 1,280, SiLU, bf16             15-17  5.4  5.3  5.2
//   8,192 x 4,096 x 4,096, fp32                 4,010                   (137 TFLOP/s; a large library product 154)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "dsattn.h"
#include "plan.h"
#include "act_pick.h"
#include "grad_tile.h"
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
    const float c = fminf(fmaxf(x, -100.f), 100.f);  // (beyond, its factor is 0, and 0 * infinity would be NaN)
    switch (act) {
    case DSATTN_ACT_RELU:
        y = x > 0.f || x != x ? x : 0.f;
        d = x > 0.f ? 1.f : x != x ? x : 0.f;
        break;
    case DSATTN_ACT_GELU: {
        const float p = 0.5f * erfcf(x * -0.70710678f);
        y = x * p;
        d = fmaf(c * 0.39894228f, expf(-0.5f * c * c), p);
        break;
    }
    case DSATTN_ACT_GELU_TANH: {
        // p = (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)), dp/dx = 2 p (1 - p) du/dx
        const float u = 0.79788456f * x * fmaf(0.044715f, x * x, 1.f);
        const float p = 1.f / (1.f + expf(-2.f * u)), q = 1.f / (1.f + expf(2.f * u));
        y = x * p;
        d = fmaf(2.f * c * p * q, 0.79788456f * fmaf(0.134145f, c * c, 1.f), p);
        break;
    }
    case DSATTN_ACT_SILU: {
        const float p = 1.f / (1.f + expf(-x)), q = 1.f / (1.f + expf(x));
        y = x * p;
        d = fmaf(c * p, q, p);
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

// How the gradients are computed.  No kernel (fn null) for dz: the vector kernels do everything.
struct GradLaunch {
    bool tiles = false;                         // on the matrix cores
    const void *dz_fn = nullptr;                // kernel of dz; null: dz is dY
    int dz_rows = 0, dz_cols = 0, dz_waves = 0, dz_lds = 0;    // its tile, wavefronts and bytes of LDS
    bool dz_large = false, dz_small = false;
    int part_rows = 256;                             // rows of a part of the column sums
    bool x_small = false;                              // dX by the kernel for few rows; else W is turned for a product
    int x_splits = 1, x_span = 0;                      // the former's splits of the contraction, and their stages
    int x_deep = 0;                                    // by tiles of 64 or 128 with two stages ahead, or 0: dsattn_linear_act
    const void *w_fn = nullptr;                          // kernel of dW
    int w_rows = 0, w_cols = 0, w_waves = 0, w_lds = 0, splits = 1, stages = 0;
    size_t dz = 0, turned = 0, sums = 0, partial = 0, x_partial = 0, bytes = 0;    // places in the workspace, and its size
};

// dX as a product of dz and the turned W
dsattn_linear_act_desc product_of_dx(const dsattn_linear_act_desc &d)
{
    return {d.rows, d.n_w * d.c_out, d.c_in, 1, DSATTN_ACT_NONE, d.io_dtype, d.io_dtype, 0};
}

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

struct GradVariant {
    int rows, cols, waves, lds, part;  // (part: rows of a wavefront's, which it sums up)
    const void *fn[2];                 // gated
};
#define DSATTN_GRAD_TILE(T, MB, NB, WVM, WVN)                                                               \
    {16 * MB * WVM, 16 * NB * WVN, WVM * WVN, 2 * (16 * MB * WVM + 16 * NB * WVN) * kRow, 16 * MB,          \
     {(const void *)&act_tile_kernel<T, MB, NB, WVM, WVN, false, T, true>,                                  \
      (const void *)&act_tile_kernel<T, MB, NB, WVM, WVN, true, T, true>}}
const GradVariant kDzTiles[2][2] = {{DSATTN_GRAD_TILE(float, 2, 4, 4, 2), DSATTN_GRAD_TILE(float, 1, 4, 4, 1)},
                                    {DSATTN_GRAD_TILE(__bf16, 2, 4, 4, 2), DSATTN_GRAD_TILE(__bf16, 1, 4, 4, 1)}};
// bf16, two stages ahead.  Where tiles are so few that all are on the card at once, a long row's stages wait for their loads less
// than with one ahead, which leaves the LDS to more workgroups.  us of 64 x 64 tiles, and of 128 x 128, one ahead and two (dz with
// its sums joined, in a captured graph), rows x c_in x c_out:
//     150 x 4,312 x 3,272 (156 tiles, 52)      44.7  28.5    65.7  48.0
//     300 x 2,560 x 2,560 (200, 60)            26.3  18.4    36.7  30.7
//   1,000 x 1,280 x 1,280 (320, 80)            17.1  14.9    21.5  20.7
//   2,560 x 1,280 x 1,280 (800, 200)           23.4  25.8    24.5  22.1
//   1,000 x 4,096 x 4,096 (1,024, 256)         61.4  82.4    51.8  48.7
//   2,560 x   640 x   640 (400, 100; 10 stages)  10.8  11.1    14.0  14.4
// dW by one split: 2,560 x 1,280 x 1,280 (400) 25.2 20.8, 5,000 x 1,280 x 2,560 (200 of 128 x 128) 56.3 48.9, (800) 71.5 75.3.
#define DSATTN_GRAD_DEEP(MB, NB, WVM, WVN)                                                                  \
    {16 * MB * WVM, 16 * NB * WVN, WVM * WVN, 3 * (16 * MB * WVM + 16 * NB * WVN) * kRow, 16 * MB,          \
     {(const void *)&act_tile_kernel<__bf16, MB, NB, WVM, WVN, false, __bf16, true, 3>,                     \
      (const void *)&act_tile_kernel<__bf16, MB, NB, WVM, WVN, true, __bf16, true, 3>}}
const GradVariant kDzDeep[2] = {DSATTN_GRAD_DEEP(2, 4, 4, 2), DSATTN_GRAD_DEEP(1, 4, 4, 1)};
const void *const kXDeep[2] = {(const void *)&act_tile_kernel<__bf16, 2, 4, 4, 2, false, __bf16, false, 3>,
                               (const void *)&act_tile_kernel<__bf16, 2, 2, 2, 2, false, __bf16, false, 3>};
bool deep_is_faster(bool f32, int size, int64_t tiles, int64_t stages)
{
    return !f32 && stages >= 16 && tiles <= (size == 64 ? 512 : 256);
}

const void *const kDzSmall[2][2] = {
    {(const void *)&act_small_kernel<float, false, float, true>, (const void *)&act_small_kernel<float, true, float, true>},
    {(const void *)&act_small_kernel<__bf16, false, __bf16, true>, (const void *)&act_small_kernel<__bf16, true, __bf16, true>}};
#define DSATTN_GRAD_LARGE(G, ACT) (const void *)&grad_dz_large_kernel<G, ACT>
const void *const kDzLarge[2][DSATTN_ACT_SILU + 1] = {
    {nullptr, DSATTN_GRAD_LARGE(false, DSATTN_ACT_RELU), DSATTN_GRAD_LARGE(false, DSATTN_ACT_GELU),
     DSATTN_GRAD_LARGE(false, DSATTN_ACT_GELU_TANH), DSATTN_GRAD_LARGE(false, DSATTN_ACT_SILU)},
    {DSATTN_GRAD_LARGE(true, DSATTN_ACT_NONE), DSATTN_GRAD_LARGE(true, DSATTN_ACT_RELU), DSATTN_GRAD_LARGE(true, DSATTN_ACT_GELU),
     DSATTN_GRAD_LARGE(true, DSATTN_ACT_GELU_TANH), DSATTN_GRAD_LARGE(true, DSATTN_ACT_SILU)}};

const void *const kWJoin[2][2] = {  // few splits, 16 and more
    {(const void *)&grad_w_join_kernel<float, 1>, (const void *)&grad_w_join_kernel<float, 8>},
    {(const void *)&grad_w_join_kernel<__bf16, 1>, (const void *)&grad_w_join_kernel<__bf16, 8>}};
const void *const kWTiles[2][2] = {  // 64 x 64, 128 x 128
    {(const void *)&grad_w_tile_kernel<float, 2, 2, 2, 2>, (const void *)&grad_w_tile_kernel<float, 2, 4, 4, 2>},
    {(const void *)&grad_w_tile_kernel<__bf16, 2, 2, 2, 2>, (const void *)&grad_w_tile_kernel<__bf16, 2, 4, 4, 2>}};
const void *const kWDeep[2] = {(const void *)&grad_w_tile_kernel<__bf16, 2, 2, 2, 2, 3>,  // two stages ahead
                               (const void *)&grad_w_tile_kernel<__bf16, 2, 4, 4, 2, 3>};

// Estimated us of the weights' gradient by tiles of a size, tm x tn of them (the last column of 256 may be half empty) and splits of
// `stages` stages.  256: rounds of one workgroup a compute unit.  Smaller ones: a stage takes its latency, or the unit's
// throughput for the workgroups that share it (two of 128 x 128, five of 64 x 64; more come after them).  The splits' sums are
// joined by a kernel of its own.  Measured us (dW alone, in a captured graph; tile / splits), rows x c_in x c_out:
//                                 64 / 1   64 / 4   128 / 1   128 / 4   256 / 1    best
//    bf16   640 x   640 x   640      6.3        -      10.0         -      22.5    64 / 1 6.3
//         2,560 x 1,280 x 1,280     25.1     27.3      32.3      25.0      56.7    128 / 2 23.8
//        10,240 x 1,280 x 1,280     83.5     61.3     113.5      50.0     192.5    256 / 8 49.6
//        10,240 x   320 x   320     78.6     24.8     107.6      33.7     189.3    64 / 8 13.5
//        40,960 x   320 x 1,280    306.2     84.0     411.9     103.6     728.3    128 / 16 50.3
//         1,000 x 4,096 x 4,096        -        -      46.2         -      37.7    256 / 1 37.7
//    fp32   640 x   640 x   640     17.2     15.6      45.0      20.8              64 / 2 13.7
//        10,240 x 1,280 x 1,280    354.0    293.7     653.7     316.4              128 / 12 282.7
//        10,240 x   320 x   320    209.8     59.7     646.5     169.8              64 / 16 32.7
double w_estimate(int size, int64_t tm, int64_t tn, int64_t cin, int64_t splits, int64_t stages, bool f32, double numbers,
                  bool deep)
{
    const double st = (double)stages, join = splits > 1 ? 4.0 + 8.0 * (double)splits * numbers / 7e6 : 0.0;
    if (size == 256) {
        const int64_t half = cin % 256 != 0 && cin % 256 <= 128 ? 1 : 0;
        const int64_t f = (tm * (tn - half) * splits + 7) / 8, h = (tm * half * splits + 7) / 8;
        const int64_t rounds = (f + 31) / 32, spare = rounds * 32 - f;
        const double t = (double)rounds + 0.6 * (double)((std::max<int64_t>(0, h - spare) + 31) / 32);
        return t * (1.2 * st + 7.0) + join;
    }
    const double latency = size == 128 ? (f32 ? 2.0 : deep ? 0.55 : 0.67) : (f32 ? 0.65 : deep ? 0.3 : 0.45);
    const double each = size == 128 ? (f32 ? 2.0 : 0.5) : (f32 ? 0.55 : 0.2);
    const int64_t n = tm * tn * splits, fit = size == 128 ? 2 : 5;
    const double c = n <= 256 * fit ? (double)((n + 255) / 256) : (double)n / 256.0 + 0.5;
    return st * std::max(latency + 0.05 * (std::min(c, (double)fit) - 1.0), each * c) + 4.0 + join;
}

GradLaunch grad_pick(const dsattn_linear_act_desc &d)
{
    GradLaunch g;
    const bool f32 = d.io_dtype == DSATTN_F32, gated = d.n_w == 2;
    const int64_t es = f32 ? 4 : 2, No = (int64_t)d.n_w * d.c_out, rowbytes = d.c_in * es;
    // rows are whole 16-byte chunks, and a tile's are addressed with 32-bit offsets
    const bool fits = rowbytes % 16 == 0 && d.c_out * es % 16 == 0 && rowbytes * 256 < ((int64_t)1 << 31) &&
                      No * es * 256 < ((int64_t)1 << 31) && No < 1 << 22 && !(d.flags & DSATTN_FLAG_FORCE_GENERIC);
    auto tiles = [&](int64_t m, int64_t n, int rows, int cols) { return (m + rows - 1) / rows * ((n + cols - 1) / cols); };
    GradLaunch vector;
    vector.bytes = grad_is_dy(d) ? 0 : (size_t)d.rows * No * sizeof(float);
    if (!fits || tiles(No, d.c_in, 64, 64) >= (1 << 20)) return vector;
    g.tiles = true;
    // dz
    const int64_t stages = (rowbytes + kRow - 1) / kRow;
    if (!grad_is_dy(d)) {
        g.part_rows = 32;
        const GradVariant *v = kDzTiles[!f32];
        const int64_t n64 = tiles(d.rows, No, 64, 64), n128 = tiles(d.rows, No, 128, 128);
        const bool deep64 = deep_is_faster(f32, 64, n64, stages), deep128 = deep_is_faster(f32, 128, n128, stages);
        const double us64 = tile_estimate(64, n64, stages), us128 = tile_estimate(128, n128, stages, deep128);
        if (small_is_faster(d.io_dtype, tiles(d.rows, No, 32, 32), stages, 0.0, deep64)) {
            g.dz_small = true;
            g.dz_fn = kDzSmall[!f32][gated];
            g.dz_rows = g.dz_cols = 32;
            g.dz_waves = 8;
            g.dz_lds = kSmallLds;
        } else if (!f32 && tile_estimate(256, tiles(d.rows, No, 256, 256), stages) < std::min(us128, us64)) {
            g.dz_large = true;
            g.dz_fn = kDzLarge[gated][d.act];
            g.dz_rows = 256;
            g.dz_cols = 128;
            g.dz_waves = 4;
            g.dz_lds = kDzLargeLds;
            g.part_rows = 64;
        } else {
            // fp32: 64 x 64 where the last round of 128 x 128 (512, two a compute unit) would be so empty that they keep less
            // than 0.8 of the card busy.  us, 128 x 128 and 64 x 64, GELU, rows x c_in x c_out:
            //    5,000 x 1,280 x 1,280   164  152 (0.78)      4,096 x 4,096 x 4,096   977  1,029 (1.0)
            //   20,000 x   640 x   640   173  147 (0.77)      8,192 x 2,560 x 2,560   777    809 (0.83)
            //   10,240 x 1,280 x 1,280   320  287 (0.78)      6,000 x   640 x 1,280  91.3   94.5 (0.92)
            const bool by64 = f32 ? n128 * 10 < (n128 + 511) / 512 * 512 * 8 : us64 < us128;
            if (by64 ? deep64 : deep128) v = kDzDeep;
            v += by64;
            g.dz_fn = v->fn[gated];
            g.dz_rows = v->rows;
            g.dz_cols = v->cols;
            g.dz_waves = v->waves;
            g.dz_lds = v->lds;
            g.part_rows = v->part;
        }
        // (a launch has less than 2^32 threads, and tiles are numbered with 32 bits)
        if (tiles(d.rows, No, g.dz_rows, g.dz_cols) >= ((int64_t)1 << 31) / (64 * g.dz_waves)) return vector;
        g.dz = g.bytes;
        g.bytes += aligned((size_t)d.rows * No * es);
    }
    // Where no workgroups of dz's turn W behind theirs, a kernel of its own does: its launch, and a read and a write of W.  us,
    // dX by the kernel for few rows and of a turned W, bf16: 160 x 2,560 x 320 5.5 and 8.8, 640 x 640 x 640 6.5 and 10.7,
    // 1,000 x 640 x 640 8.7 and 10.7, 300 x 2,560 x 2,560 25 and 32, 2,560 x 640 x 640 19 and 11.
    const double turn_us = grad_is_dy(d) || g.dz_small ? 2.5 + 5e-7 * (double)(No * rowbytes) : 0.0;
    const int64_t x_stages = (No * es + kRow - 1) / kRow, x64 = tiles(d.rows, d.c_in, 64, 64), x128 = tiles(d.rows, d.c_in, 128, 128);
    const bool x_deep64 = deep_is_faster(f32, 64, x64, x_stages), x_deep128 = deep_is_faster(f32, 128, x128, x_stages);
    g.x_small = small_is_faster(d.io_dtype, tiles(d.rows, d.c_in, 32, 32), x_stages, turn_us, x_deep64);
    if (!g.x_small && !f32) {
        const double us64 = tile_estimate(64, x64, x_stages), us128 = tile_estimate(128, x128, x_stages, x_deep128);
        if (std::min(us64, us128) <= tile_estimate(256, tiles(d.rows, d.c_in, 256, 256), x_stages))
            g.x_deep = us64 < us128 ? (x_deep64 ? 64 : 0) : x_deep128 ? 128 : 0;
    }
    if (g.x_small) {
        // One round of workgroups leaves the card to a longer contraction's splits, of three stages a wavefront or more, joined by
        // a kernel of its own.  us of a call, bf16 and fp32: 1 x 392 x 2 x 5,040 33 71, with splits 22 32; 44 x 72 x 2 x 4,040 29 52,
        // 21 22; 32 x 2,048 x 4,096 30 50, 28 40.
        const int64_t all = d.n_w * ((d.c_out * es + kRow - 1) / kRow), n = tiles(d.rows, d.c_in, 32, 32);
        const int64_t splits = std::min(256 / n, all / 24);
        g.x_span = (int)all;
        if (splits >= 2) {
            g.x_span = (int)((all + splits - 1) / splits);
            g.x_splits = (int)((all + g.x_span - 1) / g.x_span);
            g.x_partial = g.bytes;
            g.bytes += aligned((size_t)g.x_splits * d.rows * d.c_in * sizeof(float));
        }
    }
    g.turned = g.bytes;
    if (!g.x_small) g.bytes += aligned((size_t)No * d.c_in * es);
    g.sums = g.bytes;
    g.bytes += aligned((size_t)((d.rows + g.part_rows - 1) / g.part_rows) * No * sizeof(float));
    // dW
    const int KS = kRow / (int)es;
    const int64_t all = (d.rows + KS - 1) / KS;
    double us = 1e30;
    bool w_deep = false;
    for (int size : {64, 128, 256}) {
        if (size == 256 && f32) break;
        const int64_t tm = (No + size - 1) / size, tn = (d.c_in + size - 1) / size;
        for (int64_t splits = 1; splits <= std::min<int64_t>(64, std::max<int64_t>(1, all / 2)); ++splits) {
            const int64_t stages = (all + splits - 1) / splits, used = (all + stages - 1) / stages;
            if (used != splits) continue;
            const bool deep = size < 256 && deep_is_faster(f32, size, tm * tn * splits, stages);
            const double t = w_estimate(size, tm, tn, d.c_in, splits, stages, f32, (double)No * (double)d.c_in, deep);
            if (t >= us) continue;
            w_deep = deep;
            us = t;
            g.w_rows = g.w_cols = size;
            g.splits = (int)splits;
            g.stages = (int)stages;
        }
    }
    g.w_waves = g.w_rows == 64 ? 4 : 8;
    g.w_lds = g.w_rows == 256 ? kLargeLds : (w_deep ? 3 : 2) * (g.w_rows + g.w_cols) * kRow;
    g.w_fn = g.w_rows == 256 ? (const void *)&grad_w_large_kernel : w_deep ? kWDeep[g.w_rows == 128] : kWTiles[!f32][g.w_rows == 128];
    g.partial = g.bytes;
    if (g.splits > 1) g.bytes += aligned((size_t)g.splits * No * d.c_in * sizeof(float));
    return g;
}

// The kernels one after the other: dz with its parts of the column sums and W turned behind it, dX, dW with the sums joined
// behind it, its splits joined.
int grad_launch(const dsattn_linear_act_desc &d, const GradLaunch &g, const GradArgs &a, const char *who, char *space, hipStream_t st)
{
    const int No = d.n_w * d.c_out;
    const bool f32 = d.io_dtype == DSATTN_F32, sums = a.db[0] || a.db[1];
    hipError_t e = hipSuccess;
    auto launch = [&](const void *fn, dim3 grid, int threads, void **params, int lds) {
        if (e == hipSuccess) e = allow_lds(fn, lds);
        if (e == hipSuccess) e = hipLaunchKernel(fn, grid, dim3((unsigned)threads), params, (size_t)lds, st);
    };
    auto join_splits = [&](GradWArgs &w) {
        const bool many = w.items / w.tiles >= 16;
        const int fours = many ? 32 : 256;  // of a workgroup
        void *params[] = {&w};
        launch(kWJoin[!f32][many], dim3((unsigned)(((int64_t)w.No * w.Cin / 4 + fours - 1) / fours)), 256, params, 0);
    };
    const TurnArgs turn{{a.W[0], a.W[1]}, space + g.turned, d.c_in, d.c_out, No, (d.c_in + 63) / 64};
    const int turns = a.dX && !g.x_small ? (No + 63) / 64 * turn.tiles_c : 0;  // workgroups that turn W
    // W beyond what the L2s hold: the small kernels go down its columns and read it once.  us, along and down:
    // 64 x 4,096 x 4,096 41.1 37.2, 130 x 4,104 x 2,056 (dX, dW) 42.4 32.0, 128 x 4,096 x 2 x 4,096 111 95.3; 160 x 1,280 x 1,280
    // 17.6 18.4
    const bool large_w = (int64_t)No * d.c_in * (f32 ? 4 : 2) >= 8 << 20;
    bool turned = false;
    float *parts = (float *)(space + g.sums);
    const int n_parts = (int)((d.rows + g.part_rows - 1) / g.part_rows);
    const bool direct = !g.dz_fn && d.rows <= 1024;  // few rows of dY: summed up at once
    if (g.dz_fn) {
        ActGradArgs z{};
        z.X = a.X;
        z.R = a.dY;
        z.Y = a.dz;
        z.M = d.rows;
        z.Cin = d.c_in;
        z.Cout = d.c_out;
        z.n_w = d.n_w;
        z.act = d.act;
        z.sums = sums ? parts : nullptr;
        for (int k = 0; k < d.n_w; ++k) {
            z.W[k] = a.W[k];
            z.bias[k] = a.bias[k];
        }
        const int cols = g.dz_cols / d.n_w;
        z.tiles_n = (d.c_out + cols - 1) / cols;
        const int32_t tiles_m = (int32_t)((d.rows + g.dz_rows - 1) / g.dz_rows);
        z.tiles = tiles_m * z.tiles_n;
        z.tiles_m = (g.dz_small ? tiles_m > 1 && large_w : down_reads_less(tiles_m, z.tiles_n)) ? tiles_m : 0;
        z.per_xcd = (z.tiles + kXcds - 1) / kXcds;
        z.panel = g.dz_large ? act_panel(z.tiles_n) : 1;
        z.groups = g.dz_small && !z.tiles_m ? z.tiles : z.per_xcd * kXcds;
        z.turn = turn;
        void *params[] = {&z};
        turned = turns && !g.dz_small;
        launch(g.dz_fn, dim3((unsigned)(z.groups + (turned ? turns : 0))), 64 * g.dz_waves, params, g.dz_lds);
    } else if (sums && !direct) {
        const void *dz = a.dz;
        int64_t M = d.rows;
        int no = No;
        void *params[] = {&dz, &M, &no, &parts};
        launch(f32 ? (const void *)&grad_sums_kernel<float> : (const void *)&grad_sums_kernel<__bf16>,
               dim3((unsigned)n_parts, (unsigned)(No + 127) / 128), 256, params, 0);
    }
    JoinArgs join{parts, false, {a.db[0], a.db[1]}, n_parts, d.c_out, No, sums ? (No + 15) / 16 : 0};
    if (direct) {
        join.sums = a.dz;
        join.half = !f32;
        join.parts = (int)d.rows;
    }
    if (sums && !a.dW[0] && !a.dW[1]) {
        void *params[] = {(void *)&join};
        launch((const void *)&grad_join_kernel, dim3((unsigned)join.groups), 1024, params, 0);
    }
    if (a.dX && g.x_small) {
        const int tiles_m = (int)((d.rows + 31) / 32);
        GradXArgs x{a.dz, {a.W[0], a.W[1]}, a.dX, d.rows, d.c_in, d.c_out, No, (d.c_in + 31) / 32};
        x.tiles_m = tiles_m > 1 && large_w ? tiles_m : 0;
        x.tiles = tiles_m * x.tiles_n;
        x.per_xcd = (x.tiles + kXcds - 1) / kXcds;
        x.span = g.x_span;
        x.partial = g.x_splits > 1 ? (float *)(space + g.x_partial) : nullptr;
        void *params[] = {&x};
        launch(f32 ? (const void *)&grad_x_small_kernel<float> : (const void *)&grad_x_small_kernel<__bf16>,
               dim3((unsigned)(x.tiles_m ? x.per_xcd * kXcds : x.tiles), (unsigned)g.x_splits), 512, params, kSmallLds);
        if (g.x_splits > 1) {
            GradWArgs s{};  // (one matrix of rows x c_in)
            s.dW[0] = a.dX;
            s.partial = x.partial;
            s.No = s.Cout = (int)d.rows;
            s.Cin = d.c_in;
            s.tiles = 1;
            s.items = g.x_splits;
            join_splits(s);
        }
    } else if (a.dX) {
        if (!turned) {
            void *params[] = {(void *)&turn};
            launch(f32 ? (const void *)&grad_turn_kernel<float> : (const void *)&grad_turn_kernel<__bf16>, dim3((unsigned)turns), 256,
                   params, 0);
        }
        if (g.x_deep) {
            ActArgs x{};
            x.X = a.dz;
            x.W[0] = turn.Wt;
            x.Y = a.dX;
            x.M = d.rows;
            x.Cin = No;
            x.Cout = d.c_in;
            x.n_w = 1;
            x.act = DSATTN_ACT_NONE;
            x.tiles_n = (d.c_in + g.x_deep - 1) / g.x_deep;
            const int32_t tiles_m = (int32_t)((d.rows + g.x_deep - 1) / g.x_deep);
            x.tiles = tiles_m * x.tiles_n;
            x.tiles_m = down_reads_less(tiles_m, x.tiles_n) ? tiles_m : 0;
            x.per_xcd = (x.tiles + kXcds - 1) / kXcds;
            x.panel = 1;
            void *params[] = {&x};
            launch(kXDeep[g.x_deep == 64], dim3((unsigned)(x.per_xcd * kXcds)), g.x_deep == 64 ? 256 : 512, params,
                   3 * 2 * g.x_deep * kRow);
        } else {
            if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
            const dsattn_linear_act_desc x = product_of_dx(d);
            const int rc = dsattn_linear_act(&x, a.dz, nullptr, &turn.Wt, nullptr, nullptr, nullptr, a.dX, st);
            if (rc != DSATTN_OK) return rc;
        }
    }
    if (a.dW[0] || a.dW[1]) {
        GradWArgs w{};
        w.dz = a.dz;
        w.X = a.X;
        w.dW[0] = a.dW[0];
        w.dW[1] = a.dW[1];
        w.partial = (float *)(space + g.partial);
        w.M = d.rows;
        w.Cin = d.c_in;
        w.Cout = d.c_out;
        w.No = No;
        w.tiles_n = (d.c_in + g.w_cols - 1) / g.w_cols;
        w.tiles = (No + g.w_rows - 1) / g.w_rows * w.tiles_n;
        w.items = w.tiles * g.splits;
        w.per_xcd = (w.items + kXcds - 1) / kXcds;
        w.stages = g.stages;
        w.groups = w.per_xcd * kXcds;
        w.join = join;
        if (g.w_rows == 256) {
            const int half = d.c_in % 256 != 0 && d.c_in % 256 <= 128 ? 1 : 0, tm = w.tiles / w.tiles_n;
            w.whole = w.tiles_n - half;
            w.whole_xcd = (tm * w.whole * g.splits + kXcds - 1) / kXcds;
            w.rest_xcd = (tm * half * g.splits + kXcds - 1) / kXcds;
            w.groups = (w.whole_xcd + w.rest_xcd) * kXcds;
        }
        void *params[] = {&w};
        launch(g.w_fn, dim3((unsigned)(w.groups + join.groups)), 64 * g.w_waves, params, g.w_lds);
        if (g.splits > 1) join_splits(w);
    }
    if (e != hipSuccess) return fail(DSATTN_EHIP, "%s: %s", who, hipGetErrorString(e));
    return DSATTN_OK;
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
    *bytes = grad_pick(*desc).bytes;
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
    const GradLaunch g = grad_pick(d);
    const size_t need = g.bytes;
    if (need && (!workspace || workspace_bytes < need)) return fail(DSATTN_EINVAL, "%s: workspace of %zu bytes needed", who, need);
    if (((uintptr_t)X | (uintptr_t)dY | (uintptr_t)dX | (uintptr_t)workspace) & 15u)
        return fail(DSATTN_EINVAL, "%s: pointers must be 16-byte aligned", who);
    GradArgs a{};
    a.X = X;
    a.dY = dY;
    a.dX = dX;
    a.dz = grad_is_dy(d) ? (void *)dY : (char *)workspace + g.dz;
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
    if (g.tiles) {
        const dsattn_linear_act_desc x = product_of_dx(d);
        dsattn_conv_info info;
        if (dX && !g.x_small && (dsattn_linear_act_info(&x, &info) != DSATTN_OK || (!info.kernel && d.rows * d.c_in / 256 >= 0xffffff)))
            return fail(DSATTN_EUNSUPPORTED, "%s: too large for one launch", who);
        return grad_launch(d, g, a, who, (char *)workspace, st);
    }
    // (a launch has less than 2^32 threads)
    auto blocks = [](int64_t n) { return (n + 255) / 256; };
    if (blocks(d.rows * std::max(d.c_out, d.c_in)) > 0xffffff || blocks((int64_t)d.c_out * d.c_in) > 0x7fffff)
        return fail(DSATTN_EUNSUPPORTED, "%s: too large for the generic kernel", who);
    if (!grad_is_dy(d))
        e = hipLaunchKernel(f32 ? (const void *)&grad_dz_kernel<float> : (const void *)&grad_dz_kernel<__bf16>,
                            dim3((unsigned)blocks(d.rows * d.c_out)), dim3(256), params, 0, st);
    const bool wide = f32 || !grad_is_dy(d);  // dz in fp32
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
