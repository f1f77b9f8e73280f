// The matrix-core kernels of dsattn_linear_act: both operands are rows of c_in numbers, a stage of the
// contraction is one 128-byte line of each (32 fp32, 64 bf16 or 128 e4m3 channels), which goes straight
// from memory into LDS, 16-byte chunks swizzled by their row.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "dsattn.h"

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
    int32_t tiles_m;                  // gradients' tiles: row tiles where they are numbered column by column, or 0
};

// W_0 and W_1 below each other, transposed, for the product that gives dX: 64 x 64 numbers a workgroup, of workgroups behind
// those of another kernel.
struct TurnArgs {
    const void *W[2];  // [Cout][Cin] each
    void *Wt;          // [Cin][No]
    int32_t Cin, Cout, No, tiles_c;
};
// Gradients: R is dy, Y is dz.
struct ActGradArgs : ActArgs {
    float *sums;     // [parts of rows][n_w Cout], column sums, or null
    int32_t groups;  // workgroups of the product; those behind turn W
    TurnArgs turn;
};

struct e4m3 { uint8_t bits; };
struct e4m3w { uint8_t bits; };  // the same, to be multiplied in 16 bits

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kRow = 128;  // bytes of an operand row in a stage
constexpr int kXcds = 8;

// s_waitcnt of at most n outstanding vector memory operations, and all LDS operations done
__host__ __device__ constexpr int waitcnt_vm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4); }

// What a kernel multiplies with.  A fragment is a lane's 16 bytes (32 in 8 bits) of an operand row; which
// channels an instruction contracts is free as long as both operands agree.
//   bf16  v_mfma_f32_16x16x32_bf16, two a stage: chunk 4 kk + lane / 16 of row lane % 16
//   fp32  the same chunk, its four numbers with four v_mfma_f32_16x16x4_f32
//   e4m3  v_mfma_f32_32x32x64_f8f6f4, two a stage: chunks 4 kk + lane / 32 and two further on, of row lane % 32.
//         (16x16x128, one a stage, has the same rate and needs twice the fragments at a time.)  The instructions on
//         8 bits, of every shape, line the products of a group up with its largest one and drop what is more than 13
//         bits below it (the accumulator keeps its fp32): 1.3e-5 of the result's 2-norm at 64 to 1,280 channels of
//         normal numbers, 1/130 of a bf16 output's own rounding, but what large products that cancel leave may be
//         lost.  So these serve a bf16 output, unless the caller asks for fp32 sums; for those and for an fp32 output
//   e4m3w the numbers are converted to bf16, exactly, and multiplied with 16x16x32: fp32 sums at half the rate (gated
//         61,440 x 1,280 x 5,120 785 and 1,682 us, 16,384 x 5,120 x 16,384 1,068 and 2,525)
// Block: rows of a fragment, BS; the accumulator's element 4 q + e of lane l is channel 8 q + 4 (l / BS) + e
// of the block of W rows and row l % BS of the block of X rows (q = 0 only where BS is 16).
template <typename T>
struct Mul {
    static constexpr int BS = 16, QUADS = 1;
    using Acc = f32x4;
    using Frag = std::conditional_t<sizeof(T) == 4, f32x4, bf16x8>;
    static __device__ __forceinline__ int offset(int lane, int kk) { return (((4 * kk) | (lane >> 4)) ^ (lane & 7)) * 16; }
    static __device__ __forceinline__ Frag read(const unsigned char *row, int off) { return *(const Frag *)(row + off); }
    static __device__ __forceinline__ Frag from(const i32x4 &a) { return __builtin_bit_cast(Frag, a); }
    static __device__ __forceinline__ Acc mul(const Frag &w, const Frag &x, Acc c)
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[s], x[s], c, 0, 0, 0);
            return c;
        } else {
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0);
        }
    }
};
template <>
struct Mul<e4m3> {
    static constexpr int BS = 32, QUADS = 4;
    using Acc = f32x16;
    using Frag = i32x8;
    // (position p of row r holds chunk p ^ r % 8: the second chunk is two further on, another bit of the position.  Half of these
    // reads are two-way conflicts, 43 % of the LDS's cycles; by r / 2 % 8 there are none, and gated 61,440 x 1,280 x 5,120 takes
    // 796 us instead of 783: it is the chip's power that the kernel waits for, with a clock of 1.4 to 1.8 GHz.)
    static __device__ __forceinline__ int offset(int lane, int kk) { return (((4 * kk) | (lane >> 5)) ^ (lane & 7)) * 16; }
    static __device__ __forceinline__ Frag read(const unsigned char *row, int off)
    {
        const i32x4 a = *(const i32x4 *)(row + off), b = *(const i32x4 *)(row + (off ^ 32));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ Acc mul(const Frag &w, const Frag &x, Acc c)
    {
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, 0, 0, 0, 0);
    }
};

template <>
struct Mul<e4m3w> {
    static constexpr int BS = 16, QUADS = 1;
    using Acc = f32x4;
    struct Frag { bf16x8 half[2]; };
    static __device__ __forceinline__ int offset(int lane, int kk) { return Mul<__bf16>::offset(lane, kk); }
    static __device__ __forceinline__ Frag read(const unsigned char *row, int off) { return from(*(const i32x4 *)(row + off)); }
    static __device__ __forceinline__ Frag from(const i32x4 &a)
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        Frag f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a[w], 1.f, false);
            const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a[w], 1.f, true);
            f.half[w / 2][4 * (w & 1)] = lo[0];
            f.half[w / 2][4 * (w & 1) + 1] = lo[1];
            f.half[w / 2][4 * (w & 1) + 2] = hi[0];
            f.half[w / 2][4 * (w & 1) + 3] = hi[1];
        }
        return f;
    }
    static __device__ __forceinline__ Acc mul(const Frag &w, const Frag &x, Acc c)
    {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.half[0], x.half[0], c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.half[1], x.half[1], c, 0, 0, 0);
    }
};

// 2^x on the instruction
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// x / 2 * (1 + erf(x / sqrt 2)) = x P(x), P the normal distribution's function: as x / (1 + 2^(-x p(x^2))), where p is fitted to
// log2(P / (1 - P)) / x so that the largest error of P, anywhere, is least: 2.9e-8 with seven terms.  Two instructions on the
// transcendental unit and ten others; with the rational approximation 7.1.26 of Abramowitz and Stegun (1.5e-7) it is two
// and fifteen, and erff() several times that, which an epilogue at the matrix cores' heels feels.
__device__ __forceinline__ float gelu_part(float x)
{
    const float t = x * x;
    float p = fmaf(t, -5.067244690e-09f, 3.816315040e-07f);
    p = fmaf(p, t, -1.143983534e-05f);
    p = fmaf(p, t, 1.595799422e-04f);
    p = fmaf(p, t, 9.404923028e-05f);
    p = fmaf(p, t, -1.048351218e-01f);
    p = fmaf(p, t, -2.302209292e+00f);
    return __builtin_amdgcn_rcpf(1.f + exp2_fast(x * p));
}
__device__ __forceinline__ float gelu_erf(float x) { return x * gelu_part(x); }

template <int ACT>
__device__ __forceinline__ float act_fast(float x)
{
    if constexpr (ACT == DSATTN_ACT_RELU) return x > 0.f || x != x ? x : 0.f;
    if constexpr (ACT == DSATTN_ACT_GELU) return gelu_erf(x);
    if constexpr (ACT == DSATTN_ACT_GELU_TANH) {
        // -2 log2(e) sqrt(2 / pi) (x + 0.044715 x^3)
        const float u = x * fmaf(x * x, -0.10294324f, -2.3022082f);
        return x * __builtin_amdgcn_rcpf(1.f + exp2_fast(u));
    }
    if constexpr (ACT == DSATTN_ACT_SILU) return x * __builtin_amdgcn_rcpf(1.f + exp2_fast(x * -1.44269504f));
    return x;
}

// f(activation as a constant): the switch is outside of the loops that f holds
template <typename F>
__device__ __forceinline__ void with_act(int act, F &&f)
{
    switch (act) {
    case DSATTN_ACT_RELU: f(std::integral_constant<int, DSATTN_ACT_RELU>{}); break;
    case DSATTN_ACT_GELU: f(std::integral_constant<int, DSATTN_ACT_GELU>{}); break;
    case DSATTN_ACT_GELU_TANH: f(std::integral_constant<int, DSATTN_ACT_GELU_TANH>{}); break;
    case DSATTN_ACT_SILU: f(std::integral_constant<int, DSATTN_ACT_SILU>{}); break;
    default: f(std::integral_constant<int, DSATTN_ACT_NONE>{}); break;
    }
}

// The column of W behind row r of a column tile: set, and channel from the tile's first on.  Gated, blocks of BS
// rows of the gate and of the value alternate, so that a lane holds both of a channel.
template <int BS, bool GATED>
__device__ __forceinline__ int set_of(int r) { return GATED ? (r / BS) & 1 : 0; }
template <int BS, bool GATED>
__device__ __forceinline__ int channel_of(int r) { return GATED ? r / (2 * BS) * BS + r % BS : r; }

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The epilogue of a wavefront's part, MB x NB blocks from row m0 and output channel c0 on: MP x NP blocks at a time go
// through `stage`, the wavefront's own (BS MP) rows of (BS NP output channels + 4) floats, and leave as whole rows
// with the residual added.  (fp32 on the way: the sum with the residual is rounded once.)
template <typename T, int MB, int NB, int MP, int NP, bool GATED, typename TO, bool SCALED>
__device__ __forceinline__ void epilogue(const ActArgs &a, const typename Mul<T>::Acc (&acc)[MB][NB], int64_t m0, int c0,
                                         const float *bias, const float *wscale, float *stage, int lane)
{
    using M = Mul<T>;
    constexpr int BS = M::BS, NO = GATED ? 2 : 1;      // blocks of W rows behind a block of channels
    constexpr int CH = BS * NP / NO, SR = CH + 4;      // channels of a pass, floats of a staged row
    constexpr int PER = 16 / (int)sizeof(TO);          // channels of a 16-byte piece
    constexpr int CPR = CH / PER, PIECES = BS * MP * CPR;
    static_assert(MB % MP == 0 && NB % NP == 0 && NP % NO == 0 && CH % PER == 0, "whole passes");
    const int rl = lane % BS, cq = 4 * (lane / BS);
    const bool whole = a.Cout % PER == 0;
#pragma unroll
    for (int ip = 0; ip < MB; ip += MP)
#pragma unroll
        for (int jp = 0; jp < NB; jp += NP) {
            const int64_t mp = m0 + BS * ip;
            const int cp = c0 + BS * jp / NO;
            float xs[MP];
            if constexpr (SCALED) {
#pragma unroll
                for (int i = 0; i < MP; ++i) {
                    const int64_t m = mp + BS * i + rl;
                    xs[i] = a.xs ? a.xs[m < a.M ? m : a.M - 1] : 1.f;
                }
            }
            with_act(a.act, [&](auto act) __attribute__((always_inline)) {
                constexpr int ACT = decltype(act)::value;
#pragma unroll
                for (int j = 0; j < NP; j += NO)
#pragma unroll
                    for (int q = 0; q < M::QUADS; ++q) {
                        f32x4 b[NO], s[NO];
#pragma unroll
                        for (int k = 0; k < NO; ++k) {
                            const int at = BS * (jp + j + k) + 8 * q + cq;
                            b[k] = *(const f32x4 *)(bias + at);
                            if constexpr (SCALED) s[k] = *(const f32x4 *)(wscale + at);
                        }
#pragma unroll
                        for (int i = 0; i < MP; ++i) {
                            f32x4 y;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float z[NO];
#pragma unroll
                                for (int k = 0; k < NO; ++k) {
                                    z[k] = acc[ip + i][jp + j + k][4 * q + e];
                                    if constexpr (SCALED) z[k] = z[k] * xs[i] * s[k][e];  // (the scales' product may overflow)
                                    z[k] += b[k][e];
                                }
                                y[e] = act_fast<ACT>(z[0]);
                                if constexpr (GATED) y[e] *= z[1];
                            }
                            *(f32x4 *)(stage + (BS * i + rl) * SR + BS * j / NO + 8 * q + cq) = y;
                        }
                    }
            });
            wave_sync();
#pragma unroll
            for (int it = 0; it < (PIECES + 63) / 64; ++it) {
                const int p = lane + 64 * it;
                const int row = p / CPR, ch = (p - row * CPR) * PER;
                const int64_t m = mp + row;
                if ((PIECES % 64 != 0 && p >= PIECES) || m >= a.M || cp + ch >= a.Cout) continue;
                const float *from = stage + row * SR + ch;
                const int64_t at = m * a.Cout + cp + ch;
                TO *to = (TO *)a.Y + at;
                const TO *r = (const TO *)a.R + at;
                if (whole) {
                    typedef TO Piece __attribute__((ext_vector_type(PER)));
                    Piece y;
                    if (a.R) {
                        const Piece rv = *(const Piece *)r;
#pragma unroll
                        for (int e = 0; e < PER; ++e) y[e] = (TO)(from[e] + (float)rv[e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < PER; ++e) y[e] = (TO)from[e];
                    }
                    *(Piece *)to = y;
                } else {
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (cp + ch + e < a.Cout) to[e] = (TO)(a.R ? from[e] + (float)r[e] : from[e]);
                }
            }
            wave_sync();
        }
}

// Bias and scale of column r of a column tile (of the tile from output channel n0 on); past c_out: 0.
template <int BS, bool GATED, bool SCALED>
__device__ __forceinline__ void column(const ActArgs &a, int n0, int r, float &bias, float &scale)
{
    const int set = set_of<BS, GATED>(r), c = n0 + channel_of<BS, GATED>(r);
    const float *b = set ? a.bias[1] : a.bias[0], *s = set ? a.ws[1] : a.ws[0];
    bias = b && c < a.Cout ? b[c] : 0.f;
    if constexpr (SCALED) scale = !s ? 1.f : c < a.Cout ? s[c] : 0.f;
}

constexpr uint32_t kOob = 0xfffffff0u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const void *p, int64_t row, int64_t rows, int rowbytes)
{
    const int64_t left = max((int64_t)0, (rows - row) * rowbytes);
    return __builtin_amdgcn_make_buffer_rsrc((void *)((const unsigned char *)p + row * rowbytes), 0,
                                             (int)min(left, (int64_t)0x7fffffff), 0x00020000);
}

// Gradients of the activation's argument and of its gate: dz_0 = dy [* z_1] act'(z_0), dz_1 = dy act(z_0).  A wavefront's part as
// in epilogue(); 16 rows x 64 channels at a time through the wavefront's own kGradBytes, into which dy comes (up to four passes
// ahead) and from which dz leaves, as rows of n_w Cout numbers in the operands' type.  The columns' sums over the part's rows, in fp32 of unrounded dz, go
// to row `part` of a.sums.
// Both derivatives take x within +-100: beyond, its factor is 0, and 0 * infinity would be NaN.
template <int ACT>
__device__ __forceinline__ void act_slope_fast(float x, float &y, float &d)
{
    const float c = __builtin_amdgcn_fmed3f(x, -100.f, 100.f);
    if constexpr (ACT == DSATTN_ACT_RELU) {
        y = x > 0.f || x != x ? x : 0.f;
        d = x > 0.f ? 1.f : x != x ? x : 0.f;
    } else if constexpr (ACT == DSATTN_ACT_GELU) {
        const float p = gelu_part(x);
        y = x * p;
        d = fmaf(c * 0.39894228f, exp2_fast(c * c * -0.72134752f), p);
    } else if constexpr (ACT == DSATTN_ACT_GELU_TANH) {
        const float c2 = c * c, p = __builtin_amdgcn_rcpf(1.f + exp2_fast(x * fmaf(x * x, -0.10294324f, -2.3022082f)));
        y = x * p;
        d = fmaf(c * p * (1.f - p), fmaf(0.21406550f, c2, 1.5957691f), p);
    } else if constexpr (ACT == DSATTN_ACT_SILU) {
        const float p = __builtin_amdgcn_rcpf(1.f + exp2_fast(x * -1.44269504f));
        y = x * p;
        d = fmaf(c * p, 1.f - p, p);
    } else {
        y = x;
        d = 1.f;
    }
}

template <typename T, int THREADS>
__device__ __forceinline__ void turn_tile(const TurnArgs &a, int block, unsigned char *smem)
{
    constexpr int PER = 16 / (int)sizeof(T), CPR = 64 / PER, ROWS = THREADS / CPR, SR = 64 + 4 / (int)sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(PER)));
    T *tile = (T *)smem;  // [64][SR]
    const int ot = block / a.tiles_c, o0 = ot * 64, c0 = (block - ot * a.tiles_c) * 64, r = threadIdx.x / CPR, p = threadIdx.x % CPR * PER;
#pragma unroll
    for (int i = 0; i < 64; i += ROWS) {
        const int o = o0 + r + i, c = c0 + p;
        Piece x{};
        const T *w = (const T *)(o < a.Cout ? a.W[0] : a.W[1]);
        if (o < a.No && c < a.Cin) x = *(const Piece *)(w + (int64_t)(o < a.Cout ? o : o - a.Cout) * a.Cin + c);
#pragma unroll
        for (int e = 0; e < PER; ++e) tile[(p + e) * SR + r + i] = x[e];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 64; i += ROWS) {
        const int c = c0 + r + i, o = o0 + p;
        if (c >= a.Cin || o >= a.No) continue;
        Piece x;
#pragma unroll
        for (int e = 0; e < PER; ++e) x[e] = tile[(r + i) * SR + p + e];
        *(Piece *)((T *)a.Wt + (int64_t)c * a.No + o) = x;
    }
}

// 64 channels of a pass (a whole line of 16-bit numbers) or as many as the part has, and a staged row of them: 16 bytes longer, so
// that the quads of 16 rows lie in different banks
template <int NB, bool GATED>
constexpr int kGradWidth = (GATED ? 8 : 16) * NB < 64 ? (GATED ? 8 : 16) * NB : 64;
template <typename TO, int NB, bool GATED>
constexpr int kGradRow = kGradWidth<NB, GATED> * (int)sizeof(TO) + 16;
template <typename TO, int NB, bool GATED>
constexpr int kGradBytes = (GATED ? 2 : 1) * 16 * kGradRow<TO, NB, GATED>;

// the sum over 16 neighbouring lanes, in all of them
template <int ROR>
__device__ __forceinline__ float plus_turned(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + ROR, 15, 15, false));
}
__device__ __forceinline__ float sum_of_16(float v) { return plus_turned<1>(plus_turned<2>(plus_turned<4>(plus_turned<8>(v)))); }

// What comes in of dy: lane's pieces of each pass, the passes of a row block one channel group after the other.
template <typename TO, int MB, int NB, bool GATED>
struct GradIn {
    static constexpr int W = kGradWidth<NB, GATED>, PER = 16 / (int)sizeof(TO), CPR = W / PER, IT = 16 * CPR / 64;
    static constexpr int NP = W / 16 * (GATED ? 2 : 1), CP = NB / NP, PASSES = MB * CP, AHEAD = PASSES < 4 ? PASSES : 4;
    static_assert(NB % NP == 0 && IT * 64 == 16 * CPR, "whole passes");
    typedef TO Piece __attribute__((ext_vector_type(PER)));
    Piece r[AHEAD][IT];
    // (rows of Cout numbers are whole pieces)
    __device__ __forceinline__ void fetch(const ActGradArgs &a, int pass, int64_t m0, int c0, int lane, bool whole)
    {
        const int row0 = lane / CPR, ch = lane % CPR * PER;
        const TO *dy = (const TO *)a.R + m0 * a.Cout + c0;
        const uint32_t from = (uint32_t)(row0 * a.Cout + ch);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int row = pass % MB * 16 + 64 / CPR * it, c = pass / MB * W;
            Piece x{};
            if (whole || (row + row0 < a.M - m0 && c + ch < a.Cout - c0)) x = *(const Piece *)(dy + (int64_t)row * a.Cout + c + from);
            r[pass % AHEAD][it] = x;
        }
    }
};

// acc: the products on top of the biases that they began with.  WHOLE: all of the part's rows and channels are there.
template <typename T, int MB, int NB, bool GATED, typename TO, int ACT, bool WHOLE>
__device__ __forceinline__ void epilogue_grad_part(const ActGradArgs &a, const typename Mul<T>::Acc (&acc)[MB][NB],
                                                   GradIn<TO, MB, NB, GATED> &in, int64_t m0, int c0, unsigned char *stage, int lane)
{
    using In = GradIn<TO, MB, NB, GATED>;
    using Piece = typename In::Piece;
    constexpr int BS = 16, NO = GATED ? 2 : 1, ES = (int)sizeof(TO), NP = In::NP, W = In::W, CPR = In::CPR, IT = In::IT;
    constexpr int SB = kGradRow<TO, NB, GATED>, PASSES = In::PASSES, AHEAD = In::AHEAD;
    static_assert(Mul<T>::BS == BS, "blocks of 16");
    typedef TO Quad __attribute__((ext_vector_type(4)));
    const int rl = lane % BS, cq = 4 * (lane / BS), ch = lane % CPR * In::PER, row0 = lane / CPR;
    const int left_rows = (int)min(a.M - m0, (int64_t)(BS * MB)), left = a.Cout - c0;
    TO *dz = (TO *)a.Y + m0 * NO * a.Cout + c0;
    const uint32_t to = (uint32_t)(row0 * NO * a.Cout + ch);
    f32x4 sum[NP];
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        const int i = pass % MB, jp = pass / MB * NP;  // (the rows of a group of channels one after the other: fewer sums at a time)
        if (i == 0)
#pragma unroll
            for (int j = 0; j < NP; ++j) sum[j] = f32x4{};
#pragma unroll
        for (int it = 0; it < IT; ++it) *(Piece *)(stage + (row0 + 64 / CPR * it) * SB + ch * ES) = in.r[pass % AHEAD][it];
        wave_sync();
        if (pass + AHEAD < PASSES) in.fetch(a, pass + AHEAD, m0, c0, lane, WHOLE);
        const bool live = WHOLE || BS * i + rl < left_rows;  // (rows past the end: a bias that is infinite would be NaN in the sums)
#pragma unroll
        for (int j = 0; j < NP; j += NO) {
            unsigned char *at = stage + rl * SB + (BS * j / NO + cq) * ES;
            const Quad g = *(const Quad *)at;
            Quad t0, t1{};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float z0 = acc[i][jp + j][e], gy = (float)g[e];
                float y, d, dz0;
                act_slope_fast<ACT>(z0, y, d);
                if constexpr (GATED) {
                    const float z1 = acc[i][jp + j + 1][e], dz1 = gy * y;
                    dz0 = gy * (z1 * d);
                    t1[e] = (TO)dz1;
                    sum[j + 1][e] += live ? dz1 : 0.f;
                } else {
                    dz0 = gy * d;
                }
                t0[e] = (TO)dz0;
                sum[j][e] += live ? dz0 : 0.f;
            }
            *(Quad *)at = t0;
            if constexpr (GATED) *(Quad *)(at + 16 * SB) = t1;
#pragma unroll
            for (int k = 0; k < NO; ++k) asm volatile("" : "+v"(sum[j + k]));  // (added now, not all at the end)
        }
        wave_sync();
#pragma unroll
        for (int k = 0; k < NO; ++k)
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                const int row = BS * i + 64 / CPR * it, c = pass / MB * W;
                const Piece x = *(const Piece *)(stage + k * (16 * SB) + (row0 + 64 / CPR * it) * SB + ch * ES);
                if (WHOLE || (row + row0 < left_rows && c + ch < left))
                    *(Piece *)(dz + ((int64_t)row * NO + k) * a.Cout + c + to) = x;
            }
        wave_sync();
        if (i == MB - 1 && a.sums) {
            float *sums = a.sums + (m0 / (BS * MB)) * NO * a.Cout + c0;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = sum_of_16(sum[j][e]);
                const int c = pass / MB * W + BS * (j / NO) + cq;
                if (rl == 0 && c < left) *(f32x4 *)(sums + (j % NO) * a.Cout + c) = v;
            }
        }
        __builtin_amdgcn_sched_barrier(0);  // (passes that the compiler draws into each other do not fit the registers)
    }
}
template <typename T, int MB, int NB, bool GATED, typename TO, int ACT>
__device__ __forceinline__ void epilogue_grad(const ActGradArgs &a, const typename Mul<T>::Acc (&acc)[MB][NB],
                                              GradIn<TO, MB, NB, GATED> &in, int64_t m0, int c0, unsigned char *stage, int lane)
{
    if (a.M - m0 >= 16 * MB && a.Cout - c0 >= 16 * NB / (GATED ? 2 : 1))
        epilogue_grad_part<T, MB, NB, GATED, TO, ACT, true>(a, acc, in, m0, c0, stage, lane);
    else if (a.M > m0)
        epilogue_grad_part<T, MB, NB, GATED, TO, ACT, false>(a, acc, in, m0, c0, stage, lane);
}
// (the first of them: before the multiplies are through)
template <typename TO, int MB, int NB, bool GATED>
__device__ __forceinline__ void epilogue_grad_fetch(const ActGradArgs &a, GradIn<TO, MB, NB, GATED> &in, int64_t m0, int c0, int lane)
{
    if (a.M <= m0) return;
    const bool whole = a.M - m0 >= 16 * MB && a.Cout - c0 >= 16 * NB / (GATED ? 2 : 1);
    if (whole) {
#pragma unroll
        for (int q = 0; q < in.AHEAD; ++q) in.fetch(a, q, m0, c0, lane, true);
    } else {
#pragma unroll
        for (int q = 0; q < in.AHEAD; ++q) in.fetch(a, q, m0, c0, lane, false);
    }
}

// A workgroup's tile of the gradients' small kernels: along the rows, or, with tiles_m, down the columns, a run of tiles on an XCD.
template <typename A>
__device__ __forceinline__ bool small_tile(const A &a, int &mt, int &nt)
{
    if (!a.tiles_m) {
        mt = (int)blockIdx.x / a.tiles_n;
        nt = (int)blockIdx.x - mt * a.tiles_n;
        return true;
    }
    const int tile = (int)(blockIdx.x % kXcds) * a.per_xcd + (int)(blockIdx.x / kXcds);
    nt = tile / a.tiles_m;
    mt = tile - nt * a.tiles_m;
    return tile < a.tiles;
}

// Small products: 32 rows of X by 32 rows of W a workgroup, whose eight wavefronts share the contraction: a wavefront takes
// every eighth stage through two LDS slots of its own, waits for nobody, and the eight sums are added up in LDS at the
// end, in an order that does not change.  What such a call takes is latency, an eighth of a row's length of it.  (Fetched in
// the operands' layout, straight into registers, 16 neighbouring lanes are on 16 rows, and the first-level cache serves
// them one by one: 160 x 1,280 x 1,280 7.6 us, 1 x 5,120 x 1,280 13 us.)
constexpr int kSmallLds = 8 * 2 * 64 * kRow;
template <typename T, bool GATED, typename TO, bool GRAD = false>
__global__ __launch_bounds__(512, 2) void act_small_kernel(const std::conditional_t<GRAD, ActGradArgs, ActArgs> a)
{
    using M = Mul<T>;
    constexpr int BS = M::BS, NW = 8, SR = 36, SLOT = 64 * kRow;
    constexpr bool SCALED = sizeof(T) == 1;
    static_assert(BS == 16, "two blocks of 16 rows of either");
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    constexpr int BO = GATED ? 16 : 32;
    int mt, nt;
    if constexpr (GRAD) {
        if (!small_tile(a, mt, nt)) return;
    } else {
        mt = (int)blockIdx.x / a.tiles_n;
        nt = (int)blockIdx.x - mt * a.tiles_n;
    }
    const int64_t m0 = (int64_t)mt * 32;
    const int n0 = nt * BO;
    const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rowbytes = a.Cin * (int)sizeof(T);
    // rows past the end read as zeros through the descriptors' range checks
    const __amdgpu_buffer_rsrc_t xres = rows_from(a.X, m0, a.M, rowbytes);
    const __amdgpu_buffer_rsrc_t wres0 = rows_from(a.W[0], n0, a.Cout, rowbytes);
    const __amdgpu_buffer_rsrc_t wres1 = GATED ? rows_from(a.W[1], n0, a.Cout, rowbytes) : wres0;
    unsigned char *mem = smem + wv * (2 * SLOT);
    const int lr = lane >> 3, lc = (lane & 7) ^ lr;
    const uint32_t off = (uint32_t)(lr * rowbytes + lc * 16), next = (uint32_t)(8 * rowbytes);
    const int stages = (rowbytes + kRow - 1) / kRow;
    auto issue = [&](int ks, int slot) __attribute__((always_inline)) {
        const bool live = ks * kRow + lc * 16 < rowbytes;
        const uint32_t o = off + (uint32_t)(ks * kRow);
#pragma unroll
        for (int l = 0; l < 4; ++l) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xres, (__attribute__((address_space(3))) void *)(mem + slot * SLOT + l * 1024), 16,
                                                     live ? o + l * next : kOob, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(GATED && l >= 2 ? wres1 : wres0,
                                                     (__attribute__((address_space(3))) void *)(mem + slot * SLOT + 4096 + l * 1024), 16,
                                                     live ? o + (GATED ? l & 1 : l) * next : kOob, 0, 0, 0);
        }
    };
    f32x4 acc[2][2] = {};
    int koff[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) koff[kk] = M::offset(lane, kk);
    if (wv < stages) issue(wv, 0);
    int slot = 0;
    for (int ks = wv; ks < stages; ks += NW) {
        const bool more = ks + NW < stages;
        if (more) issue(ks + NW, slot ^ 1);
        asm volatile("" ::: "memory");
        if (more)
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(8));  // all but the stage just asked for have landed
        else
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        const unsigned char *buf = mem + slot * SLOT + l16 * kRow;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            typename M::Frag x[2], w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[i] = M::read(buf + i * (16 * kRow), koff[kk]);
                w[i] = M::read(buf + 4096 + i * (16 * kRow), koff[kk]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[i][j] = M::mul(w[j], x[i], acc[i][j]);
        }
        // the slot's reads are done before it is asked to be filled again
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xc07f);  // (LDS operations only)
        asm volatile("" ::: "memory");
        slot ^= 1;
    }
    // the sums, in the place of the wavefront's slots
    float(*sums)[32][SR] = (float(*)[32][SR])smem;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) *(f32x4 *)&sums[wv][16 * i + l16][16 * j + 4 * lg] = acc[i][j];
    __syncthreads();
    const int row = (int)threadIdx.x >> 4, c = (int)threadIdx.x & 15;
    const int64_t m = m0 + row;
    if constexpr (GRAD) {
        constexpr int NO = GATED ? 2 : 1;
        float dz[32 / 16];  // of column c + 16 o; gated, of channel c: dz_0 and dz_1
        const bool live = m < a.M;
#pragma unroll
        for (int o = 0; o < BO / 16; ++o) {
            const int ch = n0 + c + 16 * o;
            float z[NO];
#pragma unroll
            for (int k = 0; k < NO; ++k) {
                z[k] = 0.f;
#pragma unroll
                for (int v = 0; v < NW; ++v) z[k] += sums[v][row][c + 16 * (GATED ? k : o)];
                if (a.bias[k] && ch < a.Cout) z[k] += a.bias[k][ch];
            }
            const float g = live && ch < a.Cout ? (float)((const TO *)a.R)[m * a.Cout + ch] : 0.f;
            float y = 0.f, d = 0.f;
            with_act(a.act, [&](auto act) __attribute__((always_inline)) { act_slope_fast<decltype(act)::value>(z[0], y, d); });
            if constexpr (GATED) {
                dz[0] = g * (z[1] * d);
                dz[1] = g * y;
            } else {
                dz[o] = g * d;
            }
#pragma unroll
            for (int k = 0; k < NO; ++k)
                if (live && ch < a.Cout) ((TO *)a.Y)[(m * NO + k) * a.Cout + ch] = (TO)dz[GATED ? k : o];
        }
        if (!a.sums) return;
        __syncthreads();
#pragma unroll
        for (int o = 0; o < 2; ++o) sums[0][row][c + 16 * o] = live ? dz[o] : 0.f;
        __syncthreads();
        if (threadIdx.x < 32) {
            float v = 0.f;
#pragma unroll
            for (int q = 0; q < 32; ++q) v += sums[0][q][threadIdx.x];
            const int o = (int)threadIdx.x >> 4, ch = n0 + c + (GATED ? 0 : 16 * o);
            if (ch < a.Cout) a.sums[((int64_t)mt * NO + (GATED ? o : 0)) * a.Cout + ch] = v;
        }
        return;
    }
    if (m >= a.M) return;
    const float xs = SCALED && a.xs ? a.xs[m] : 1.f;
#pragma unroll
    for (int o = 0; o < BO / 16; ++o) {
        const int ch = n0 + c + 16 * o;
        if (ch >= a.Cout) continue;
        float z[GATED ? 2 : 1];
#pragma unroll
        for (int k = 0; k < (GATED ? 2 : 1); ++k) {
            z[k] = 0.f;
#pragma unroll
            for (int v = 0; v < NW; ++v) z[k] += sums[v][row][c + 16 * (GATED ? k : o)];
            if (SCALED) z[k] = a.ws[k] ? z[k] * xs * a.ws[k][ch] : z[k] * xs;
            if (a.bias[k]) z[k] += a.bias[k][ch];
        }
        float y = 0.f;
        with_act(a.act, [&](auto act) __attribute__((always_inline)) { y = act_fast<decltype(act)::value>(z[0]); });
        if constexpr (GATED) y *= z[1];
        if (a.R) y += (float)((const TO *)a.R)[m * a.Cout + ch];
        ((TO *)a.Y)[m * a.Cout + ch] = (TO)y;
    }
}

// One tile a workgroup: two LDS slots, two to four workgroups on a compute unit, whose loads and barriers hide behind each
// other's multiplies; three slots, two stages ahead, for workgroups that are alone.  A workgroup of WVM x WVN wavefronts computes
// a (BS MB WVM) x (BS NB WVN) tile.
template <typename T, int MB, int NB, int WVM, int WVN, bool GATED, typename TO, bool GRAD = false, int SLOTS = 2>
__global__ __launch_bounds__(64 * WVM * WVN, 2) void act_tile_kernel(const std::conditional_t<GRAD, ActGradArgs, ActArgs> a)
{
    using M = Mul<T>;
    constexpr int BS = M::BS, NW = WVM * WVN;
    constexpr bool SCALED = sizeof(T) == 1;
    constexpr int BM = BS * MB * WVM, BN = BS * NB * WVN;
    constexpr int GA = BM / 8 / NW, GB = BN / 8 / NW;  // 8-row groups (one load instruction) per wavefront
    static_assert(GA * 8 * NW == BM && GB * 8 * NW == BN, "the wavefronts share the loads evenly");
    static_assert(SLOTS == 2 || SLOTS == 3, "one stage or two ahead");
    constexpr int ABYTES = BM * kRow, BUF = (BM + BN) * kRow;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ __attribute__((aligned(16))) float cols[2][BN];

    if constexpr (GRAD)
        if ((int)blockIdx.x >= a.groups) return turn_tile<T, 64 * NW>(a.turn, (int)blockIdx.x - a.groups, smem);
    // workgroup -> tile: XCD x (= blockIdx % 8) owns a contiguous run of tiles
    const int tile = (int)(blockIdx.x % kXcds) * a.per_xcd + (int)(blockIdx.x / kXcds);
    if (tile >= a.tiles) return;  // whole workgroup: no barrier has been reached yet
    const bool by_column = (GRAD || SLOTS > 2) && a.tiles_m;
    const int mt = by_column ? tile % a.tiles_m : tile / a.tiles_n, nt = by_column ? tile / a.tiles_m : tile - mt * a.tiles_n;
    const int64_t m0 = (int64_t)mt * BM;
    constexpr int BO = GATED ? BN / 2 : BN;  // output channels of the tile
    const int n0 = nt * BO;

    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wv / WVN, wn = wv - wm * WVN;
    const int rowbytes = a.Cin * (int)sizeof(T);

    // Lane l fetches chunk (l % 8) ^ (l / 8) of row l / 8 of an 8-row group.  Rows past the end and chunks past
    // c_in read as zeros through the descriptors' range checks.
    const int lr = lane >> 3, lc = (lane & 7) ^ lr;
    const __amdgpu_buffer_rsrc_t xres = rows_from(a.X, m0, a.M, rowbytes);
    const __amdgpu_buffer_rsrc_t wres0 = rows_from(a.W[0], n0, a.Cout, rowbytes);
    const __amdgpu_buffer_rsrc_t wres1 = GATED ? rows_from(a.W[1], n0, a.Cout, rowbytes) : wres0;
    const uint32_t xoff = (uint32_t)((wv * (8 * GA) + lr) * rowbytes + lc * 16);
    int stage_no = 0, to = 0;  // the next stage that is asked for, and its slot
    auto issue_stage = [&]() __attribute__((always_inline)) {
        const bool live = stage_no * kRow + lc * 16 < rowbytes;
        unsigned char *as = smem + to * BUF + wv * (GA * 1024);
        unsigned char *bs = smem + to * BUF + ABYTES + wv * (GB * 1024);
#pragma unroll
        for (int l = 0; l < GA; ++l)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                xres, (__attribute__((address_space(3))) void *)(as + l * 1024), 16,
                live ? xoff + (uint32_t)(8 * l * rowbytes + stage_no * kRow) : kOob, 0, 0, 0);
#pragma unroll
        for (int l = 0; l < GB; ++l) {
            const int r = wv * (8 * GB) + 8 * l;  // (an 8-row group is within a block)
            const uint32_t off = (uint32_t)((channel_of<BS, GATED>(r) + lr) * rowbytes + lc * 16 + stage_no * kRow);
            if (GATED && set_of<BS, GATED>(r))
                __builtin_amdgcn_raw_ptr_buffer_load_lds(wres1, (__attribute__((address_space(3))) void *)(bs + l * 1024), 16,
                                                         live ? off : kOob, 0, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(wres0, (__attribute__((address_space(3))) void *)(bs + l * 1024), 16,
                                                         live ? off : kOob, 0, 0, 0);
        }
        ++stage_no;
        to = SLOTS == 2 ? to ^ 1 : to + 1 == SLOTS ? 0 : to + 1;
    };
    const int stages = (rowbytes + kRow - 1) / kRow;
    issue_stage();
#pragma unroll
    for (int s = 1; s < SLOTS - 1; ++s)
        if (s < stages) issue_stage();
    for (int r = threadIdx.x; r < BN; r += 64 * NW) {
        float b, s = 1.f;
        column<BS, GATED, SCALED>(a, n0, r, b, s);
        cols[0][r] = b;
        if constexpr (SCALED) cols[1][r] = s;
    }

    typename M::Acc acc[MB][NB];
    if constexpr (GRAD) __syncthreads();
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        typename M::Acc first{};
        if constexpr (GRAD) first = *(const f32x4 *)(&cols[0][wn * BS * NB] + BS * j + 4 * (lane / BS));
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[i][j] = first;
    }
    int koff[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) koff[kk] = M::offset(lane, kk);
    const int abase = (wm * BS * MB + lane % BS) * kRow, bbase = ABYTES + (wn * BS * NB + lane % BS) * kRow;
    int slot = 0;
    for (int ks = 0; ks < stages; ++ks) {
        // This wavefront's loads of stage ks have landed (those of the one behind it may be on their way) and its reads of
        // stage ks - 1 are done; behind the barrier everybody's are, and the slot of stage ks - 1 is free.
        asm volatile("" ::: "memory");
        if (SLOTS > 2 && ks + 1 < stages)
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(GA + GB));
        else
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (ks + SLOTS - 1 < stages) issue_stage();
        const unsigned char *buf = smem + slot * BUF;
        slot = SLOTS == 2 ? slot ^ 1 : slot + 1 == SLOTS ? 0 : slot + 1;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            typename M::Frag af[MB], bf[NB];
#pragma unroll
            for (int i = 0; i < MB; ++i) af[i] = M::read(buf + abase + i * (BS * kRow), koff[kk]);
#pragma unroll
            for (int j = 0; j < NB; ++j) bf[j] = M::read(buf + bbase + j * (BS * kRow), koff[kk]);
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < MB; ++i) acc[i][j] = M::mul(bf[j], af[i], acc[i][j]);
        }
    }
    // everybody is through with the ring: it becomes the staging area
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    constexpr int CHP = BS * NB / (GATED ? 2 : 1);  // output channels of the part
    if constexpr (GRAD) {
        static_assert(NW * kGradBytes<TO, NB, GATED> <= 2 * BUF, "the staging area fits in the ring");
        GradIn<TO, MB, NB, GATED> in;
        epilogue_grad_fetch(a, in, m0 + wm * BS * MB, n0 + wn * CHP, lane);
        with_act(a.act, [&](auto act) __attribute__((always_inline)) {
            epilogue_grad<T, MB, NB, GATED, TO, decltype(act)::value>(a, acc, in, m0 + wm * BS * MB, n0 + wn * CHP,
                                                                      smem + wv * kGradBytes<TO, NB, GATED>, lane);
        });
        return;
    }
    // all of the part at once, or a block of rows, or half of its channels
    constexpr int per = NW * BS * (CHP + 4) * 4;
    constexpr int MP = MB * per <= 2 * BUF ? MB : 1, NP = MP * per <= 2 * BUF ? NB : NB / 2;
    constexpr int SR = CHP * NP / NB + 4;
    static_assert(NW * BS * MP * SR * 4 <= 2 * BUF, "the staging area fits in the ring");
    if constexpr (!GRAD)
        epilogue<T, MB, NB, MP, NP, GATED, TO, SCALED>(a, acc, m0 + wm * BS * MB, n0 + wn * CHP, &cols[0][wn * BS * NB],
                                                       &cols[1][wn * BS * NB], (float *)smem + wv * (BS * MP * SR), lane);
}

// The same for the persistent kernels, in an area of its own beside the ring (the ring goes on loading meanwhile): 32 rows x 32
// output channels at a time (16 rows in fp32), in the output's type.  The residual comes the same way in, one or two passes
// ahead, and its sum is rounded once.
constexpr int kPassBytes = 2304;  // of a wavefront
template <typename T, int MB, int NB, bool GATED, typename TO, bool SCALED, int ACT, bool RES>
__device__ __forceinline__ void epilogue_beside(const ActArgs &a, const typename Mul<T>::Acc (&acc)[MB][NB], int64_t m0, int c0,
                                                const float *bias, const float *wscale, const float (&xscale)[MB],
                                                unsigned char *stage, int lane)
{
    using M = Mul<T>;
    constexpr int BS = M::BS, NO = GATED ? 2 : 1, ES = (int)sizeof(TO);
    constexpr int ROWS = 64 / ES > 16 ? 32 : 16, MP = ROWS / BS, NP = 32 * NO / BS;  // of a pass
    static_assert(MP >= 1 && MB % MP == 0 && NB % NP == 0, "whole passes");
    constexpr int SB = 32 * ES + (ES == 2 ? 8 : 16);  // bytes of a staged row
    static_assert(ROWS * SB <= kPassBytes, "the staging area holds a pass");
    constexpr int PER = 16 / ES, CPR = 32 / PER, IT = ROWS * CPR / 64;  // channels of a piece, pieces of a row, of a lane
    constexpr int PASSES = (MB / MP) * (NB / NP), AHEAD = GATED && SCALED ? 1 : 2;
    typedef TO Piece __attribute__((ext_vector_type(PER)));
    typedef TO Quad __attribute__((ext_vector_type(4)));
    typedef uint32_t Half __attribute__((ext_vector_type(2)));
    const int rl = lane % BS, cq = 4 * (lane / BS);
    const bool whole = a.Cout % PER == 0;
    // this lane's piece `it` of a pass: row and channel within it, and their place from the part's first number on
    auto row_of = [&](int it) __attribute__((always_inline)) { return (lane + 64 * it) / CPR; };
    const int ch = lane % CPR * PER;
    const int left_rows = (int)min(a.M - m0, (int64_t)(BS * MB)), left = a.Cout - c0;
    auto row_at = [&](int pass) __attribute__((always_inline)) { return pass / (NB / NP) * ROWS; };
    auto channel_at = [&](int pass) __attribute__((always_inline)) { return pass % (NB / NP) * 32; };
    const int64_t base = m0 * a.Cout + c0;
    auto there = [&](int pass, int it) __attribute__((always_inline)) {
        return row_at(pass) + row_of(it) < left_rows && channel_at(pass) + ch < left;
    };
    auto offset = [&](int pass, int it) __attribute__((always_inline)) {
        return (uint32_t)((row_at(pass) + row_of(it)) * a.Cout + channel_at(pass) + ch);
    };
    Piece r[AHEAD][IT];
    auto fetch = [&](int pass) __attribute__((always_inline)) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            Piece x{};
            if (there(pass, it)) {
                const TO *from = (const TO *)a.R + base + offset(pass, it);
                if (whole) {
                    x = *(const Piece *)from;
                } else {
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (channel_at(pass) + ch + e < left) x[e] = from[e];
                }
            }
            r[pass % AHEAD][it] = x;
        }
    };
    // (8-byte accesses: a staged row of bf16 is 72 bytes)
    auto put_piece = [&](unsigned char *at, const Piece &x) __attribute__((always_inline)) {
        if constexpr (ES == 2) {
            const i32x4 w = __builtin_bit_cast(i32x4, x);
            *(Half *)at = Half{(uint32_t)w[0], (uint32_t)w[1]};
            *(Half *)(at + 8) = Half{(uint32_t)w[2], (uint32_t)w[3]};
        } else {
            *(Piece *)at = x;
        }
    };
    auto get_piece = [&](const unsigned char *at) __attribute__((always_inline)) {
        if constexpr (ES == 2) {
            const Half lo = *(const Half *)at, hi = *(const Half *)(at + 8);
            return __builtin_bit_cast(Piece, (i32x4){(int)lo[0], (int)lo[1], (int)hi[0], (int)hi[1]});
        } else {
            return *(const Piece *)at;
        }
    };
    if constexpr (RES) {
#pragma unroll
        for (int p = 0; p < AHEAD && p < PASSES; ++p) fetch(p);
    }
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        const int ip = pass / (NB / NP) * MP, jp = pass % (NB / NP) * NP;
        if constexpr (RES) {
#pragma unroll
            for (int it = 0; it < IT; ++it) put_piece(stage + row_of(it) * SB + ch * ES, r[pass % AHEAD][it]);
            wave_sync();
            if (pass + AHEAD < PASSES) fetch(pass + AHEAD);
        }
#pragma unroll
        for (int j = 0; j < NP; j += NO)
#pragma unroll
            for (int q = 0; q < M::QUADS; ++q) {
                f32x4 b[NO], s[NO];
#pragma unroll
                for (int k = 0; k < NO; ++k) {
                    const int at = BS * (jp + j + k) + 8 * q + cq;
                    b[k] = *(const f32x4 *)(bias + at);
                    if constexpr (SCALED) s[k] = *(const f32x4 *)(wscale + at);
                }
#pragma unroll
                for (int i = 0; i < MP; ++i) {
                    f32x4 y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float z[NO];
#pragma unroll
                        for (int k = 0; k < NO; ++k) {
                            z[k] = acc[ip + i][jp + j + k][4 * q + e];
                            if constexpr (SCALED) z[k] = z[k] * xscale[ip + i] * s[k][e];
                            z[k] += b[k][e];
                        }
                        y[e] = act_fast<ACT>(z[0]);
                        if constexpr (GATED) y[e] *= z[1];
                    }
                    unsigned char *at = stage + (BS * i + rl) * SB + (BS * j / NO + 8 * q + cq) * ES;
                    Quad t;
                    if constexpr (RES) {
                        t = *(const Quad *)at;
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] += (float)t[e];
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) t[e] = (TO)y[e];
                    *(Quad *)at = t;
                }
            }
        wave_sync();
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const Piece x = get_piece(stage + row_of(it) * SB + ch * ES);
            if (there(pass, it)) {
                TO *to = (TO *)a.Y + base + offset(pass, it);
                if (whole) {
                    *(Piece *)to = x;
                } else {
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (channel_at(pass) + ch + e < left) to[e] = x[e];
                }
            }
        }
        wave_sync();
    }
}

// Large products: persistent workgroups of eight wavefronts (two per SIMD), at most one per compute unit, on 256 x 256 tiles.
// The stages of successive tiles are one stream through two LDS slots: while a tile's last stage is multiplied out, the
// next tile's first one is on its way into the other slot.  A wavefront's part is MB x NB blocks; its multiplies run in
// halves (X blocks [0, HB), then [HB, MB)) so that one set of fragments, refilled in place under the multiplies, is
// enough beside the accumulators: LDS reads and the next stage's loads sit between the matrix instructions by hand.
template <typename T, int MB, int NB, bool GATED, typename TO, int ACT>
__global__ __launch_bounds__(512, 2) void act_stream_kernel(const ActArgs a)
{
    using M = Mul<T>;
    constexpr int BS = M::BS, NW = 8, WVM = 4, WVN = 2;
    constexpr bool SCALED = sizeof(T) == 1;
    constexpr int BM = BS * MB * WVM, BN = BS * NB * WVN, BO = GATED ? BN / 2 : BN;
    static_assert(BM == 256 && BN == 256, "tiles of 256 x 256");
    constexpr int GA = BM / 8 / NW, GB = BN / 8 / NW, NL = GA + GB;
    constexpr int ABYTES = BM * kRow, BUF = (BM + BN) * kRow;
    constexpr int SLOT = BUF, CHP = BS * NB / (GATED ? 2 : 1), COLS = BS * NB;  // output channels, columns of the part
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    // behind the ring, of each wavefront: the epilogue's staging area; bias and scale of its columns
    unsigned char *own = smem + 2 * SLOT + (threadIdx.x >> 6) * (kPassBytes + 2 * COLS * 4);
    float *cols = (float *)(own + kPassBytes);

    // workgroup -> tiles: XCD x (= blockIdx % 8) owns tiles [x * per_xcd, (x + 1) * per_xcd), which its workgroups take in
    // turn; column tiles are numbered in panels of a.panel of them, row tile by row tile (see act_panel())
    const int xcd = (int)(blockIdx.x % kXcds), nper = (int)(gridDim.x / kXcds);
    const int t_end = min((xcd + 1) * a.per_xcd, a.tiles);
    int tile = xcd * a.per_xcd + (int)(blockIdx.x / kXcds);
    if (tile >= t_end) return;  // whole workgroup: no barrier has been reached yet
    const int tiles_m = a.tiles / a.tiles_n;
    struct Place {
        int first, c, mt;  // column tile first + c, row tile mt
    };
    const int dmt = nper / a.panel, dc = nper - dmt * a.panel;
    auto step = [&](Place &p) __attribute__((always_inline)) {
        p.c += dc;
        p.mt += dmt;
        if (p.c >= a.panel) {
            p.c -= a.panel;
            ++p.mt;
        }
        while (p.mt >= tiles_m) {
            p.mt -= tiles_m;
            p.first += a.panel;
        }
    };
    Place place;
    {
        const int row = tile / a.panel, pn = row / tiles_m;
        place = {pn * a.panel, tile - row * a.panel, row - pn * tiles_m};
    }

    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wv / WVN, wn = wv - wm * WVN;
    const int rowbytes = a.Cin * (int)sizeof(T);
    const int stages = (rowbytes + kRow - 1) / kRow;
    const int lr = lane >> 3, lc = (lane & 7) ^ lr;
    // (the empty asm keeps an offset in a register: recomputing it would put multiplies between the matrix instructions)
    int xoff = (wv * (8 * GA) + lr) * rowbytes + lc * 16;
    asm volatile("" : "+v"(xoff));
    int woff[GB];
#pragma unroll
    for (int l = 0; l < GB; ++l) {
        woff[l] = (channel_of<BS, GATED>(wv * (8 * GB) + 8 * l) + lr) * rowbytes + lc * 16;
        asm volatile("" : "+v"(woff[l]));
    }
    const int group_bytes = 8 * rowbytes;

    // ---- the load side, up to two stages ahead of the multiplies
    int ld_tile = tile, su_ks = 0, ld_gs = 0;
    Place ld_place = place;
    bool ld_has = true, ld_live = false;
    __amdgpu_buffer_rsrc_t xres, wres0, wres1;
    uint32_t ld_x = 0, ld_w = 0;
    unsigned char *ld_as = smem, *ld_bs = smem;
    auto ld_open = [&]() __attribute__((always_inline)) {
        xres = rows_from(a.X, (int64_t)ld_place.mt * BM, a.M, rowbytes);
        const int n0 = (ld_place.first + ld_place.c) * BO;
        wres0 = rows_from(a.W[0], n0, a.Cout, rowbytes);
        wres1 = GATED ? rows_from(a.W[1], n0, a.Cout, rowbytes) : wres0;
        su_ks = 0;
    };
    // Past the workgroup's last tile every lane of the loads is an out-of-range one: no traffic, the same number of loads in
    // flight, no branch among the multiplies.
    auto stage_setup = [&]() __attribute__((always_inline)) {
        if (su_ks == stages) {
            ld_tile += nper;
            ld_has = ld_tile < t_end;
            if (ld_has) step(ld_place);
            ld_open();
        }
        ld_live = ld_has && su_ks * kRow + lc * 16 < rowbytes;
        ld_x = ld_w = (uint32_t)(su_ks * kRow);
        ++su_ks;
        const int slot = ld_gs++ & 1;
        ld_as = smem + slot * SLOT + wv * (GA * 1024);
        ld_bs = smem + slot * SLOT + ABYTES + wv * (GB * 1024);
    };
    auto issue_one = [&](int l) __attribute__((always_inline)) {
        if (l < GA) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xres, (__attribute__((address_space(3))) void *)(ld_as + l * 1024), 16,
                                                     ld_live ? (uint32_t)xoff + ld_x : kOob, 0, 0, 0);
            ld_x += group_bytes;
        } else {
            // (a wavefront's 32 rows of W: one block of 32, or two of 16)
            const bool second = GATED && (BS == 32 ? (wv & 1) : (l - GA) >= GB / 2);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(second ? wres1 : wres0,
                                                     (__attribute__((address_space(3))) void *)(ld_bs + (l - GA) * 1024), 16,
                                                     ld_live ? (uint32_t)woff[l - GA] + ld_w : kOob, 0, 0, 0);
        }
    };
    static_assert(GB * 8 == 32, "a wavefront loads 32 rows of W");

    typename M::Acc acc[MB][NB];
    auto clear_acc = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = typename M::Acc{};
    };
    clear_acc();
    int koff[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) koff[kk] = M::offset(lane, kk);
    const int abase = (wm * BS * MB + lane % BS) * kRow, bbase = ABYTES + (wn * BS * NB + lane % BS) * kRow;
    constexpr int HB = MB / 2, NMH = HB * NB;  // X blocks and multiplies of a half
    typename M::Frag af[MB], bf[NB];
    // the loads of the next stage are spread over this many multiplies from the barrier on (of 4 NMH between two of them)
    constexpr int TAIL = NMH, kSpread = 5 * NMH / 2;
    auto read_a = [&](const unsigned char *base, int kk, int i) __attribute__((always_inline)) {
        af[i] = M::read(base + abase + i * (BS * kRow), koff[kk]);
    };
    auto read_b = [&](const unsigned char *base, int kk, int j) __attribute__((always_inline)) {
        bf[j] = M::read(base + bbase + j * (BS * kRow), koff[kk]);
    };
    auto loads_at = [&](int g, bool do_loads) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < NL; ++q)
            if (do_loads && (q * kSpread) / NL == g) {
                issue_one(q);
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    // first half of a sub-step; fetches the second half's X fragments
    auto half1 = [&](const unsigned char *base, int kk, int g0) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < NMH; ++m) {
            loads_at(g0 + m, true);
#pragma unroll
            for (int r = 0; r < HB; ++r)
                if ((r * (NMH / 2)) / HB == m) {
                    read_a(base, kk, HB + r);
                    __builtin_amdgcn_sched_barrier(0);
                }
            // (back and forth: one operand stays the same from one multiply to the next)
            const int j = m / HB, i0 = m - j * HB, i = j & 1 ? HB - 1 - i0 : i0;
            acc[i][j] = M::mul(bf[j], af[i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // second half; fetches the next sub-step's first X fragments and, column by column, its W fragments
    auto half2 = [&](const unsigned char *nbase, int nkk, int g0, bool do_loads) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < NMH; ++m) {
            loads_at(g0 + m, do_loads);
            const int j = m / HB, i0 = m - j * HB, i = j & 1 ? HB - 1 - i0 : i0;
            if (i0 == 0 && j > 0) {
                read_b(nbase, nkk, j - 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (i0 == HB - 1 && j < HB) {
                read_a(nbase, nkk, j);
                __builtin_amdgcn_sched_barrier(0);
            }
            acc[HB + i][j] = M::mul(bf[j], af[HB + i], acc[HB + i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        read_b(nbase, nkk, NB - 1);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto issue_tail_loads = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < NL; ++q)
            if ((q * kSpread) / NL < TAIL) issue_one(q);
    };

    ld_open();
    stage_setup();
#pragma unroll
    for (int l = 0; l < NL; ++l) issue_one(l);
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    stage_setup();
    issue_tail_loads();
#pragma unroll
    for (int i = 0; i < HB; ++i) read_a(smem, 0, i);
#pragma unroll
    for (int j = 0; j < NB; ++j) read_b(smem, 0, j);

    int cs = 0;  // stages multiplied out so far
    for (;;) {
        const int64_t m0 = (int64_t)place.mt * BM;
        const int n0 = (place.first + place.c) * BO;
        // the tile's biases and scales: fetched now, put into LDS before the epilogue
        float cb[COLS / 64], csc[COLS / 64];
#pragma unroll
        for (int u = 0; u < COLS / 64; ++u) column<BS, GATED, SCALED>(a, n0, wn * COLS + lane + 64 * u, cb[u], csc[u]);
        // (and the scales of its rows: a load in the epilogue would be waited for behind the stores)
        float xs[MB];
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            const int64_t m = m0 + BS * (wm * MB + i) + lane % BS;
            xs[i] = SCALED && a.xs ? a.xs[m < a.M ? m : a.M - 1] : 1.f;
        }
        for (int ks = 0; ks < stages; ++ks, ++cs) {
            const unsigned char *bufc = smem + (cs & 1) * SLOT, *bufn = smem + ((cs + 1) & 1) * SLOT;
            // (the younger of two wavefronts on a SIMD goes first here, so that they draw apart)
            if (wv >= NW / 2) __builtin_amdgcn_s_setprio(1);
            half1(bufc, 0, TAIL);
            half2(bufc, 1, TAIL + NMH, true);
            __builtin_amdgcn_s_setprio(0);
            stage_setup();
            half1(bufc, 1, TAIL + 2 * NMH);
            // this wavefront's loads of the next stage have landed and its reads of this slot are done; behind the barrier
            // everybody's are
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            half2(bufn, 0, 0, true);
        }
        int le = lane;
        asm volatile("" : "+v"(le));  // (or the epilogue's addresses are kept alive through the main loop)
#pragma unroll
        for (int u = 0; u < COLS / 64; ++u) {
            cols[le + 64 * u] = cb[u];
            if constexpr (SCALED) cols[COLS + le + 64 * u] = csc[u];
        }
        wave_sync();
        if (a.R)
            epilogue_beside<T, MB, NB, GATED, TO, SCALED, ACT, true>(a, acc, m0 + wm * BS * MB, n0 + wn * CHP, cols, cols + COLS,
                                                                     xs, own, le);
        else
            epilogue_beside<T, MB, NB, GATED, TO, SCALED, ACT, false>(a, acc, m0 + wm * BS * MB, n0 + wn * CHP, cols, cols + COLS,
                                                                      xs, own, le);
        tile += nper;
        if (tile >= t_end) break;
        step(place);
        clear_acc();
    }
}
constexpr int kStreamLds = 2 * 512 * kRow + 8 * (kPassBytes + 2 * 128 * 4);

}  // namespace
}  // namespace dsattn
