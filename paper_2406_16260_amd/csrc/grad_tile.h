// The weights' gradient on the matrix cores: dW = dz^T X, a contraction over the rows of both operands, which lie row by row
// in memory.  A stage is KS rows (64 bf16, 32 fp32) of a tile's columns, straight from memory into LDS; a lane's fragment,
// consecutive rows of one column, comes out of it transposed: in 16 bits by ds_read_b64_tr_b16, which hands the 4 x 16
// numbers that 16 lanes read to them column by column; in 32 bits number by number.  16-byte chunks are swizzled by
// their row so that the rows of a read lie in different banks.
#pragma once

#include "act_tile.h"

namespace dsattn {
namespace {

// Column sums of parts of the rows, to be added up: by workgroups of their own behind those of another kernel.
struct JoinArgs {
    const void *sums;   // [parts][No]
    bool half;          // of bf16: few rows of dY itself
    float *db[2];       // [Cout] each, or null
    int32_t parts, Cout, No, groups;  // groups: workgroups, of 16 columns each
};

struct GradWArgs {
    const void *dz, *X;  // [M][No], [M][Cin]
    void *dW[2];         // [Cout][Cin] each, or null
    float *partial;      // [splits][No][Cin] where there are several
    int64_t M;
    int32_t Cin, Cout, No;               // No: n_w Cout
    int32_t tiles_n, tiles, items, per_xcd;  // column tiles (of X); all; tiles * splits; ceil(items / 8)
    int32_t stages;                      // of a split
    int32_t groups;                      // workgroups of the product; those behind join the column sums
    JoinArgs join;
    // 256 x 256 tiles: column tiles that are not half empty; items of an XCD of those and of the others
    int32_t whole, whole_xcd, rest_xcd;
};

// Four numbers of a column, transposed by the LDS.  (The pointer is restrict for what the compiler makes of it: a read that it
// knows nothing about waits for all loads into LDS that are on their way, and the kernels' own waits do that where it is needed.)
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ s16x4 read_turned(__attribute__((address_space(3))) s16x4 *__restrict at)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(at);
}

// Columns of an operand, W of them a tile.
template <typename T, int W>
struct Cols {
    static constexpr int ES = (int)sizeof(T), KS = kRow / ES, RB = W * ES, CPR = RB / 16, PER = 16 / ES;
    static constexpr int RPI = 64 / CPR;  // rows of a load instruction
    static_assert(CPR * RPI == 64 && (ES == 2 ? CPR >= 4 : CPR >= 8), "whole rows");
    using Frag = typename Mul<T>::Frag;
    // where chunk c of row k lies: position c ^ swizzle(k)
    static __device__ __forceinline__ int swizzle(int k)
    {
        if constexpr (ES == 4) return 4 * ((k >> 2) & (CPR >= 16 ? 3 : 1));
        return 2 * (CPR >= 16 ? (k & 3) | ((k >> 1) & 4) : CPR == 8 ? k & 3 : (k >> 1) & 1);
    }
    // a lane's place within row 0 of a fragment of columns 16 blk .., and the row (of the first read)
    static __device__ __forceinline__ int row(int lane) { return ES == 4 ? 4 * (lane >> 4) : 8 * (lane >> 4) + ((lane & 15) >> 2); }
    static __device__ __forceinline__ int place(int lane, int blk)
    {
        const int l = lane & 15;
        if constexpr (ES == 4) return ((4 * blk + (l >> 2)) ^ swizzle(row(lane))) * 16 + (l & 3) * 4;
        return ((2 * blk + ((l & 3) >> 1)) ^ swizzle(row(lane))) * 16 + (l & 1) * 8;
    }
    static __device__ __forceinline__ Frag read(const unsigned char *at)
    {
        if constexpr (ES == 4) {
            Frag f;
#pragma unroll
            for (int s = 0; s < 4; ++s) f[s] = *(const float *)(at + s * RB);
            return f;
        } else {
            const s16x4 lo = read_turned((__attribute__((address_space(3))) s16x4 *)at);
            const s16x4 hi = read_turned((__attribute__((address_space(3))) s16x4 *)(at + 4 * RB));
            return __builtin_bit_cast(Frag, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Rows k.. of columns c0.. of a matrix of `rows` x `cols`: what lies past its last row reads as zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t cols_from(const void *p, int64_t k, int64_t rows, int rowbytes, int c0bytes)
{
    const int64_t left = max((int64_t)0, (rows - k) * rowbytes - c0bytes);
    return __builtin_amdgcn_make_buffer_rsrc((void *)((const unsigned char *)p + k * rowbytes + c0bytes), 0,
                                             (int)min(left, (int64_t)0x7fffffff), 0x00020000);
}

// What a lane's accumulator holds goes out: four neighbouring channels of a row.
template <typename T>
__device__ __forceinline__ void grad_w_store(const GradWArgs &a, int split, bool parts, int o, int c, const f32x4 &v)
{
    if (o >= a.No || c >= a.Cin) return;
    if (parts) {
        *(f32x4 *)(a.partial + ((int64_t)split * a.No + o) * a.Cin + c) = v;
        return;
    }
    T *to = (T *)(o < a.Cout ? a.dW[0] : a.dW[1]);
    if (!to) return;
    typedef T Quad __attribute__((ext_vector_type(4)));
    Quad q;
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = (T)v[e];
    *(Quad *)(to + (int64_t)(o < a.Cout ? o : o - a.Cout) * a.Cin + c) = q;
}

// 16 columns a workgroup; `part`: 16 floats for every 16 threads and one more.
template <int THREADS>
__device__ __forceinline__ void join_columns(const JoinArgs &a, int block, float *part)
{
    constexpr int W = THREADS / 16;
    const int l = threadIdx.x & 15, w = threadIdx.x >> 4, c = block * 16 + l;
    float v = 0.f;
    if (c < a.No) {
        if (a.half) {
#pragma unroll 8
            for (int p = w; p < a.parts; p += W) v += (float)((const __bf16 *)a.sums)[(int64_t)p * a.No + c];
        } else {
#pragma unroll 8
            for (int p = w; p < a.parts; p += W) v += ((const float *)a.sums)[(int64_t)p * a.No + c];
        }
    }
    part[w * 17 + l] = v;
    __syncthreads();
    for (int h = W / 2; h > 0; h >>= 1) {
        if (w < h) part[w * 17 + l] += part[(w + h) * 17 + l];
        __syncthreads();
    }
    float *to = c < a.Cout ? a.db[0] : a.db[1];
    if (w == 0 && c < a.No && to) to[c < a.Cout ? c : c - a.Cout] = part[l];
}
__global__ __launch_bounds__(1024) void grad_join_kernel(const JoinArgs a)
{
    __shared__ float part[64 * 17];
    join_columns<1024>(a, (int)blockIdx.x, part);
}

// One tile of one split a workgroup, two LDS slots, two workgroups on a compute unit.
template <typename T, int MB, int NB, int WVM, int WVN, int SLOTS = 2>
__global__ __launch_bounds__(64 * WVM * WVN, 2) void grad_w_tile_kernel(const GradWArgs a)
{
    using M = Mul<T>;
    constexpr int NW = WVM * WVN, BM = 16 * MB * WVM, BN = 16 * NB * WVN;
    using A = Cols<T, BM>;
    using B = Cols<T, BN>;
    constexpr int KS = A::KS, GA = BM / 8 / NW, GB = BN / 8 / NW;
    static_assert(GA * 8 * NW == BM && GB * 8 * NW == BN, "the wavefronts share the loads evenly");
    constexpr int ABYTES = BM * kRow, BUF = (BM + BN) * kRow;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    // workgroup -> split and tile: XCD x (= blockIdx % 8) owns a contiguous run of items, the tiles of a split one after the other
    if ((int)blockIdx.x >= a.groups) return join_columns<64 * NW>(a.join, (int)blockIdx.x - a.groups, (float *)smem);
    const int item = (int)(blockIdx.x % kXcds) * a.per_xcd + (int)(blockIdx.x / kXcds);
    if (item >= a.items) return;  // whole workgroup: no barrier has been reached yet
    const int split = item / a.tiles, tile = item - split * a.tiles;
    const int mt = tile / a.tiles_n, o0 = mt * BM, c0 = (tile - mt * a.tiles_n) * BN;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv / WVN, wn = wv - wm * WVN;
    const int zbytes = a.No * A::ES, xbytes = a.Cin * B::ES;
    uint32_t aoff[GA], boff[GB];
#pragma unroll
    for (int l = 0; l < GA; ++l) {
        const int r = (wv * GA + l) * A::RPI + lane / A::CPR, c = (lane % A::CPR) ^ A::swizzle(r);
        aoff[l] = o0 + c * A::PER < a.No ? (uint32_t)(r * zbytes + c * 16) : kOob;
    }
#pragma unroll
    for (int l = 0; l < GB; ++l) {
        const int r = (wv * GB + l) * B::RPI + lane / B::CPR, c = (lane % B::CPR) ^ B::swizzle(r);
        boff[l] = c0 + c * B::PER < a.Cin ? (uint32_t)(r * xbytes + c * 16) : kOob;
    }
    const int64_t first = (int64_t)split * a.stages * KS;
    const int stages = (int)min((int64_t)a.stages, (a.M - first + KS - 1) / KS);
    // (without the casts of the offsets the compiler's host pass has no stub of this kernel)
    auto issue_stage = [&](int ks, int to) __attribute__((always_inline)) {
        unsigned char *as = smem + to * BUF + wv * (GA * 1024), *bs = smem + to * BUF + ABYTES + wv * (GB * 1024);
        const int64_t k0 = first + (int64_t)ks * KS;
        const __amdgpu_buffer_rsrc_t zres = cols_from(a.dz, k0, a.M, zbytes, o0 * A::ES);
        const __amdgpu_buffer_rsrc_t xres = cols_from(a.X, k0, a.M, xbytes, c0 * B::ES);
#pragma unroll
        for (int l = 0; l < GA; ++l)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(zres, (__attribute__((address_space(3))) void *)(as + l * 1024), 16,
                                                     (uint32_t)aoff[l], 0, 0, 0);
#pragma unroll
        for (int l = 0; l < GB; ++l)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xres, (__attribute__((address_space(3))) void *)(bs + l * 1024), 16,
                                                     (uint32_t)boff[l], 0, 0, 0);
    };
    typename M::Acc acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = typename M::Acc{};
    int ap[MB], bp[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) ap[i] = A::row(lane) * A::RB + A::place(lane, wm * MB + i);
#pragma unroll
    for (int j = 0; j < NB; ++j) bp[j] = ABYTES + B::row(lane) * B::RB + B::place(lane, wn * NB + j);
    constexpr int AHEAD = SLOTS - 1;
    static_assert(SLOTS <= 3, "one stage or two ahead");
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
        if (s < stages) issue_stage(s, s);
    int slot = 0, next = AHEAD;
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
        if (ks + AHEAD < stages) issue_stage(ks + AHEAD, next);
        const unsigned char *buf = smem + slot * BUF;
        slot = slot + 1 == SLOTS ? 0 : slot + 1;
        next = next + 1 == SLOTS ? 0 : next + 1;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            typename M::Frag af[MB], bf[NB];
#pragma unroll
            for (int i = 0; i < MB; ++i) af[i] = A::read(buf + kk * (KS / 2 * A::RB) + ap[i]);
#pragma unroll
            for (int j = 0; j < NB; ++j) bf[j] = B::read(buf + kk * (KS / 2 * B::RB) + bp[j]);
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < MB; ++i) acc[i][j] = M::mul(bf[j], af[i], acc[i][j]);
        }
    }
    const bool parts = a.items > a.tiles;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            grad_w_store<T>(a, split, parts, o0 + 16 * (wm * MB + i) + (lane & 15), c0 + 16 * (wn * NB + j) + 4 * (lane >> 4), acc[i][j]);
}

// dz of many rows: tiles of 256 rows of X by 128 of W, four wavefronts with 64 x 128 each, two workgroups on a compute unit.  The
// epilogue, 28 vector instructions for each number of a gated dz, takes as long as the multiplies; with two wavefronts of
// different workgroups on a SIMD the one's runs under the other's in part.  40,960 x 640 x 2 x 2,560, GELU: 363 us, 412 in a
// loop that heats the chip (without its epilogue 264 before the fragments were read ahead; the product's persistent kernel with
// this epilogue 401).  Stages of 64 bytes of a row, three LDS slots: a stage's loads have two stages to arrive.  Chunk c of
// row r lies at position c ^ r / 2 % 4.
template <bool GATED, int ACT>
__global__ __launch_bounds__(256, 2) void grad_dz_large_kernel(const ActGradArgs a)
{
    using T = __bf16;
    using M = Mul<T>;
    constexpr int BS = 16, MB = 4, NB = 8, BM = 256, BN = 128, RB = 64, G = 4, H = 2;  // load instructions of a wavefront
    constexpr int ABYTES = BM * RB, SLOT = (BM + BN) * RB, BO = GATED ? BN / 2 : BN;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ __attribute__((aligned(16))) float cols[BN];
    if ((int)blockIdx.x >= a.groups) return turn_tile<T, 256>(a.turn, (int)blockIdx.x - a.groups, smem);
    // workgroup -> tile: XCD x (= blockIdx % 8) owns a contiguous run of tiles, numbered in panels of a.panel column tiles
    const int tile = (int)(blockIdx.x % kXcds) * a.per_xcd + (int)(blockIdx.x / kXcds);
    if (tile >= a.tiles) return;  // whole workgroup: no barrier has been reached yet
    const int tiles_m = a.tiles / a.tiles_n, row = tile / a.panel, pn = row / tiles_m, mt = row - pn * tiles_m;
    const int64_t m0 = (int64_t)mt * BM;
    const int n0 = (pn * a.panel + tile - row * a.panel) * BO;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rowbytes = a.Cin * 2, stages = (rowbytes + RB - 1) / RB;
    const int lr = lane >> 2, lc = (lane & 3) ^ ((lr >> 1) & 3);
    const __amdgpu_buffer_rsrc_t xres = rows_from(a.X, m0, a.M, rowbytes);
    const __amdgpu_buffer_rsrc_t wres0 = rows_from(a.W[0], n0, a.Cout, rowbytes);
    const __amdgpu_buffer_rsrc_t wres1 = GATED ? rows_from(a.W[1], n0, a.Cout, rowbytes) : wres0;
    const uint32_t xoff = (uint32_t)((wv * (16 * G) + lr) * rowbytes + lc * 16);
    uint32_t woff[H];
#pragma unroll
    for (int l = 0; l < H; ++l) woff[l] = (uint32_t)((channel_of<BS, GATED>(wv * (16 * H) + 16 * l) + lr) * rowbytes + lc * 16);
    auto issue_stage = [&](int ks, int slot) __attribute__((always_inline)) {
        const bool live = ks * RB + lc * 16 < rowbytes;
        unsigned char *as = smem + slot * SLOT + wv * (G * 1024), *bs = smem + slot * SLOT + ABYTES + wv * (H * 1024);
#pragma unroll
        for (int l = 0; l < G; ++l)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xres, (__attribute__((address_space(3))) void *)(as + l * 1024), 16,
                                                     live ? xoff + (uint32_t)(16 * l * rowbytes + ks * RB) : kOob, 0, 0, 0);
#pragma unroll
        for (int l = 0; l < H; ++l) {
            const uint32_t off = live ? woff[l] + (uint32_t)(ks * RB) : kOob;
            if (GATED && l == 1)  // (blocks of 16 rows of the gate and of the value by turns)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(wres1, (__attribute__((address_space(3))) void *)(bs + l * 1024), 16,
                                                         (uint32_t)off, 0, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(wres0, (__attribute__((address_space(3))) void *)(bs + l * 1024), 16,
                                                         (uint32_t)off, 0, 0, 0);
        }
    };
    if (threadIdx.x < BN) {
        float b, s;
        column<BS, GATED, false>(a, n0, threadIdx.x, b, s);
        cols[threadIdx.x] = b;
    }
    issue_stage(0, 0);
    issue_stage(1, 1);  // (past the last stage: zeros)
    issue_stage(2, 2);
    const int l16 = lane & 15, at = l16 * RB + (((lane >> 4) ^ ((l16 >> 1) & 3)) * 16), aat = at + wv * (16 * MB * RB);
    typename M::Frag af[2][MB], bf[NB];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * (G + H)));  // stage 0 has landed
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    typename M::Acc acc[MB][NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const f32x4 first = *(const f32x4 *)(cols + BS * j + 4 * (lane >> 4));
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[i][j] = first;
    }
#pragma unroll
    for (int i = 0; i < MB; ++i) af[0][i] = *(const bf16x8 *)(smem + aat + i * (16 * RB));
#pragma unroll
    for (int j = 0; j < NB; ++j) bf[j] = *(const bf16x8 *)(smem + ABYTES + at + j * (16 * RB));
    int slot = 0;
    // stage ks, whose fragments are there; the next stage's are read as these are used up, into their places
    auto step = [&](int ks, auto turn) __attribute__((always_inline)) {
        constexpr int now = decltype(turn)::value;
        // this wavefront's loads of the next stage have landed (those of the one after may be on their way), and its reads of this
        // one, whose slot is filled again, are done; behind the barrier everybody's are
        asm volatile("" ::: "memory");
        if (ks + 2 < stages)
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(G + H));
        else
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (ks + 3 < stages) issue_stage(ks + 3, slot);
        slot = slot == 2 ? 0 : slot + 1;
        const unsigned char *next = smem + slot * SLOT;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
#pragma unroll
            for (int i = 0; i < MB; ++i) acc[i][j] = M::mul(bf[j], af[now][i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            bf[j] = *(const bf16x8 *)(next + ABYTES + at + j * (16 * RB));
            if (j < MB) af[1 - now][j] = *(const bf16x8 *)(next + aat + j * (16 * RB));
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int ks = 0;;) {
        step(ks, std::integral_constant<int, 0>{});
        if (++ks == stages) break;
        step(ks, std::integral_constant<int, 1>{});
        if (++ks == stages) break;
    }
    int le = lane;
    asm volatile("" : "+v"(le));  // (or the epilogue's addresses are kept alive through the main loop)
    GradIn<T, MB, NB, GATED> in;
    epilogue_grad_fetch(a, in, m0 + wv * (16 * MB), n0, le);
    // everybody is through with the ring: it becomes the staging area
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // (LDS operations only)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    epilogue_grad<T, MB, NB, GATED, T, ACT>(a, acc, in, m0 + wv * (16 * MB), n0, smem + wv * kGradBytes<T, NB, GATED>, le);
}
constexpr int kDzLargeLds = 3 * 384 * 64;

// Large ones: 256 x 256 tiles, eight wavefronts (two per SIMD) whose parts are 64 columns of dz by 128 of X.  Two LDS slots; the
// multiplies of a stage run in halves (columns of dz [0, 32), then [32, 64) of a part) over one set of fragments that is refilled in
// place, and LDS reads and the loads of the next stage but one sit between the matrix instructions by hand, as in the
// product's persistent kernel.  Where X has no more than 128 columns left, the four wavefronts of its other half, one
// of each SIMD, only load, and the tile takes little more than half the time.  No bank conflicts (counted).  5,120 x 640 over 40,960
// rows: 241 us, 1,117 TFLOP/s, 4 splits and 10 us to join them (tiles of 128 x 128 412 us).
__global__ __launch_bounds__(512, 2) void grad_w_large_kernel(const GradWArgs a)
{
    using T = __bf16;
    using M = Mul<T>;
    using K = Cols<T, 256>;
    constexpr int MB = 4, NB = 8, KS = K::KS, G = 4, NL = 2 * G;
    constexpr int ABYTES = 256 * kRow, SLOT = 2 * ABYTES;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    if ((int)blockIdx.x >= a.groups) return join_columns<512>(a.join, (int)blockIdx.x - a.groups, (float *)smem);
    // workgroup -> item: every XCD has a run of the items of whole tiles, and then one of the others
    const int xcd = (int)(blockIdx.x % kXcds), idx = (int)(blockIdx.x / kXcds), tiles_m = a.tiles / a.tiles_n;
    const int splits = a.items / a.tiles;
    int split, mt, nt;
    if (idx < a.whole_xcd) {
        const int item = xcd * a.whole_xcd + idx, per = tiles_m * a.whole;
        if (item >= per * splits) return;  // whole workgroup: no barrier has been reached yet
        split = item / per;
        mt = (item - split * per) / a.whole;
        nt = item - split * per - mt * a.whole;
    } else {
        const int item = xcd * a.rest_xcd + idx - a.whole_xcd;
        if (item >= tiles_m * splits) return;
        split = item / tiles_m;
        mt = item - split * tiles_m;
        nt = a.whole;
    }
    const int o0 = mt * 256, c0 = nt * 256;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv & 3, wn = wv >> 2;
    const bool busy = c0 + 128 * wn < a.Cin;
    const int zbytes = a.No * 2, xbytes = a.Cin * 2;
    uint32_t aoff[G], boff[G];
#pragma unroll
    for (int l = 0; l < G; ++l) {
        const int r = (wv * G + l) * K::RPI + lane / K::CPR, c = (lane % K::CPR) ^ K::swizzle(r);
        aoff[l] = o0 + c * K::PER < a.No ? (uint32_t)(r * zbytes + c * 16) : kOob;
        boff[l] = c0 + c * K::PER < a.Cin ? (uint32_t)(r * xbytes + c * 16) : kOob;
    }
    const int64_t first = (int64_t)split * a.stages * KS;
    const int stages = (int)min((int64_t)a.stages, (a.M - first + KS - 1) / KS);
    // ---- the load side, up to two stages ahead of the multiplies; past the last stage all lanes are out of range
    int ld = 0;
    __amdgpu_buffer_rsrc_t zres, xres;
    unsigned char *ld_to = smem;
    auto stage_setup = [&]() __attribute__((always_inline)) {
        const int64_t k = ld < stages ? first + (int64_t)ld * KS : a.M;
        zres = cols_from(a.dz, k, a.M, zbytes, o0 * 2);
        xres = cols_from(a.X, k, a.M, xbytes, c0 * 2);
        ld_to = smem + (ld & 1) * SLOT + wv * (G * 1024);
        ++ld;
    };
    auto issue_one = [&](int l) __attribute__((always_inline)) {
        if (l < G)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(zres, (__attribute__((address_space(3))) void *)(ld_to + l * 1024), 16,
                                                     (uint32_t)aoff[l], 0, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xres, (__attribute__((address_space(3))) void *)(ld_to + ABYTES + (l - G) * 1024), 16,
                                                     (uint32_t)boff[l - G], 0, 0, 0);
    };
    typename M::Acc acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = typename M::Acc{};
    // fragment i of a part is 32 i bytes from the first, exclusive-or'd: the swizzle is one of whole fragments
    const int ap = K::row(lane) * K::RB + K::place(lane, wm * MB), bp = ABYTES + K::row(lane) * K::RB + K::place(lane, wn * NB);
    constexpr int HB = MB / 2, NMH = HB * NB;
    typename M::Frag af[MB], bf[NB];
    constexpr int TAIL = NMH, kSpread = 5 * NMH / 2;
    auto read_a = [&](int slot, int kk, int i) __attribute__((always_inline)) {
        af[i] = K::read(smem + (((ap + slot) ^ (32 * i)) + kk * (KS / 2 * K::RB)));
    };
    auto read_b = [&](int slot, int kk, int j) __attribute__((always_inline)) {
        bf[j] = K::read(smem + (((bp + slot) ^ (32 * j)) + kk * (KS / 2 * K::RB)));
    };
    auto loads_at = [&](int g) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < NL; ++q)
            if ((q * kSpread) / NL == g) {
                issue_one(q);
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    auto half1 = [&](int slot, int kk, int g0) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < NMH; ++m) {
            loads_at(g0 + m);
#pragma unroll
            for (int r = 0; r < HB; ++r)
                if ((r * (NMH / 2)) / HB == m) {
                    read_a(slot, kk, HB + r);
                    __builtin_amdgcn_sched_barrier(0);
                }
            const int j = m / HB, i0 = m - j * HB, i = j & 1 ? HB - 1 - i0 : i0;
            acc[i][j] = M::mul(bf[j], af[i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto half2 = [&](int nslot, int nkk, int g0) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < NMH; ++m) {
            loads_at(g0 + m);
            const int j = m / HB, i0 = m - j * HB, i = j & 1 ? HB - 1 - i0 : i0;
            if (i0 == 0 && j > 0) {
                read_b(nslot, nkk, j - 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (i0 == HB - 1 && j < HB) {
                read_a(nslot, nkk, j);
                __builtin_amdgcn_sched_barrier(0);
            }
            acc[HB + i][j] = M::mul(bf[j], af[HB + i], acc[HB + i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        read_b(nslot, nkk, NB - 1);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto issue_tail = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < NL; ++q)
            if ((q * kSpread) / NL < TAIL) issue_one(q);
    };
    auto wait_all = [&]() __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    stage_setup();
#pragma unroll
    for (int l = 0; l < NL; ++l) issue_one(l);
    wait_all();
    stage_setup();
    issue_tail();
    if (busy) {
#pragma unroll
        for (int i = 0; i < HB; ++i) read_a(0, 0, i);
#pragma unroll
        for (int j = 0; j < NB; ++j) read_b(0, 0, j);
        for (int ks = 0; ks < stages; ++ks) {
            const int slot = (ks & 1) * SLOT, next = SLOT - slot;
            if (wv >= 4) __builtin_amdgcn_s_setprio(1);
            half1(slot, 0, TAIL);
            half2(slot, 1, TAIL + NMH);
            __builtin_amdgcn_s_setprio(0);
            stage_setup();
            half1(slot, 1, TAIL + 2 * NMH);
            // this wavefront's loads of the next stage have landed and its reads of this slot are done; behind the barrier
            // everybody's are
            wait_all();
            half2(next, 0, 0);
        }
    } else {
        for (int ks = 0; ks < stages; ++ks) {
#pragma unroll
            for (int q = 0; q < NL; ++q)
                if ((q * kSpread) / NL >= TAIL) issue_one(q);
            stage_setup();
            wait_all();
            issue_tail();
        }
    }
    __builtin_amdgcn_s_waitcnt(0);  // (nothing is on its way into LDS when the workgroup ends)
    if (!busy) return;
    const bool parts = splits > 1;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            grad_w_store<T>(a, split, parts, o0 + 16 * (wm * MB + i) + (lane & 15), c0 + 16 * (wn * NB + j) + 4 * (lane >> 4), acc[i][j]);
}
constexpr int kLargeLds = 2 * 512 * kRow;

// The splits' sums added up: G threads for four numbers, every G-th split each, these in their order (with many splits a thread
// would wait for one read after the other).
template <typename T, int G>
__global__ __launch_bounds__(256) void grad_w_join_kernel(const GradWArgs a)
{
    constexpr int Q = 256 / G;  // fours of a workgroup
    const int64_t n = (int64_t)a.No * a.Cin, i = ((int64_t)blockIdx.x * Q + (threadIdx.x % Q)) * 4;
    const int splits = a.items / a.tiles, g = threadIdx.x / Q;
    f32x4 v{};
    if (i < n)
#pragma unroll 4
        for (int s = g; s < splits; s += G) v += *(const f32x4 *)(a.partial + s * n + i);
    if constexpr (G > 1) {
        __shared__ f32x4 part[G][Q];
        part[g][threadIdx.x % Q] = v;
        __syncthreads();
        if (g) return;
#pragma unroll
        for (int q = 1; q < G; ++q) v += part[q][threadIdx.x];
    }
    if (i >= n) return;
    const int64_t half = (int64_t)a.Cout * a.Cin;
    T *to = (T *)(i < half ? a.dW[0] : a.dW[1]);
    if (!to) return;
    typedef T Quad __attribute__((ext_vector_type(4)));
    Quad q;
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = (T)v[e];
    *(Quad *)(to + (i < half ? i : i - half)) = q;
}

// dX of few rows: dX = sum dz_k W_k, 32 x 32 a workgroup, whose eight wavefronts share the contraction as in act_small_kernel
// (a wavefront takes every eighth stage through two LDS slots of its own).  W's rows are what is contracted over, and are
// read transposed; stages do not cross from one set to the other.  A long contraction for few tiles is split over workgroups.
// 160 x 1,280 x 1,280: 4.9 us, and 3.4 + 5.1 where a kernel of its own turns W first.
struct GradXArgs {
    const void *dz;  // [M][No]
    const void *W[2];
    void *dX;
    int64_t M;
    int32_t Cin, Cout, No, tiles_n;
    int32_t tiles_m, tiles, per_xcd;  // tiles_m: row tiles where tiles are numbered down the columns, or 0
    int32_t span;                     // stages of a split (blockIdx.y)
    float *partial;                   // [splits][M][Cin], or null: one split
};
template <typename T>
__global__ __launch_bounds__(512, 2) void grad_x_small_kernel(const GradXArgs a)
{
    using M = Mul<T>;
    using B = Cols<T, 32>;
    constexpr int NW = 8, SR = 36, SLOT = 64 * kRow, KS = B::KS;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    int mt, nt;
    if (!small_tile(a, mt, nt)) return;
    const int64_t m0 = (int64_t)mt * 32;
    const int n0 = nt * 32;
    const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int zbytes = a.No * B::ES, xbytes = a.Cin * B::ES, setbytes = a.Cout * B::ES;
    const __amdgpu_buffer_rsrc_t zres = rows_from(a.dz, m0, a.M, zbytes);
    unsigned char *mem = smem + wv * (2 * SLOT);
    const int lr = lane >> 3, lc = (lane & 7) ^ lr;
    const uint32_t zoff = (uint32_t)(lr * zbytes + lc * 16), next = (uint32_t)(8 * zbytes);
    uint32_t woff[4];
#pragma unroll
    for (int l = 0; l < 4; ++l) {
        const int r = l * B::RPI + lane / B::CPR, c = (lane % B::CPR) ^ B::swizzle(r);
        woff[l] = n0 + c * B::PER < a.Cin ? (uint32_t)(r * xbytes + c * 16) : kOob;
    }
    const int per = (a.Cout + KS - 1) / KS;  // stages of a set
    const int first = (int)blockIdx.y * a.span, stages = min(a.No / a.Cout * per, first + a.span);
    auto issue = [&](int ks, int slot) __attribute__((always_inline)) {
        const int set = ks >= per ? 1 : 0, k = ks - set * per;
        const bool live = k * kRow + lc * 16 < setbytes;
        const uint32_t o = zoff + (uint32_t)(set * setbytes + k * kRow);
        const __amdgpu_buffer_rsrc_t wres = cols_from(set ? a.W[1] : a.W[0], (int64_t)k * KS, a.Cout, xbytes, n0 * B::ES);
#pragma unroll
        for (int l = 0; l < 4; ++l) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(zres, (__attribute__((address_space(3))) void *)(mem + slot * SLOT + l * 1024), 16,
                                                     live ? o + l * next : kOob, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wres, (__attribute__((address_space(3))) void *)(mem + slot * SLOT + 4096 + l * 1024),
                                                     16, (uint32_t)woff[l], 0, 0, 0);
        }
    };
    f32x4 acc[2][2] = {};
    int koff[2], wp[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) koff[kk] = M::offset(lane, kk);
#pragma unroll
    for (int j = 0; j < 2; ++j) wp[j] = 4096 + B::row(lane) * B::RB + B::place(lane, j);
    if (first + wv < stages) issue(first + wv, 0);
    int slot = 0;
    for (int ks = first + wv; ks < stages; ks += NW) {
        const bool more = ks + NW < stages;
        if (more) issue(ks + NW, slot ^ 1);
        asm volatile("" ::: "memory");
        if (more)
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(8));  // all but the stage just asked for have landed
        else
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        const unsigned char *buf = mem + slot * SLOT;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            typename M::Frag x[2], w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[i] = M::read(buf + l16 * kRow + i * (16 * kRow), koff[kk]);
                w[i] = B::read(buf + kk * (KS / 2 * B::RB) + wp[i]);
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
    const int row = (int)threadIdx.x >> 4, c = 2 * ((int)threadIdx.x & 15);
    const int64_t m = m0 + row;
    if (m >= a.M || n0 + c >= a.Cin) return;
    typedef T Pair __attribute__((ext_vector_type(2)));  // (Cin is even)
    typedef float Floats __attribute__((ext_vector_type(2)));
    Floats z{};
#pragma unroll
    for (int v = 0; v < NW; ++v) z += *(const Floats *)&sums[v][row][c];
    if (a.partial) {
        *(Floats *)(a.partial + ((int64_t)blockIdx.y * a.M + m) * a.Cin + n0 + c) = z;
        return;
    }
    Pair y;
#pragma unroll
    for (int o = 0; o < 2; ++o) y[o] = (T)z[o];
    *(Pair *)((T *)a.dX + m * a.Cin + n0 + c) = y;
}

template <typename T>
__global__ __launch_bounds__(256) void grad_turn_kernel(const TurnArgs a)
{
    __shared__ __attribute__((aligned(16))) unsigned char smem[64 * (64 * sizeof(T) + 4)];
    turn_tile<T, 256>(a, (int)blockIdx.x, smem);
}

// Column sums of 256 rows of a matrix, 128 columns a workgroup: part blockIdx.x.
template <typename T>
__global__ __launch_bounds__(256) void grad_sums_kernel(const void *dz, int64_t M, int No, float *sums)
{
    constexpr int PER = 8, ES = (int)sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(16 / ES)));
    __shared__ float part[16][128 + 4];
    const int l = threadIdx.x & 15, w = threadIdx.x >> 4, c = (int)blockIdx.y * 128 + l * PER;
    const int64_t first = (int64_t)blockIdx.x * 256;
    float v[PER] = {};
    if (c < No)
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
            const int64_t m = first + w + 16 * i;
            if (m >= M) break;
#pragma unroll
            for (int h = 0; h < PER * ES / 16; ++h) {
                const int at = h * (16 / ES);
                if (c + at >= No) break;
                const Piece x = *(const Piece *)((const T *)dz + m * No + c + at);
#pragma unroll
                for (int e = 0; e < 16 / ES; ++e) v[at + e] += (float)x[e];
            }
        }
#pragma unroll
    for (int e = 0; e < PER; ++e) part[w][l * PER + e] = v[e];
    __syncthreads();
    const int cc = (int)blockIdx.y * 128 + (int)threadIdx.x;
    if (threadIdx.x >= 128 || cc >= No) return;
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 16; ++q) t += part[q][threadIdx.x];
    sums[(int64_t)blockIdx.x * No + cc] = t;
}

}  // namespace
}  // namespace dsattn
