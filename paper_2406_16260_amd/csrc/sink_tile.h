// dsattn_sink_forward on the matrix cores: more than a few queries of one head of K and V.
//
// The rows of a unit (a position and a head of K and V) are its queries, frame by frame and within a frame the query
// heads that share the head: row r is new frame r / g, query head r % g of the group.  A wavefront owns 16 RB rows and
// walks the frames that they see between them in tiles of KT with a running maximum:
//   S^T = K Q^T   keys on M, queries on N, both operands 16-byte pieces of rows: lane l has piece l / 16 of row l % 16
//   O^T = V^T P^T a lane's weights are the operand as they stand (any order of the keys contracts the same); bf16: V^T by
//                 transposing LDS reads, weights rounded to bf16, and divided by the sum of the rounded ones: an error of 2^-8 each
//                 at most, which their weighted mean makes smaller than the output's own; fp32: 16x16x4 on both
// K and V pass through LDS.  Two ways to share them:
//   SHARED   the wavefronts of a workgroup have neighbouring rows of one unit and one tile of 64 or 32 frames, which is
//            double-buffered: long windows, bound by the matrix cores and the exponentials
//   else     a wavefront has LDS of its own, and a unit or a part of its frames (`splits`) of its own: short windows,
//            bound by memory, and few rows over a long window
#pragma once

namespace dsattn {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void wave_lds_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// maximum (NaN where one is: fmaxf() takes an instruction more for each of its operands, to drop it) / sum over the lanes
// l, l ^ 16, l ^ 32, l ^ 48
template <bool MAX>
__device__ __forceinline__ float over_quarters(float x)
{
    unsigned a = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const unsigned r0 = r[0], r1 = r[1];
    const float y0 = __builtin_bit_cast(float, r0), y1 = __builtin_bit_cast(float, r1);
    x = MAX ? __builtin_elementwise_maximum(y0, y1) : y0 + y1;
    a = __builtin_bit_cast(unsigned, x);
    const auto s = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const unsigned s0 = s[0], s1 = s[1];
    const float z0 = __builtin_bit_cast(float, s0), z1 = __builtin_bit_cast(float, s1);
    return MAX ? __builtin_elementwise_maximum(z0, z1) : z0 + z1;
}

// LDS rows of NB 64-byte blocks.  K is read by 16-byte pieces: the 16 lanes that are served together are on rows 0 - 3 and
// 12 - 15 of one piece and 4 - 11 of the next, which are in different banks where a row is 2 pieces more than a multiple
// of four.  V by 8 bytes of four rows of a group of 16 lanes (bf16): a row is an odd number of blocks; or by 4 bytes of
// rows four apart (fp32): one piece more than whole blocks.  (Both one piece more than whole blocks: 61 % of the LDS's
// busy cycles were conflicts, and it was busy 90 % of the time.)
constexpr int k_row_bytes(int NB) { return 64 * NB + 32; }
constexpr int v_row_bytes(bool F32, int NB) { return F32 ? 64 * NB + 16 : NB % 2 ? 64 * NB : 64 * NB + 64; }
constexpr int tile_bytes(bool F32, int NB, int KT) { return KT * (k_row_bytes(NB) + v_row_bytes(F32, NB)); }
constexpr int tile_lds_bytes(bool F32, int NB, int KT, bool SHARED) { return (SHARED ? 2 : 4) * tile_bytes(F32, NB, KT); }

// Blocks of 16 rows of a wavefront, frames of a tile and wavefronts of a workgroup, as many as leave a wavefront its registers
// (bf16, head_dim 160: 40 registers of sums a block of rows, 20 of queries, and what is on its way of the next tile).
constexpr int tile_blocks(bool F32, int NB, bool SHARED, bool many) { return F32 || (!SHARED && !many) || NB > 4 ? 1 : 2; }
constexpr int tile_frames(bool F32, bool SHARED, bool many) { return SHARED ? (F32 || !many ? 32 : 64) : F32 ? 16 : 32; }
// (many: of rows, more than 16; shared: of frames, a window of 128 or more)
constexpr int tile_group(bool F32, int NB, bool SHARED) { return SHARED && !F32 && NB > 4 ? 8 : 4; }
// Numbers of blocks that kernels are compiled for, and how many of them every head that a kernel takes fills.
constexpr int round_blocks(int NB) { return NB <= 6 ? NB : NB <= 8 ? 8 : NB <= 10 ? 10 : NB <= 12 ? 12 : 16; }
constexpr int full_blocks(int NB) { return NB <= 6 ? NB - 1 : NB == 8 ? 6 : NB == 10 ? 8 : NB == 12 ? 10 : 12; }
// Wavefronts per SIMD that the registers have to leave room for.
constexpr int tile_waves(int NB, int RB, bool SHARED, int WV)
{
    if (SHARED && WV == 8) return 2;
    return NB > 8 || (NB > 6 && !SHARED) ? 1 : SHARED || NB >= 4 || NB * RB > 4 ? 2 : 3;
}

// NB = 64-byte blocks of a head's row, rounded up.
template <typename T, int NB, int RB, int KT, bool SHARED, int WV>
__global__ __launch_bounds__(64 * WV, tile_waves(NB, RB, SHARED, WV)) void sink_tile_kernel(const SinkArgs a)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int V = 16 / (int)sizeof(T), DB = 4 * V;  // numbers of a piece, of a block
    constexpr int RK = k_row_bytes(NB), RV = v_row_bytes(F32, NB), TILE = tile_bytes(F32, NB, KT);  // K, behind it V
    constexpr int KB = KT / 16;                           // blocks of 16 keys
    // threads that fetch a tile, LPR neighbouring lanes a row (64 bytes at least), in PASSES of RP rows, NP pieces a lane and row
    constexpr int THREADS = SHARED ? 64 * WV : 64, LPR = THREADS / KT > 4 ? THREADS / KT : 4;
    constexpr int RP = THREADS / LPR, PASSES = KT / RP, NP = (4 * NB + LPR - 1) / LPR;
    static_assert(PASSES * RP == KT, "whole passes");
    constexpr int ROWS = 16 * RB * (SHARED ? WV : 1);     // rows of a task
    typedef T Piece __attribute__((ext_vector_type(V)));
    using Frag = std::conditional_t<F32, f32x4, bf16x8>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

    const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = a.h / a.hk, D = a.D;
    // workgroup -> tasks: XCD x (= blockIdx % 8) takes a contiguous run of them
    // (32-bit divisions: a 64-bit one is some hundred scalar instructions)
    const uint32_t wg = (blockIdx.x % 8u) * (uint32_t)a.per_xcd + blockIdx.x / 8u;
    uint32_t id = SHARED ? wg : wg * 4u + (uint32_t)wv;
    if (id >= (uint32_t)a.tasks) return;  // shared: the whole workgroup; else nobody waits for anybody
    // Shared: the row tiles of a unit are neighbours, the longest first.  (A unit's K and V stay in one XCD's L2, and the short
    // ones at a stream's start are spread over the XCDs.)  Else the heads are (they share memory pages and lines), then the
    // row tiles of a unit (they share frames).
    const uint32_t parts = (uint32_t)a.splits, inner = (uint32_t)(SHARED ? a.row_tiles : a.hk);
    const uint32_t outer = (uint32_t)(SHARED ? a.hk : a.row_tiles);
    uint32_t rest = parts > 1 ? id / parts : id;
    const int split = parts > 1 ? (int)(id - rest * parts) : 0;
    id = rest;
    rest = id / inner;
    const int in = (int)(id - rest * inner);
    id = rest;
    rest = id / outer;
    const int out = (int)(id - rest * outer);
    const int kvh = SHARED ? out : in, rt = SHARED ? a.row_tiles - 1 - in : out;
    const int b = (int)(rest / (uint32_t)a.P), p = (int)(rest - (uint32_t)b * a.P);
    const Stream st = stream_of(a, b);
    const int rows = st.count * g, first = rt * ROWS;
    if (first >= rows) return;  // (the same for all wavefronts of a task)
    const int last = min(first + ROWS, rows) - 1;
    const Frames fr = frames_of(a, st, first / g, last / g);

    // this lane's rows of each block: what the mask needs, in the numbering of fr
    const int r0 = first + (SHARED ? wv * 16 * RB : 0);
    const int shift = fr.lo - fr.ns, always = max(fr.ns, a.sinks - shift);
    int hi[RB], lw[RB];
    int64_t qrow[RB];  // element offset of the row in Q and O
    Frag q[RB][NB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const int r = r0 + 16 * i + l16, t = min(r, rows - 1) / g, gi = min(r, rows - 1) - t * g;
        const int frame = st.start + t;
        hi[i] = r < rows ? frame - shift : -1;
        lw[i] = frame - a.window - shift;
        qrow[i] = (((int64_t)b * a.T + t) * a.P + p) * a.h * D + (kvh * g + gi) * D;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            q[i][kb] = Frag{};
            if (DB * kb + V * lg < D) q[i][kb] = *(const Frag *)((const T *)a.Q + qrow[i] + DB * kb + V * lg);
        }
    }
    // the wavefront's: keys that all of its rows see, that any may see (rows ascend by frame)
    const int ra = min(r0, rows - 1) / g, rz = min(r0 + 16 * RB, rows) - 1;
    const int hi_all = r0 + 16 * RB <= rows ? st.start + ra - shift : -1;
    const int lw_all = st.start + max(rz, 0) / g - a.window - shift, lw_any = st.start + ra - a.window - shift;
    const int hi_any = r0 < rows ? st.start + max(rz, 0) / g - shift : -1;

    // ---- K and V into LDS: LPR neighbouring lanes a row, every LPR-th piece each
    const int tid = SHARED ? (int)threadIdx.x : lane;
    const int lrow = tid / LPR, lc = tid % LPR;
    unsigned char *mem = smem + (SHARED ? 0 : wv * TILE);
    const int64_t frow = (int64_t)a.P * a.hk * D, at = ((int64_t)p * a.hk + kvh) * D;
    // (kept in registers: a choice between arguments is otherwise a load by every lane, which the loop then waits for)
    typedef const __attribute__((address_space(1))) T *Rows;
    Rows kf = (Rows)a.K + (int64_t)b * a.T * frow + at, vf = (Rows)a.V + (int64_t)b * a.T * frow + at;
    typedef __attribute__((address_space(1))) T *Cache;
    Cache kc = (Cache)a.Kc + (int64_t)b * (a.sinks + a.ring) * frow + at, vc = (Cache)a.Vc + (int64_t)b * (a.sinks + a.ring) * frow + at;
    asm volatile("" : "+s"(kf), "+s"(vf), "+s"(kc), "+s"(vc));
    // (unconditional loads: behind a branch each would be waited for at its end; past the head the row's first piece)
    auto in_row = [&](int i) __attribute__((always_inline)) { return LPR * i + LPR <= 4 * NB || LPR * i + lc < 4 * NB; };
    auto within = [&](int i) __attribute__((always_inline)) {
        return LPR * i + LPR <= 4 * full_blocks(NB) || (LPR * i + lc) * V < D;
    };
    Piece kr[PASSES][NP], vr[PASSES][NP];
    auto fetch = [&](int tile) __attribute__((always_inline)) {
        typedef const __attribute__((address_space(1))) Piece *Pieces;
#pragma unroll
        for (int n = 0; n < PASSES; ++n) {
            const int j = min(tile * KT + n * RP + lrow, fr.n - 1), f = fr.frame(j);
            const bool fresh = f >= st.start;
            const int64_t off = (fresh ? f - st.start : fr.slot(a, f)) * frow;
            const Rows kp = (fresh ? kf : (Rows)kc) + off, vp = (fresh ? vf : (Rows)vc) + off;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = within(i) ? (LPR * i + lc) * V : 0;
                kr[n][i] = *(Pieces)(kp + c);
                vr[n][i] = *(Pieces)(vp + c);
            }
        }
    };
    // (K's pieces past the head are zeros, as Q's are; V's are never stored)
    // The task's own new frames go into the cache on the way (each is fetched by one part of the task's frames).
    const int own_first = st.start + first / g, own_last = st.start + last / g;
    const bool puts = puts_frames(a, st);
    auto put = [&](int tile, int buf) __attribute__((always_inline)) {
        if (puts && tile * KT + KT - 1 >= own_first - shift) {  // (a frame's number past the last one's may not fit)
            typedef __attribute__((address_space(1))) Piece *Slots;
#pragma unroll
            for (int n = 0; n < PASSES; ++n) {
                const int j = tile * KT + n * RP + lrow, f = fr.frame(j);
                if (j >= fr.n || f < own_first || f > own_last || !stays(a, st, f)) continue;
                const int64_t off = slot_of(a, f) * frow;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    if (!in_row(i) || !within(i)) continue;
                    *(Slots)(kc + off + (LPR * i + lc) * V) = kr[n][i];
                    *(Slots)(vc + off + (LPR * i + lc) * V) = vr[n][i];
                }
            }
        }
#pragma unroll
        for (int n = 0; n < PASSES; ++n) {
            unsigned char *tok = mem + (SHARED ? buf * TILE : 0) + (n * RP + lrow) * RK + 16 * lc;
            unsigned char *tov = mem + (SHARED ? buf * TILE : 0) + KT * RK + (n * RP + lrow) * RV + 16 * lc;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                if (!in_row(i)) continue;
                *(Piece *)(tok + 16 * LPR * i) = within(i) ? kr[n][i] : Piece{};
                *(Piece *)(tov + 16 * LPR * i) = vr[n][i];
            }
        }
    };

    constexpr int OB = F32 ? NB : 2 * NB;  // blocks of 16 channels
    f32x4 o[RB][OB] = {};
    float m[RB], l[RB];  // the row's maximum; fp32: this lane's part of the sum
    f32x4 ls[RB] = {};   // bf16: the sum, of the rounded weights, in every element: a row of ones times P^T
    bf16x8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.f;
#pragma unroll
    for (int i = 0; i < RB; ++i) m[i] = -INFINITY, l[i] = 0.f;

    auto multiply = [&](int tile, const unsigned char *ks) __attribute__((always_inline)) {
        const int j0 = tile * KT;
        // no row of this wavefront sees a frame of the tile
        if (j0 > hi_any || (j0 + KT - 1 <= lw_any && j0 >= always)) return;
        const unsigned char *vs = ks + KT * RK;
        f32x4 s[RB][KB];
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int i = 0; i < RB; ++i) s[i][k] = f32x4{};
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                const Frag kf = *(const Frag *)(ks + (16 * k + l16) * RK + 64 * kb + 16 * lg);
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    if constexpr (F32) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], q[i][kb][e], s[i][k], 0, 0, 0);
                    } else {
                        s[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[i][kb], s[i][k], 0, 0, 0);
                    }
                }
            }
        // Eight pieces of K on their way ahead of the multiplies, all the time (by itself the compiler reads two and waits for them:
        // 287 -> 277 us on one card, 295 -> 287 on another, 2 prompts of 8,192, 16 heads on 4 x 128, window 2,048).
        if constexpr (!F32 && SHARED && KB == 4 && RB == 2) {
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 1);
#pragma unroll
            for (int x = 0; x < 4 * NB - 8; x += 2) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2 * RB, 1);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 8 * RB, 1);
        }
        // hidden keys: key 16 k + 4 lg + e of the tile
        if (j0 + KT - 1 > hi_all || (j0 <= lw_all && j0 + KT - 1 >= always)) {
            if (j0 >= always) {  // behind the sinks a row sees the keys from lw + 1 to hi
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    const uint32_t span = (uint32_t)max(hi[i] - lw[i], 0);
                    const int from = j0 + 4 * lg - lw[i] - 1;
#pragma unroll
                    for (int k = 0; k < KB; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i][k][e] = (uint32_t)(from + 16 * k + e) < span ? s[i][k][e] : -INFINITY;
                }
            } else {
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int k = 0; k < KB; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int j = j0 + 16 * k + 4 * lg + e;
                            const bool sees = j <= hi[i] && (j > lw[i] || j < always);
                            s[i][k][e] = sees ? s[i][k][e] : -INFINITY;
                        }
            }
        }
        float shiftv[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            float top = s[i][0][0];
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = __builtin_elementwise_maximum(top, s[i][k][e]);
            top = __builtin_elementwise_maximum(m[i], over_quarters<true>(top) * a.sc);
            shiftv[i] = top == -INFINITY ? 0.f : top;
            if (__any(top > m[i])) {
                const float old = __builtin_amdgcn_exp2f(m[i] - shiftv[i]);
                l[i] *= old;
                ls[i] *= old;
#pragma unroll
                for (int c = 0; c < OB; ++c) o[i][c] *= old;
            }
            m[i] = top;
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[i][k][e] = __builtin_amdgcn_exp2f(fmaf(s[i][k][e], a.sc, -shiftv[i]));
                    if constexpr (F32) l[i] += s[i][k][e];
                }
        }
        // (while the other wavefront of the SIMD is elsewhere: 330 -> 315 us, 2 prompts of 8,192, 16 heads on 4 x 128, window 2,048)
        if constexpr (SHARED) __builtin_amdgcn_s_setprio(1);
        if constexpr (F32) {
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < OB; ++c) {
                        const float vf = *(const float *)(vs + (16 * k + 4 * lg + e) * RV + 64 * c + 4 * l16);
#pragma unroll
                        for (int i = 0; i < RB; ++i) o[i][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf, s[i][k][e], o[i][c], 0, 0, 0);
                    }
        } else {
#pragma unroll
            for (int k = 0; k < KB; k += 2) {
                bf16x8 w[RB];
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[i][e] = (__bf16)s[i][k][e];
                        w[i][4 + e] = (__bf16)s[i][k + 1][e];
                    }
#pragma unroll
                for (int i = 0; i < RB; ++i) ls[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, w[i], ls[i], 0, 0, 0);
                // V^T: within a group of 16 lanes the transposing read hands lane i element i % 4 of the 8 bytes
                // that lanes i / 4, 4 + i / 4, 8 + i / 4 and 12 + i / 4 point at.  Lane i points at key 4 lg + i / 4,
                // channels 8 (i % 4) + 4 x .. of the block, and so gets keys 4 lg .. 4 lg + 3 of channel
                // 8 (i / 4) + 4 x + i % 4: a lane ends up with eight neighbouring channels of its query.
#pragma unroll
                for (int c = 0; c < OB; ++c) {
                    s16x4 r[2];
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        r[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (__attribute__((address_space(3))) s16x4 *)(vs + (16 * (k + t) + 4 * lg + (l16 >> 2)) * RV +
                                                                        64 * (c / 2) + 16 * (l16 & 3) + 8 * (c & 1)));
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int i = 0; i < RB; ++i) o[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, w[i], o[i][c], 0, 0, 0);
                }
            }
        }
    };

    // this task's tiles: all, or a part of them
    const int tiles = (fr.n + KT - 1) / KT, per = (tiles + a.splits - 1) / a.splits;
    const int t0 = split * per, t1 = min(tiles, t0 + per);
    if constexpr (SHARED) {
        if (t0 < t1) fetch(t0);
        for (int t = t0; t < t1; ++t) {
            put(t, t & 1);
            if (t + 1 < t1) fetch(t + 1);
            __builtin_amdgcn_s_setprio(0);
            __syncthreads();  // everybody's part of tile t is there, and tile t - 1, whose buffer is next, is done with
            multiply(t, mem + (t & 1) * TILE);
        }
    } else {
        if (t0 < t1) fetch(t0);
        for (int t = t0; t < t1; ++t) {
            wave_lds_sync();
            put(t, 0);
            wave_lds_sync();
            if (t + 1 < t1) fetch(t + 1);
            multiply(t, mem);
        }
    }

#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const float sum = F32 ? over_quarters<false>(l[i]) : ls[i][0];
        const int r = r0 + 16 * i + l16;
        if (a.splits > 1) {
            if (r >= rows) continue;
            float *to = part_of(a, b, (int64_t)p * a.hk + kvh, r, a.T * g, split);
            if (lg == 0) {
                to[0] = m[i];
                to[1] = sum;
            }
#pragma unroll
            for (int c = 0; c < OB; ++c) {
                const int ch = F32 ? 16 * c + 4 * lg : 32 * (c / 2) + 8 * lg + 4 * (c & 1);
                if (ch < D) *(f32x4 *)(to + kPartHead + ch) = o[i][c];
            }
            continue;
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        bool nan = false;
#pragma unroll
        for (int c = 0; c < OB; ++c) {
            o[i][c] *= inv;
            nan = nan || __builtin_isunordered(o[i][c][0], o[i][c][1]) || __builtin_isunordered(o[i][c][2], o[i][c][3]);
        }
        // (a hidden frame's infinity times its weight of zero)
        const uint64_t again = __ballot(nan && r < rows), quarters = 0x0001000100010001ull;
        if (r < rows && !(again >> l16 & quarters)) {
            if constexpr (F32) {
#pragma unroll
                for (int c = 0; c < OB; ++c)
                    if (16 * c + 4 * lg < D) *(f32x4 *)((float *)a.O + qrow[i] + 16 * c + 4 * lg) = o[i][c];
            } else {
#pragma unroll
                for (int c = 0; c < OB; c += 2) {
                    bf16x8 y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[e] = (__bf16)o[i][c][e];
                        y[4 + e] = (__bf16)o[i][c + 1][e];
                    }
                    if (16 * c + 8 * lg < D) *(bf16x8 *)((__bf16 *)a.O + qrow[i] + 16 * c + 8 * lg) = y;
                }
            }
        }
        if (again) {
            for (int u = 0; u < 16; ++u) {
                if (!(again >> u & quarters)) continue;
                const int ru = r0 + 16 * i + u, t = ru / g;
                vector_row<T>(a, b, st, t, p, kvh * g + ru - t * g, lane);
            }
        }
    }
}

template <typename T, bool SHARED, bool MANY>
const void *tile_kernel_of(int NB)
{
    constexpr bool F32 = sizeof(T) == 4;
#define DSATTN_TILE(nb) \
    if (NB == nb) return (const void *)&sink_tile_kernel<T, nb, tile_blocks(F32, nb, SHARED, MANY), tile_frames(F32, SHARED, MANY), SHARED, \
                                                    tile_group(F32, nb, SHARED)>
    DSATTN_TILE(1);
    DSATTN_TILE(2);
    DSATTN_TILE(3);
    DSATTN_TILE(4);
    DSATTN_TILE(5);
    DSATTN_TILE(6);
    DSATTN_TILE(8);
    if constexpr (F32) {
        DSATTN_TILE(10);
        DSATTN_TILE(12);
        DSATTN_TILE(16);
    }
#undef DSATTN_TILE
    return nullptr;
}

// The launch on the matrix cores; fn null: none.
struct TileLaunch {
    const void *fn;
    int row_tiles, splits, lds, waves;
    int rows, frames;  // of a task, of a tile
    bool shared;
    int64_t tasks, workgroups;
};
TileLaunch tile_launch(const dsattn_sink_desc &d)
{
    TileLaunch k{};
    const bool f32 = d.io_dtype == DSATTN_F32;
    const int V = f32 ? 4 : 8;
    if (d.head_dim % V != 0 || d.head_dim > 256) return k;
    const int NB = round_blocks((d.head_dim + 4 * V - 1) / (4 * V));
    const int64_t rows = (int64_t)d.frames * (d.heads / d.kv_heads), units = (int64_t)d.streams * d.spatial * d.kv_heads;
    // Row tiles that share their frames, us apart (32 rows a wavefront) and shared, in tiles of 32 and of 64 frames:
    //   128 frames x 640 positions, 8 x 80, 4 sinks, window 32      126.5  108.7  115.4
    //   256 frames x 160 positions, 8 x 128, 4 sinks, window 64      87.0   85.0   88.5
    //   256 frames x 160 positions, 8 x 128, 4 sinks, window 130            89.6   86.4
    //   64 frames x 2,560 positions, 8 x 40, 4 sinks, window 16     132.1  149.2  168.0
    const int64_t sees = (int64_t)d.sinks + d.window;
    const bool shared = rows >= 64 && sees >= 32;
    const bool many = shared ? sees >= 128 : rows > 16;
    const int RB = tile_blocks(f32, NB, shared, many), KT = tile_frames(f32, shared, many);
    k.waves = tile_group(f32, NB, shared);
    k.shared = shared;
    k.frames = KT;
    const int per = 16 * RB * (shared ? k.waves : 1);
    if (rows > 0x7fffff00) return k;  // (numbered with 32 bits)
    k.rows = per;
    k.row_tiles = (int)((rows + per - 1) / per);
    k.tasks = units * k.row_tiles;
    // Few tasks (for a card's 256 compute units: the workspace has to follow from the shape alone): parts of the frames each, of
    // four tiles at least, up to 1,024 wavefronts apart (16 streams of 4 tokens, 32 heads on 8 x 128, over 8,192: 129 us up to
    // 2,048, 122 up to 1,024; 4 streams of 8 tokens over 4,096: 26.5 and 26.6) or 512 workgroups shared.
    const int64_t n = std::min<int64_t>((int64_t)d.sinks + d.window + (shared ? per / (d.heads / d.kv_heads) : d.frames), 1 << 24);
    const int64_t tiles = (n + KT - 1) / KT;
    k.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(shared ? 512 : 1024) / k.tasks, tiles / 4, kMaxSplits}));
    // What the join costs, 5 us and 1.5 ns a row, against what the parts save, 1.6 us a shared tile (fp32 2.5).  Measured us, whole
    // and in parts: 384 tokens, 8 heads on 2 x 32, window 3,372, 53.9 and 21.3; 512, 16 on 4 x 128, 4,096, 109 and 53; 1,035,
    // 20 on 5 x 40, 911, 24.1 and 54.9; 2,048, 16 on 4 x 128, 4,096, 57.6 and 96.3.
    const double tile_us = f32 ? 2.5 : 1.6, join_us = 5.0 + 1.5e-3 * (double)d.streams * d.frames * d.spatial * d.heads;
    if (shared && (double)(tiles - (tiles + k.splits - 1) / k.splits) * tile_us < join_us) k.splits = 1;
    k.tasks *= k.splits;
    k.workgroups = shared ? k.tasks : (k.tasks + 3) / 4;
    if (k.workgroups > 0xffffff - 8) return TileLaunch{};
    k.lds = tile_lds_bytes(f32, NB, KT, shared);
    k.fn = f32 ? (shared ? tile_kernel_of<float, true, true>(NB) : tile_kernel_of<float, false, true>(NB))
           : shared ? (many ? tile_kernel_of<__bf16, true, true>(NB) : tile_kernel_of<__bf16, true, false>(NB))
                    : (many ? tile_kernel_of<__bf16, false, true>(NB) : tile_kernel_of<__bf16, false, false>(NB));
    return k;
}

}  // namespace
}  // namespace dsattn
