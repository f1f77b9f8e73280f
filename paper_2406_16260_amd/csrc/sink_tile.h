// dsattn_sink_forward on the matrix cores: more than a few queries of one head of K and V.
//
// The rows of a unit (a position and a head of K and V) are its queries, frame by frame and within a frame the query
// heads that share the head: row r is new frame r / g, query head r % g of the group.  A wavefront owns 16 RB rows and
// walks the frames that they see between them in tiles of KT with a running maximum:
//   S^T = K Q^T   keys on M, queries on N, both operands 16-byte pieces of rows: lane l has piece l / 16 of row l % 16
//   O^T = V^T P^T a lane's weights are the operand as they stand (any order of the keys contracts the same); bf16: V^T by
//                 transposing LDS reads, weights rounded to bf16 (2^-9 each, as far from the output's own rounding as
//                 their mean; the sum that they are divided by is of the unrounded ones); fp32: 16x16x4 on both
// K and V pass through LDS in rows padded by 16 bytes.  Two ways to share them:
//   SHARED   the four wavefronts of a workgroup have neighbouring rows of one unit and one tile of 64 or 32 frames, which is
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

// maximum / sum over the lanes l, l ^ 16, l ^ 32, l ^ 48
template <bool MAX>
__device__ __forceinline__ float over_quarters(float x)
{
    unsigned a = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const unsigned r0 = r[0], r1 = r[1];
    const float y0 = __builtin_bit_cast(float, r0), y1 = __builtin_bit_cast(float, r1);
    x = MAX ? fmaxf(y0, y1) : y0 + y1;
    a = __builtin_bit_cast(unsigned, x);
    const auto s = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const unsigned s0 = s[0], s1 = s[1];
    const float z0 = __builtin_bit_cast(float, s0), z1 = __builtin_bit_cast(float, s1);
    return MAX ? fmaxf(z0, z1) : z0 + z1;
}

// LDS row of NB 64-byte blocks, padded so that the rows spread over the banks
constexpr int tile_row_bytes(int NB) { return 64 * NB + 16; }
constexpr int tile_lds_bytes(int NB, int KT, bool SHARED) { return (SHARED ? 2 : 4) * 2 * KT * tile_row_bytes(NB); }

// Blocks of 16 rows of a wavefront and frames of a tile, as many as leave a wavefront its registers (bf16, head_dim 160:
// 40 registers of sums a block of rows, 20 of queries, and 40 of rows on their way for every 16 or 64 frames).
constexpr int tile_blocks(bool F32, int NB, bool SHARED, bool many) { return F32 || NB > 5 || (!SHARED && (!many || NB > 4)) ? 1 : 2; }
constexpr int tile_frames(bool F32, int NB, bool SHARED) { return SHARED ? (F32 || NB == 5 ? 32 : 64) : F32 ? 16 : 32; }
// Wavefronts per SIMD that the registers have to leave room for.
constexpr int tile_waves(int NB, int RB, bool SHARED) { return NB > 8 || (NB > 6 && !SHARED) ? 1 : SHARED || NB * RB > 4 ? 2 : 3; }

// NB = 64-byte blocks of a head's row, rounded up.
template <typename T, int NB, int RB, int KT, bool SHARED>
__global__ __launch_bounds__(256, tile_waves(NB, RB, SHARED)) void sink_tile_kernel(const SinkArgs a)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int V = 16 / (int)sizeof(T), DB = 4 * V;  // numbers of a piece, of a block
    constexpr int RS = tile_row_bytes(NB), TILE = KT * RS;
    constexpr int KB = KT / 16;                           // blocks of 16 keys
    constexpr int PASS = SHARED ? 64 : 16;                // rows that the threads fetch at a time, four lanes a row
    constexpr int NP = (KT + PASS - 1) / PASS;
    constexpr int ROWS = 16 * RB * (SHARED ? 4 : 1);      // rows of a task
    typedef T Piece __attribute__((ext_vector_type(V)));
    using Frag = std::conditional_t<F32, f32x4, bf16x8>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

    const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = a.h / a.hk, D = a.D;
    // workgroup -> tasks: XCD x (= blockIdx % 8) takes a contiguous run of them
    const int64_t wg = (int64_t)(blockIdx.x % 8u) * a.per_xcd + blockIdx.x / 8u;
    int64_t id = SHARED ? wg : wg * 4 + wv;
    if (id >= a.tasks) return;  // shared: the whole workgroup; else nobody waits for anybody
    // heads are neighbours (they share memory pages and lines), then the row tiles of a unit (they share frames)
    const int split = (int)(id % a.splits);
    id /= a.splits;
    const int kvh = (int)(id % a.hk);
    id /= a.hk;
    const int rt = (int)(id % a.row_tiles);
    id /= a.row_tiles;
    const int p = (int)(id % a.P), b = (int)(id / a.P);
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

    // ---- K and V into LDS: four lanes a row, each a piece of every block
    const int tid = SHARED ? (int)threadIdx.x : lane;
    const int lrow = tid >> 2, lc = tid & 3;
    unsigned char *mem = smem + (SHARED ? 0 : wv * 2 * TILE);
    const int64_t frow = (int64_t)a.P * a.hk * D, at = ((int64_t)p * a.hk + kvh) * D + V * lc;
    const int64_t fresh0 = (int64_t)b * a.T * frow + at, cache0 = (int64_t)b * (a.sinks + a.ring) * frow + at;
    Piece kr[NP][NB], vr[NP][NB];
    auto fetch = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int j = min(tile * KT + n * PASS + lrow, fr.n - 1), f = fr.frame(j);
            const bool fresh = f >= st.start;
            const int64_t off = fresh ? fresh0 + (f - st.start) * frow : cache0 + fr.slot(a, f) * frow;
            const T *kp = (const T *)(fresh ? a.K : a.Kc) + off, *vp = (const T *)(fresh ? a.V : a.Vc) + off;
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                kr[n][kb] = vr[n][kb] = Piece{};
                if ((KT % PASS == 0 || n * PASS + lrow < KT) && DB * kb + V * lc < D) {
                    kr[n][kb] = *(const Piece *)(kp + DB * kb);
                    vr[n][kb] = *(const Piece *)(vp + DB * kb);
                }
            }
        }
    };
    // (pieces past the head are zeros: what K has there is multiplied with Q's zeros)
    auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            if (KT % PASS != 0 && n * PASS + lrow >= KT) continue;
            unsigned char *to = mem + (SHARED ? buf * 2 * TILE : 0) + (n * PASS + lrow) * RS + 16 * lc;
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                *(Piece *)(to + 64 * kb) = kr[n][kb];
                *(Piece *)(to + TILE + 64 * kb) = vr[n][kb];
            }
        }
    };

    constexpr int OB = F32 ? NB : 2 * NB;  // blocks of 16 channels
    f32x4 o[RB][OB] = {};
    float m[RB], l[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) m[i] = -INFINITY, l[i] = 0.f;

    auto multiply = [&](int tile, const unsigned char *ks) __attribute__((always_inline)) {
        const int j0 = tile * KT;
        // no row of this wavefront sees a frame of the tile
        if (j0 > hi_any || (j0 + KT - 1 <= lw_any && j0 >= always)) return;
        const unsigned char *vs = ks + TILE;
        f32x4 s[RB][KB];
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int i = 0; i < RB; ++i) s[i][k] = f32x4{};
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                const Frag kf = *(const Frag *)(ks + (16 * k + l16) * RS + 64 * kb + 16 * lg);
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
        // hidden keys: key 16 k + 4 lg + e of the tile
        if (j0 + KT - 1 > hi_all || (j0 <= lw_all && j0 + KT - 1 >= always)) {
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
        float shiftv[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            float top = s[i][0][0];
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, s[i][k][e]);
            top = fmaxf(m[i], over_quarters<true>(top) * a.sc);
            shiftv[i] = top == -INFINITY ? 0.f : top;
            if (__any(top > m[i])) {
                const float old = __builtin_amdgcn_exp2f(m[i] - shiftv[i]);
                l[i] *= old;
#pragma unroll
                for (int c = 0; c < OB; ++c) o[i][c] *= old;
            }
            m[i] = top;
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[i][k][e] = __builtin_amdgcn_exp2f(fmaf(s[i][k][e], a.sc, -shiftv[i]));
                    l[i] += s[i][k][e];
                }
        }
        if constexpr (F32) {
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < OB; ++c) {
                        const float vf = *(const float *)(vs + (16 * k + 4 * lg + e) * RS + 64 * c + 4 * l16);
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
                            (__attribute__((address_space(3))) s16x4 *)(vs + (16 * (k + t) + 4 * lg + (l16 >> 2)) * RS +
                                                                        64 * (c / 2) + 16 * (l16 & 3) + 8 * (c & 1)));
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int i = 0; i < RB; ++i) o[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, w[i], o[i][c], 0, 0, 0);
                }
            }
        }
    };

    const int tiles = (fr.n + KT - 1) / KT;
    if constexpr (SHARED) {
        // tiles that no row of the workgroup sees: between the sinks in their window and the next row's window there
        // are none (frames_of() leaves them out)
        if (tiles > 0) fetch(0);
        for (int t = 0; t < tiles; ++t) {
            put(t & 1);
            if (t + 1 < tiles) fetch(t + 1);
            __syncthreads();  // everybody's part of tile t is there, and tile t - 1, whose buffer is next, is done with
            multiply(t, mem + (t & 1) * 2 * TILE);
        }
    } else {
        const int per = (tiles + a.splits - 1) / a.splits, t0 = split * per, t1 = min(tiles, t0 + per);
        if (t0 < t1) fetch(t0);
        for (int t = t0; t < t1; ++t) {
            wave_lds_sync();
            put(0);
            wave_lds_sync();
            if (t + 1 < t1) fetch(t + 1);
            multiply(t, mem);
        }
    }

#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const float sum = over_quarters<false>(l[i]);
        const int r = r0 + 16 * i + l16;
        if (!SHARED && a.splits > 1) {
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
    if (NB == nb) return (const void *)&sink_tile_kernel<T, nb, tile_blocks(F32, nb, SHARED, MANY), tile_frames(F32, nb, SHARED), SHARED>
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
    int row_tiles, splits, lds;
    int64_t tasks, workgroups;
};
TileLaunch tile_launch(const dsattn_sink_desc &d)
{
    TileLaunch k{};
    const bool f32 = d.io_dtype == DSATTN_F32;
    const int V = f32 ? 4 : 8;
    if (d.head_dim % V != 0 || d.head_dim > 256) return k;
    int NB = (d.head_dim + 4 * V - 1) / (4 * V);
    NB = NB <= 6 ? NB : NB <= 8 ? 8 : NB <= 10 ? 10 : NB <= 12 ? 12 : 16;
    const int64_t rows = (int64_t)d.frames * (d.heads / d.kv_heads), units = (int64_t)d.streams * d.spatial * d.kv_heads;
    const bool shared = rows >= 64 && (int64_t)d.sinks + d.window >= 128;
    const bool many = rows > 16;
    const int RB = tile_blocks(f32, NB, shared, many), KT = tile_frames(f32, NB, shared);
    const int per = 16 * RB * (shared ? 4 : 1);
    if ((rows + per - 1) / per > 0x7fffffff) return k;
    k.row_tiles = (int)((rows + per - 1) / per);
    k.tasks = units * k.row_tiles;
    k.splits = 1;
    if (!shared) {
        // few wavefronts: up to 2,048 with parts of the frames each, of four tiles at least
        const int64_t n = std::min<int64_t>((int64_t)d.sinks + d.window + d.frames, 1 << 24), tiles = (n + KT - 1) / KT;
        k.splits = (int)std::max<int64_t>(1, std::min<int64_t>({2048 / std::max<int64_t>(k.tasks, 1), tiles / 4, 64}));
        k.tasks *= k.splits;
    }
    k.workgroups = shared ? k.tasks : (k.tasks + 3) / 4;
    if (k.workgroups > 0xffffff - 8) return TileLaunch{};
    k.lds = tile_lds_bytes(NB, KT, shared);
    k.fn = f32 ? (shared ? tile_kernel_of<float, true, true>(NB) : tile_kernel_of<float, false, true>(NB))
               : (shared ? tile_kernel_of<__bf16, true, true>(NB)
                  : many ? tile_kernel_of<__bf16, false, true>(NB)
                         : tile_kernel_of<__bf16, false, false>(NB));
    return k;
}

}  // namespace
}  // namespace dsattn
