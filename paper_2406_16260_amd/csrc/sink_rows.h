// dsattn_sink_forward for few rows: up to four queries of one head of K and V (a frame of one to four query heads
// on it, or a few frames), which is a stream of the cache through the vector ALUs.
//
// A unit is a position and a head of K and V; the units of a frame are neighbours in memory.  LG lanes have a unit's
// head_dim in PV 16-byte pieces each (interleaved, so that the lanes of a piece read neighbouring bytes); a wavefront has U units and
// 64 / (LG U) groups of lanes, which take frames in turn, as do the four wavefronts of a workgroup and `splits`
// workgroups.  Each group runs its own softmax (running maximum, sum, weighted sum); they are joined through lane
// exchanges, LDS, and, between workgroups, the caller's workspace and a kernel of its own.
//
// Bound by memory: K and V of the visible frames once, 2 + 2 bytes per channel and frame against about 12 vector
// instructions a lane, piece and query.
#pragma once

namespace dsattn {
namespace {

// frames of a step: their rows are in flight together, and one maximum serves them
constexpr int step_frames(int PV) { return PV == 1 ? 4 : 2; }

// sum over a group of LG neighbouring lanes, in all of them
template <int LG>
__device__ __forceinline__ float group_sum(float x)
{
    auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if constexpr (LG >= 2) x += dpp(x, std::integral_constant<int, 0xb1>{});   // quad_perm 1 0 3 2
    if constexpr (LG >= 4) x += dpp(x, std::integral_constant<int, 0x4e>{});   // quad_perm 2 3 0 1
    if constexpr (LG >= 8) x += dpp(x, std::integral_constant<int, 0x141>{});  // mirror of half a row of 16
    if constexpr (LG >= 16) x += dpp(x, std::integral_constant<int, 0x140>{}); // mirror of the row
    if constexpr (LG >= 32) {
        const unsigned b = __builtin_bit_cast(unsigned, x);
        const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        const unsigned r0 = r[0], r1 = r[1];
        x = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
    }
    if constexpr (LG >= 64) {
        const unsigned b = __builtin_bit_cast(unsigned, x);
        const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        const unsigned r0 = r[0], r1 = r[1];
        x = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
    }
    return x;
}

// A softmax's running maximum (in powers of two), sum, and weighted sum of N numbers.
template <int N>
struct Running {
    float m = -INFINITY, l = 0.f, o[N] = {};

    // takes another one's in
    __device__ __forceinline__ void join(float m2, float l2, const float *o2)
    {
        const float top = fmaxf(m, m2), shift = top == -INFINITY ? 0.f : top;
        const float f = __builtin_amdgcn_exp2f(m - shift), f2 = __builtin_amdgcn_exp2f(m2 - shift);
        m = top;
        l = l * f + l2 * f2;
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = o[e] * f + o2[e] * f2;
    }
};

template <typename T, int LG, int PV, int R>
__global__ __launch_bounds__(256) void sink_rows_kernel(const SinkArgs a)
{
    constexpr int V = 16 / (int)sizeof(T), N = V * PV, kFrames = step_frames(PV);
    typedef T Piece __attribute__((ext_vector_type(V)));
    extern __shared__ float lds[];  // [3 wavefronts][R][N + 2][lanes]
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int units = a.P * a.hk, blocks = (units + a.U - 1) / a.U;
    int id = (int)blockIdx.x;
    const int split = id % a.splits;
    id /= a.splits;
    const int ub = id % blocks, b = id / blocks;
    const Stream st = stream_of(a, b);
    if (st.count == 0) return;
    const int li = lane % LG, u = lane / LG % a.U, fg = lane / (LG * a.U), groups = 64 / (LG * a.U);
    const bool mine = ub * a.U + u < units;
    const int unit = min(ub * a.U + u, units - 1);
    const int p = unit / a.hk, kvh = unit - p * a.hk, g = a.h / a.hk;
    const int D = a.D, rows = a.T * g;

    float q[R][N];
    int fa[R];  // the row's frame, -1 for none
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int t = r / g;
        fa[r] = r < rows && t < st.count ? st.start + t : -1;
        const T *from = (const T *)a.Q + (((int64_t)b * a.T + t) * a.P + p) * a.h * D + (kvh * g + r - t * g) * D;
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            const int c = (i * LG + li) * V;
            Piece x{};
            if (fa[r] >= 0 && c < D) x = *(const Piece *)(from + c);
#pragma unroll
            for (int e = 0; e < V; ++e) q[r][i * V + e] = (float)x[e] * a.sc;
        }
    }

    // the frames that any of the rows sees: [0, ns) and from lo on
    const Frames fr = frames_of(a, st, 0, st.count - 1);
    const int64_t row = (int64_t)a.P * a.hk * D, at = (int64_t)unit * D + li * V;
    const T *Kf = (const T *)a.K + (int64_t)b * a.T * row + at, *Vf = (const T *)a.V + (int64_t)b * a.T * row + at;
    T *Kc = (T *)a.Kc + (int64_t)b * (a.sinks + a.ring) * row + at, *Vc = (T *)a.Vc + (int64_t)b * (a.sinks + a.ring) * row + at;
    const int all = groups * 4 * a.splits, me = (split * 4 + wv) * groups + fg;
    const int steps = (fr.n + all * kFrames - 1) / (all * kFrames);
    const bool masked = a.T > 1, fuse = puts_frames(a, st);
    Running<N> run[R];
    for (int step = 0; step < steps; ++step) {
        const int j0 = (step * all + me) * kFrames;
        Piece k[kFrames][PV], v[kFrames][PV];
        int f[kFrames];
#pragma unroll
        for (int i = 0; i < kFrames; ++i) {
            const int j = min(j0 + i, fr.n - 1);
            f[i] = fr.frame(j);
            const bool fresh = f[i] >= st.start;
            const int64_t off = (fresh ? f[i] - st.start : fr.slot(a, f[i])) * row;
            const T *kp = (fresh ? Kf : Kc) + off, *vp = (fresh ? Vf : Vc) + off;
#pragma unroll
            for (int c = 0; c < PV; ++c) {
                k[i][c] = v[i][c] = Piece{};
                if (PV > 1 || (c * LG + li) * V < D) {
                    k[i][c] = *(const Piece *)(kp + c * (LG * V));
                    v[i][c] = *(const Piece *)(vp + c * (LG * V));
                }
            }
            // a new frame goes into the cache from here: one group has it
            if (fuse && fresh && j0 + i < fr.n && mine && stays(a, st, f[i])) {
                const int64_t to = slot_of(a, f[i]) * row;
#pragma unroll
                for (int c = 0; c < PV; ++c)
                    if (PV > 1 || (c * LG + li) * V < D) {
                        *(Piece *)(Kc + to + c * (LG * V)) = k[i][c];
                        *(Piece *)(Vc + to + c * (LG * V)) = v[i][c];
                    }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s[kFrames];
            bool sees[kFrames];
#pragma unroll
            for (int i = 0; i < kFrames; ++i) {
                float x = 0.f;
#pragma unroll
                for (int c = 0; c < PV; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) x = fmaf(q[r][c * V + e], (float)k[i][c][e], x);
                sees[i] = j0 + i < fr.n;
                if (masked) sees[i] = sees[i] && f[i] <= fa[r] && (f[i] < a.sinks || fa[r] - f[i] < a.window);
                s[i] = group_sum<LG>(x);
                s[i] = sees[i] ? s[i] : -INFINITY;
            }
            Running<N> &w = run[r];
            float top = w.m;
#pragma unroll
            for (int i = 0; i < kFrames; ++i) top = fmaxf(top, s[i]);
            const float shift = top == -INFINITY ? 0.f : top;
            const float old = __builtin_amdgcn_exp2f(w.m - shift);
            w.m = top;
            w.l *= old;
#pragma unroll
            for (int e = 0; e < N; ++e) w.o[e] *= old;
#pragma unroll
            for (int i = 0; i < kFrames; ++i) {
                if (!sees[i]) continue;  // (not zero times what may be no number)
                const float x = __builtin_amdgcn_exp2f(s[i] - shift);
                w.l += x;
#pragma unroll
                for (int c = 0; c < PV; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) w.o[c * V + e] = fmaf(x, (float)v[i][c][e], w.o[c * V + e]);
            }
        }
    }

    // the groups of a wavefront
    for (int w = LG * a.U; w < 64; w *= 2)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float o2[N];
            const float m2 = __shfl_xor(run[r].m, w), l2 = __shfl_xor(run[r].l, w);
#pragma unroll
            for (int e = 0; e < N; ++e) o2[e] = __shfl_xor(run[r].o[e], w);
            run[r].join(m2, l2, o2);
        }
    // the wavefronts
    const int lanes = LG * a.U;
    if (wv > 0 && lane < lanes)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float *to = lds + ((wv - 1) * R + r) * (N + 2) * lanes + lane;
            to[0] = run[r].m;
            to[lanes] = run[r].l;
#pragma unroll
            for (int e = 0; e < N; ++e) to[(e + 2) * lanes] = run[r].o[e];
        }
    __syncthreads();
    if (wv > 0 || lane >= lanes || !mine) return;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (fa[r] < 0) continue;
        for (int w = 0; w < 3; ++w) {
            const float *from = lds + (w * R + r) * (N + 2) * lanes + lane;
            float o2[N];
#pragma unroll
            for (int e = 0; e < N; ++e) o2[e] = from[(e + 2) * lanes];
            run[r].join(from[0], from[lanes], o2);
        }
        const int t = r / g, head = kvh * g + r - t * g;
        if (a.splits > 1) {
            float *to = part_of(a, b, unit, r, rows, split);
            if (li == 0) {
                to[0] = run[r].m;
                to[1] = run[r].l;
            }
#pragma unroll
            for (int i = 0; i < PV; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if ((i * LG + li) * V < D) to[kPartHead + (i * LG + li) * V + e] = run[r].o[i * V + e];
            continue;
        }
        const float inv = run[r].l == 0.f ? 0.f : 1.f / run[r].l;
        T *to = (T *)a.O + (((int64_t)b * a.T + t) * a.P + p) * a.h * D + head * D;
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            const int c = (i * LG + li) * V;
            Piece x;
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = (T)(run[r].o[i * V + e] * inv);
            if (c < D) *(Piece *)(to + c) = x;
        }
    }
}

template <typename T, int R>
const void *rows_kernel_of(int LG, int PV)
{
#define DSATTN_ROWS(lg, pv) \
    if (LG == lg && PV == pv) return (const void *)&sink_rows_kernel<T, lg, pv, R>
    DSATTN_ROWS(1, 1);
    DSATTN_ROWS(2, 1);
    DSATTN_ROWS(4, 1);
    DSATTN_ROWS(8, 1);
    DSATTN_ROWS(16, 1);
    DSATTN_ROWS(32, 1);
    DSATTN_ROWS(64, 1);
    if constexpr (R == 1) {
        DSATTN_ROWS(1, 3);
        DSATTN_ROWS(2, 3);
        DSATTN_ROWS(1, 5);
        DSATTN_ROWS(2, 5);
    }
#undef DSATTN_ROWS
    return nullptr;
}

// The launch for few rows; fn null: none.
struct RowsLaunch {
    const void *fn;
    int LG, PV, R, U, splits;
    int64_t blocks;
    int lds;
};
RowsLaunch rows_launch(const dsattn_sink_desc &d)
{
    RowsLaunch k{};
    const bool f32 = d.io_dtype == DSATTN_F32;
    const int V = f32 ? 4 : 8;
    if (d.frames > 4 || d.heads / d.kv_heads > 4 / d.frames || d.head_dim % V != 0) return k;
    const int rows = d.frames * (d.heads / d.kv_heads);
    const int pieces = d.head_dim / V;
    if (pieces > 64) return k;
    k.R = rows > 2 ? 4 : rows;
    // Lanes of a unit: as many as there are pieces, up to a power of two; or three or five pieces a lane where one or two
    // lanes then hold a unit and one row's sums leave the registers for it.  One frame over 4 first and some last ones, us in
    // a captured graph, pieces a lane and idle lanes: 640 positions, 8 x 80, 32 frames 15.3 and 17.5; 2,560 positions, 8 x 40,
    // 16 frames 18.0 and 19.9; but four lanes: 160 positions, 8 x 160, 60 frames 14.7 and 13.6, 300 positions, 8 x 96, 150
    // frames 33.1 and 30.7.
    const int two = pieces & -pieces, odd = pieces / two;
    k.PV = 1;
    for (k.LG = 1; k.LG < pieces;) k.LG *= 2;
    if (k.R == 1 && (odd == 3 || odd == 5) && two <= 2) {
        k.LG = two;
        k.PV = odd;
    }
    // Units of a wavefront: as many as leave about 512 wavefronts (2,048: 640 positions, 8 x 80, 21.1 us instead of 15.3), of a
    // step's frames a group of lanes at least.  Then workgroups for one unit's frames, up to 2,048 wavefronts, of eight
    // frames a group at least, or of 64 where there are 512 wavefronts already: a kernel joins them (16 streams over 16,384
    // frames, 32 heads on 8 x 128: 688 us by one, 228 by four; one token of 32 heads on 8 x 128 over 4,096: 39 us by 8 workgroups a unit,
    // 20 by 32; 160 positions, 8 x 128, over 64: 11.2 us by one, 15.8 by two).
    const int64_t units = (int64_t)d.spatial * d.kv_heads, n = (int64_t)d.sinks + d.window + d.frames;
    auto waves = [&](int U) { return d.streams * ((units + U - 1) / U) * 4; };
    for (k.U = 64 / k.LG; k.U > 1 && (waves(k.U) < 512 || k.U / 2 >= units) && n / (4 * 64 / (k.LG * k.U)) > step_frames(k.PV);) k.U /= 2;
    const int64_t groups = 4 * 64 / (k.LG * k.U);
    k.splits = (int)std::max<int64_t>(1, std::min<int64_t>({2048 / waves(k.U), n / (groups * (waves(k.U) < 512 ? 8 : 64)), kMaxSplits}));
    k.blocks = waves(k.U) / 4 * k.splits;
    if (k.blocks > 0xffffff) return RowsLaunch{};
    k.lds = 3 * k.R * (V * k.PV + 2) * k.LG * k.U * 4;
    k.fn = f32 ? (k.R == 1 ? rows_kernel_of<float, 1>(k.LG, k.PV) : k.R == 2 ? rows_kernel_of<float, 2>(k.LG, k.PV)
                                                                                : rows_kernel_of<float, 4>(k.LG, k.PV))
               : (k.R == 1 ? rows_kernel_of<__bf16, 1>(k.LG, k.PV) : k.R == 2 ? rows_kernel_of<__bf16, 2>(k.LG, k.PV)
                                                                                 : rows_kernel_of<__bf16, 4>(k.LG, k.PV));
    return k;
}

}  // namespace
}  // namespace dsattn
