// Estimates that choose between the kernels of a product (host only).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

namespace dsattn {
namespace {

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
// `more`: us that the tiles cost besides; `deep`: with two stages ahead.
bool small_is_faster(int32_t type, int64_t small_tiles, int64_t stages, double more = 0.0, bool deep = false)
{
    static const double small_stage[] = {0.17, 0.07, 0.1}, tile_stage[] = {0.6, 0.27, 0.35};  // by dsattn_dtype
    const double rounds = (double)((small_tiles + 255) / 256);
    return 1.5 + rounds * (1.2 + small_stage[type] * (double)stages) < 2.0 + (deep ? 0.24 : tile_stage[type]) * (double)stages + more;
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
// `deep`: with two stages ahead.
double tile_estimate(int size, int64_t tiles, int64_t stages, bool deep = false)
{
    const double st = (double)stages, n = (double)tiles;
    const int64_t full = tiles / 512, rest = tiles - 512 * full, rounds = (tiles + 255) / 256;
    if (size == 256) return 3.0 + (double)rounds * (1.22 * st + 5.0);
    if (size == 128)
        return 3.0 + (double)full * (0.95 * st + 2.0) + (rest > 256 ? 0.82 * st + 2.6 : rest > 0 ? (deep ? 0.54 : 0.61) * st + 2.9 : 0.0);
    static const double stage[] = {0.25, 0.3, 0.41, 0.61};
    return 4.0 + 1.3e-3 * n + st * (rounds > 4 ? std::max(1.0, 8.2e-4 * n) : stage[rounds - 1]);
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

// Whether an XCD's run of tiles, one after the other on its L2, reads less if it goes down the columns: counted in tiles' rows of
// the two operands.  (Few rows of X and a large W, across and down: 400 x 4,096 x 4,096 and its gradients 109 and 95 us,
// 600 x 2,560 x 2 x 2,560 105 and 97.)
bool down_reads_less(int64_t tiles_m, int64_t tiles_n)
{
    const int64_t run = (tiles_m * tiles_n + 7) / 8;
    auto reads = [&](int64_t along, int64_t across) { return std::min(run, along) + std::min((run + along - 1) / along, across); };
    return reads(tiles_m, tiles_n) < reads(tiles_n, tiles_m);
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

// The default cap on dynamic LDS is 64 KB; it is raised once for a kernel and device, not at every call.
hipError_t allow_lds(const void *fn, int lds)
{
    if (lds <= 64 << 10) return hipSuccess;
    struct Slot {
        std::atomic<const void *> fn;
        std::atomic<uint64_t> devices;
    };
    static Slot slots[64];  // (a kernel that finds no place is asked for each time)
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    Slot *mine = nullptr;
    const size_t at = ((uintptr_t)fn >> 3) * 0x9e3779b97f4a7c15ull >> 58;
    for (size_t i = 0; dev < 64 && i < 64 && !mine; ++i) {
        Slot &s = slots[(at + i) % 64];
        const void *there = s.fn.load(std::memory_order_acquire);
        if (!there && s.fn.compare_exchange_strong(there, fn, std::memory_order_acq_rel)) there = fn;
        if (there == fn) mine = &s;
    }
    const uint64_t bit = (uint64_t)1 << (dev & 63);
    if (mine && (mine->devices.load(std::memory_order_acquire) & bit)) return hipSuccess;
    e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e == hipSuccess && mine) mine->devices.fetch_or(bit, std::memory_order_acq_rel);
    return e;
}

}  // namespace
}  // namespace dsattn
