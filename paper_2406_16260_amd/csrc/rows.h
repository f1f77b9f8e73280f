// What the kernels that normalise rows share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dsattn {
namespace {

// y in 8 bits, to nearest, ties to even
__device__ __forceinline__ uint8_t to_e4m3(float y)
{
    return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 255);
}

// The maximum of two numbers, NaN if one is: what fmaxf() would drop.
__device__ __forceinline__ float max_or_nan(float a, float b) { return a > b || a != a ? a : b; }

bool overlap(const void *a, int64_t an, const void *b, int64_t bn)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + (uintptr_t)bn && y < x + (uintptr_t)an;
}

}  // namespace
}  // namespace dsattn
