// e4m3 codes (gfx950 device code of the 8-bit cache).
#pragma once
#include "ragc_internal.h"

namespace ragc {
namespace {

constexpr uint32_t kCodeNan = 0x7f;

// Four numbers to the nearest codes, ties to even; at most 448 in magnitude, or not finite, which gives NaN.
__device__ __forceinline__ uint32_t encode4(const float* x) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], v, true);
    uint32_t u = (uint32_t)v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(__builtin_fabsf(x[i]) <= 448.f)) u = (u & ~(0xffu << 8 * i)) | kCodeNan << 8 * i;
    return u;
}

}  // namespace
}  // namespace ragc
