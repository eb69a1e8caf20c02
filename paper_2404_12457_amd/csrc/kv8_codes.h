// e4m3 codes (gfx950 device code of the 8-bit cache).
#pragma once
#include "ragc_internal.h"

namespace ragc {
namespace {

constexpr uint32_t kNoNan = 0x7f7f7f7fu;

// 0x80 in every byte that is a NaN code, or with another `to_top` (0x80 less the smallest code, in every byte) a code of at least so much
__device__ __forceinline__ uint32_t nan_bytes(uint32_t codes, uint32_t to_top = 0x01010101u) { return ((codes & kNoNan) + to_top) & 0x80808080u; }

// Four numbers to the nearest codes, ties to even; at most 448 in magnitude, or not finite, which gives NaN (0x7f).
__device__ __forceinline__ uint32_t encode4(const float* x) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], v, true);
    return (uint32_t)v & ~nan_bytes((uint32_t)v);
}

}  // namespace
}  // namespace ragc
