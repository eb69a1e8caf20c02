// Device helpers of the attention kernels over the 8-bit cache (gfx950 only): e4m3 numbers with a power-of-two scale per
// block, plane and kv head, in the layout of kv8_append.hip.
#pragma once
#include "attn_bf16_common.h"
#include "attn_work.h"
#include "kv8_codes.h"

namespace ragc {
namespace {

// Four codes times 2^(s-127), `scale` = that number: exact in bf16 (four bits of mantissa) down to its smallest number, 2^-133.
__device__ __forceinline__ bf16x4 widen4(uint32_t codes, float scale) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
}
__device__ __forceinline__ bf16x8 join(bf16x4 lo, bf16x4 hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// What bf16 does not hold of a block with scale byte s, as `to_top` of nan_bytes: NaN, and numbers of 2^128 or more, which are the codes
// from exponent 262 - s on (there are none up to s = 246).
__device__ __forceinline__ uint32_t not_finite_from(int s) { return (uint32_t)(0x80 - min(0x7f, (262 - s) * 8)) * 0x01010101u; }
// the codes with those made 0, but for the bytes of `except`
__device__ __forceinline__ uint32_t without_nan(uint32_t codes, uint32_t to_top, uint32_t except = 0) {
    return codes & (except | ~((nan_bytes(codes, to_top) >> 7) * 0xffu));
}
// 1.0 (0x38) where there is one and 0 elsewhere
__device__ __forceinline__ uint32_t where_nan(uint32_t codes, uint32_t to_top) { return (nan_bytes(codes, to_top) >> 7) * 0x38u; }
// bytes of the four keys from `key` on that lie below `limit`
__device__ __forceinline__ uint32_t below(int key, int limit) {
    const int n = limit - key;
    return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << 8 * n) - 1;
}

// The copies of one request's row tiles along its keys: as many as it takes for `chunk` blocks each (0: one copy).
__device__ __host__ __forceinline__ int copies_of(int keys, int chunk) {
    return chunk == 0 ? 1 : ((keys + kBlock - 1) / kBlock + chunk - 1) / chunk;
}

}  // namespace
}  // namespace ragc
