// Append to the 8-bit cache: e4m3 numbers with one power-of-two scale per block of 16 tokens, plane and kv head.
//
// Mathematics.  With amax the largest finite |x| of the tokens that join a block and e the smallest integer with amax <= 448 2^e
// (448 is the largest e4m3 number), a number is stored as the e4m3 number nearest to x 2^-e, ties to even, and 2^e as the byte
// e + 127 (at least 1).  A power of two costs nothing in relative precision, takes part in the attention's conversions
// without a multiply, and lets a block be raised from e to a larger e' without a second rounding of any number that stays
// normal: tokens that join a partly filled block take max(e_old, e_new), and only where that is above e_old are the stored ones
// rounded anew.  Numbers that are not finite become NaN (0x7f; the type has no infinity) and leave the scale alone.
//
// K may be turned by its position first (kv_rope.h has the pairs).  That is done in fp64, where both products of a bf16 and
// an fp32 number are exact, and comes down to fp32 with the last bit set where anything was lost (round to odd), so that the one
// rounding that counts, to three bits of mantissa, is the correct one: the bytes are those of the definition.
//
// Layout, in the order in which the matrix cores take their operands: a K tile is [D/16][token][16], a V tile
// [D/64][token/4][16][4][token%4] with element 64 i0 + 16 i3 + i2.
//
// Mapping.  A wave owns one (block, kv head), K and V: lane i has token i % 16 and the elements 16 c .. 16 c + 15 of every
// fourth chunk c from i / 16 on.  V codes turn around in LDS.  Which block: item j of the launch belongs to the largest request
// r with (new_start[r] - new_start[0] + 30 r) / 16 <= j, which leaves every request room for as many blocks as n tokens can touch
// from any offset, (n + 30) / 16, so no list has to be made on the host and a captured launch follows the device arrays.
// Workgroups behind the last item of the blocks turn Q (kv_rope.h).
//
// What bounds it: HBM on large calls, the chain of memory trips, of rotations and of the fetching of instructions on small ones: a lane turns,
// rounds and converts 32 numbers one after the other, for one token too, whose row all sixteen lanes of a group repeat.  16 requests
// of 7.6k tokens in all, 32/8 heads of 128: 38 us (4.6 TB/s), of these 22 for Q, 4 for the fp64 rotation of K; angles are fetched in fours and both
// ends of a pair stay in one lane (62 us with an exchange between lanes).  Pairs of neighbours 44 us, head_dim 64 25, K as it is and no Q 12
// (3.9 TB/s).  64 tokens of 64 requests 7.1 us (neighbours 7.4, K as it is 5.7), one token 7.6 (12 with one kernel for every kind of rotation).
#include <type_traits>

#include "kv8_codes.h"
#include "kv_rope.h"

namespace ragc {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// What is done to K before it is rounded: nothing, every pair of a head of 128 by halves (the usual case: a lane has both ends of
// its pairs), or any other rotation.  A kernel each: one call's latency is the fetching of its instructions as much as anything.
enum Turn { kAsItIs, kWholeHalves, kAnyPairs };

// |x| of a finite number as a whole number that keeps its order and whether it lies above a border of 20 bits; 0 for others
__device__ __forceinline__ uint32_t size_key(double x) {
    const uint64_t b = __double_as_longlong(x);
    const uint32_t hi = (uint32_t)(b >> 32) & 0x7fffffffu;
    return hi >= 0x7ff00000u ? 0u : hi << 1 | ((uint32_t)b != 0);
}
// e + 127 for the largest key: 448 = 1.75 * 2^8
__device__ __forceinline__ int scale_byte(uint32_t key) {
    const int e = (int)(key >> 21) - 1023 - 8 + ((key & 0x1fffff) > 0x180000u);
    return key == 0 ? 1 : max(1, min(254, e + 127));
}
// the same for the largest |x| in bf16, as its bits
__device__ __forceinline__ int scale_byte_bf16(uint32_t top) { return max(1, (int)(top >> 7) - 8 + ((top & 0x7f) > 0x60)); }

// fp64 to fp32 towards zero, with the last bit set where something was lost
__device__ __forceinline__ float round_to_odd(double x) {
    const float f = (float)x;
    const double back = (double)f;
    uint32_t u = __float_as_uint(f);
    if (back != x) u = (__builtin_fabs(back) > __builtin_fabs(x) ? u - 1 : u) | 1;
    return __uint_as_float(u);
}
// codes of a scale 2^by times the new one, rounded to that
__device__ __forceinline__ uint32_t raise4(uint32_t codes, int by) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    const float x[4] = {__builtin_ldexpf(a[0], by), __builtin_ldexpf(a[1], by), __builtin_ldexpf(b[0], by), __builtin_ldexpf(b[1], by)};
    return encode4(x);
}
// the bytes of `held` in N dwords at `at` rounded to a scale 2^-by times theirs; not unrolled: it happens once in a block's life or twice
__device__ __forceinline__ void raise_held(uint32_t* at, int n, uint32_t held, int by) {
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        const uint32_t was = at[i];
        at[i] = (raise4(was, by) & held) | (was & ~held);
    }
}

// Rows in bf16 that are rounded as they are: a lane's part of a tile, [chunk][half of it].
template <int NC>
struct Plain {
    bf16x8 x[NC][2];
    __device__ __forceinline__ void load(const __bf16* src, int cq) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) x[c][h] = *reinterpret_cast<const bf16x8*>(src + (cq + 4 * c) * 16 + h * 8);
    }
    // bits of the largest finite |x|, two numbers of 16 bits at a time
    __device__ __forceinline__ uint32_t top() const {
        typedef __attribute__((ext_vector_type(8))) unsigned short u16x8;
        u16x8 m = u16x8(0);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u16x8 a = __builtin_bit_cast(u16x8, x[c][h]) & (unsigned short)0x7fff;
                const u16x8 fine = __builtin_bit_cast(u16x8, a < (unsigned short)0x7f80);  // all bits where it is
                m = __builtin_elementwise_max(m, a & fine);
            }
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, (uint32_t)m[i]);
        return t;
    }
    __device__ __forceinline__ uint32_t codes(int c, int w, int s) const {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __builtin_ldexpf((float)x[c][w >> 1][(w & 1) * 4 + i], 127 - s);
        return encode4(y);
    }
};

// K turned in fp64, which is exact but for the last of 53 bits.
template <int D, int TURN>
struct Turned {
    static constexpr int NC = D / 64;
    double k[NC][16];
    __device__ __forceinline__ void load(const __bf16* src, int cq, const float* angles, const RopeArgs& rope) {
        const int rot = rope.rot_dim, half = rot / 2;
        // four angles from number i on; rot_dim and the tables make them 16-byte aligned
        auto four = [&](int i) { return *reinterpret_cast<const f32x4*>(angles + i); };
        if constexpr (TURN == kWholeHalves) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int d0 = cq * 16 + h * 8;
                const bf16x8 lower = *reinterpret_cast<const bf16x8*>(src + d0), upper = *reinterpret_cast<const bf16x8*>(src + d0 + D / 2);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const f32x4 cs4 = four(d0 + q * 4), sn4 = four(D / 2 + d0 + q * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const double x = (double)(float)lower[q * 4 + i], y = (double)(float)upper[q * 4 + i], cs = (double)cs4[i], sn = (double)sn4[i];
                        k[0][h * 8 + q * 4 + i] = __builtin_fma(x, cs, -(y * sn));
                        k[NC - 1][h * 8 + q * 4 + i] = __builtin_fma(x, sn, y * cs);
                    }
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int d0 = (cq + 4 * c) * 16 + h * 8;
                    const bf16x8 own = *reinterpret_cast<const bf16x8*>(src + d0);
                    double* const out = k[c] + h * 8;
                    if (d0 >= rot) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) out[i] = (double)(float)own[i];
                    } else if (rope.interleaved) {
                        const f32x4 cs = four(d0 / 2), sn = four(half + d0 / 2);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const double x = (double)(float)own[2 * i], y = (double)(float)own[2 * i + 1];
                            out[2 * i] = __builtin_fma(x, (double)cs[i], -(y * (double)sn[i]));
                            out[2 * i + 1] = __builtin_fma(x, (double)sn[i], y * (double)cs[i]);
                        }
                    } else {
                        const bool first = d0 < half;
                        const bf16x8 other = *reinterpret_cast<const bf16x8*>(src + (first ? d0 + half : d0 - half));
                        const int at = first ? d0 : d0 - half;
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const f32x4 cs = four(at + q * 4), sn = four(half + at + q * 4);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const double turn = (double)(first ? -sn[i] : sn[i]);
                                out[q * 4 + i] = __builtin_fma((double)(float)own[q * 4 + i], (double)cs[i], (double)(float)other[q * 4 + i] * turn);
                            }
                        }
                    }
                }
        }
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t t = 0;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) t = max(t, size_key(k[c][i]));
        return t;
    }
    __device__ __forceinline__ uint32_t codes(int c, int w, int s) const {
        const double down = __longlong_as_double((long long)(1023 + 127 - s) << 52);
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = round_to_odd(k[c][w * 4 + i] * down);
        return encode4(y);
    }
};

template <int D, int TURN>
__device__ __forceinline__ void append_block(const PagedBatch& b, const RopeArgs& rope, const RopeRows& x, int item, int head, char* lds) {
    constexpr int NC = D / 64;  // 16-element chunks per lane
    const int lane = threadIdx.x & 63, tok = lane & 15, cq = lane >> 4;
    const int first_row = b.new_start[0];
    // ---- which block of which request
    auto first_item = [&](int start, int r) { return (start - first_row + 30 * r) >> 4; };
    int r, start, prefix, n;
    if (b.num_reqs <= 64) {
        const int mine = min(lane, b.num_reqs - 1);
        const int starts = b.new_start[mine], prefixes = b.prefix_len[mine], news = b.new_len[mine];
        const uint64_t below = __builtin_amdgcn_ballot_w64(lane < b.num_reqs && first_item(starts, lane) <= item);
        r = 63 - __builtin_clzll(below);
        start = __builtin_amdgcn_readlane(starts, r);
        prefix = __builtin_amdgcn_readlane(prefixes, r);
        n = __builtin_amdgcn_readlane(news, r);
    } else {
        int lo = 0, hi = b.num_reqs;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first_item(b.new_start[mid], mid) <= item) lo = mid; else hi = mid;
        }
        r = lo;
        start = b.new_start[r];
        prefix = b.prefix_len[r];
        n = b.new_len[r];
    }
    const int p = item - first_item(start, r), offset = prefix & (kBlock - 1);
    if (n == 0 || p * kBlock >= offset + n) return;  // fewer blocks than there is room for
    const int have = p == 0 ? offset : 0;            // tokens the block holds already
    const int i0 = p == 0 ? 0 : p * kBlock - offset;  // first new token of the block
    const int end = min(kBlock, have + n - i0);
    const bool fresh = tok >= have && tok < end;
    const int blk = b.block_table[(long long)r * b.table_stride + (prefix >> 4) + p];
    // lanes without a token of their own take the nearest one's row
    const int i = i0 + min(max(tok, have), end - 1) - have;
    const long long row = start + i;
    Plain<NC> v;
    v.load(static_cast<const __bf16*>(x.v_new) + (row * b.kv_heads + head) * D, cq);
    const __bf16* const src_k = static_cast<const __bf16*>(x.k_new) + (row * b.kv_heads + head) * D;
    std::conditional_t<TURN == kAsItIs, Plain<NC>, Turned<D, TURN>> k;
    if constexpr (TURN == kAsItIs) k.load(src_k, cq);
    else k.load(src_k, cq, rope.cos_sin + (long long)(prefix + i) * rope.rot_dim, rope);

    uint8_t* const base_k = static_cast<uint8_t*>(x.pool_k) + (long long)blk * b.block_stride;
    uint8_t* const base_v = static_cast<uint8_t*>(x.pool_v) + (long long)blk * b.block_stride;
    const long long scale_at = (long long)b.kv_heads * (kBlock * D) + head, tile_at = (long long)head * (kBlock * D) + lane * 16;
    int old_k = 0, old_v = 0;
    if (have > 0) {
        old_k = base_k[scale_at];
        old_v = base_v[scale_at];
    }
    // the nearest token's row is one of the new ones, so no lane has to be left out
    uint32_t top_k = k.top(), top_v = v.top();
#pragma unroll
    for (int step = 32; step > 0; step >>= 1) {
        top_k = max(top_k, (uint32_t)__shfl_xor((int)top_k, step, 64));
        top_v = max(top_v, (uint32_t)__shfl_xor((int)top_v, step, 64));
    }
    const int sk = max(old_k, TURN == kAsItIs ? scale_byte_bf16(top_k) : scale_byte(top_k)), sv = max(old_v, scale_byte_bf16(top_v));

    // ---- K: a 16-byte piece per token and chunk
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        u32x4* const to = reinterpret_cast<u32x4*>(base_k + tile_at + c * 1024);
        if (fresh) {
            u32x4 codes;
#pragma unroll
            for (int w = 0; w < 4; ++w) codes[w] = k.codes(c, w, sk);
            *to = codes;
        } else if (tok < have && sk != old_k) {
            raise_held(reinterpret_cast<uint32_t*>(to), 4, ~0u, old_k - sk);
        }
    }

    // ---- V: the codes turn around in LDS, [token][element] with 4 bytes behind each row
    constexpr int LROW = D + 4;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int w = 0; w < 4; ++w) *reinterpret_cast<uint32_t*>(lds + tok * LROW + (cq + 4 * c) * 16 + w * 4) = v.codes(c, w, sv);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // other lanes of the wave read them
    const int t4 = cq * 4;  // this lane's four tokens, element 64 c + 16 w + lane % 16
    // bytes of the tokens below `to`
    auto bytes_to = [&](int to) { return to - t4 >= 4 ? ~0u : to <= t4 ? 0u : (1u << 8 * (to - t4)) - 1; };
    const uint32_t held = bytes_to(have), mask = bytes_to(end) & ~held;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        u32x4* const to = reinterpret_cast<u32x4*>(base_v + tile_at + c * 1024);
        if (held != 0 && sv != old_v) raise_held(reinterpret_cast<uint32_t*>(to), 4, held, old_v - sv);
        if (mask == 0) continue;
        u32x4 codes = u32x4(0);
        if (mask != ~0u) codes = *to;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t u = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) u |= (uint32_t)(uint8_t)lds[(t4 + e) * LROW + c * 64 + w * 16 + tok] << 8 * e;
            codes[w] = (u & mask) | (codes[w] & ~mask);
        }
        *to = codes;
    }
    if (lane == 0) {
        base_k[scale_at] = (uint8_t)sk;
        base_v[scale_at] = (uint8_t)sv;
    }
}

constexpr int kWaves = 4;
constexpr int kTurnHeads = 4;

template <int D, int TURN>
__global__ __launch_bounds__(64 * kWaves) void kv8_append_kernel(PagedBatch b, RopeArgs rope, RopeRows x, int block_groups, int head_groups, int rows, int q_groups) {
    __shared__ __attribute__((aligned(16))) char lds[kWaves][kBlock * (D + 4)];
    if ((int)blockIdx.x < block_groups) {
        const int w = threadIdx.x >> 6;
        const int head = (int)blockIdx.x % head_groups * kWaves + w;
        if (head < b.kv_heads) append_block<D, TURN>(b, rope, x, __builtin_amdgcn_readfirstlane((int)blockIdx.x / head_groups), __builtin_amdgcn_readfirstlane(head), lds[w]);
        return;
    }
    if constexpr (TURN != kAsItIs) {
        const int id = (int)blockIdx.x - block_groups;
        rope_rows<__bf16, kTurnHeads>(b, rope, x, 0, id / q_groups * rows, id % q_groups);
    }
}

template <int D, int TURN>
void launch_one(const PagedBatch& b, const RopeArgs& rope, const RopeRows& x, int grid, int block_groups, int head_groups, int rows, int q_groups, hipStream_t s) {
    hipLaunchKernelGGL((kv8_append_kernel<D, TURN>), dim3((unsigned)grid), dim3(64 * kWaves), 0, s, b, rope, x, block_groups, head_groups, rows, q_groups);
}

}  // namespace

hipError_t launch_kv8_append(const PagedBatch& b, const RopeArgs& rope, const RopeRows& x, hipStream_t s) {
    const int head_groups = (b.kv_heads + kWaves - 1) / kWaves;
    const long long items = ((long long)x.total_new + 30LL * b.num_reqs) >> 4;
    const int rows = 256 / (b.head_dim * 2 / 32), q_groups = (x.q_heads + kTurnHeads - 1) / kTurnHeads;
    const long long blocks = items * head_groups, turns = (long long)((x.total_new + rows - 1) / rows) * q_groups;
    if (blocks + turns > 0xffffff) return hipErrorInvalidValue;  // grid times workgroup size stays below 2^32 threads
    const int grid = (int)(blocks + turns);
    const auto launch = [&](auto kernel) { kernel(b, rope, x, grid, (int)blocks, head_groups, rows, q_groups, s); };
    if (b.head_dim == 64) launch(rope.rot_dim == 0 ? launch_one<64, kAsItIs> : launch_one<64, kAnyPairs>);
    else launch(rope.rot_dim == 0 ? launch_one<128, kAsItIs> : rope.rot_dim == 128 && !rope.interleaved ? launch_one<128, kWholeHalves> : launch_one<128, kAnyPairs>);
    return hipGetLastError();
}

}  // namespace ragc
