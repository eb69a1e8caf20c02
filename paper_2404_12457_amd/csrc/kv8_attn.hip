// Attention over the 8-bit cache for many rows: prompts and longer questions (plan_kv8 holds the rule).
//
// out[t,h,:] = softmax_j(scale * q[t,h,:].K_j) V_j over j = 0..prefix+i, every key and value from the request's blocks.
//
// Mapping.  One work item = (request, kv head, 128 rows[, copy]); a row is a (new token, q head of the group) pair, token-major, a wave
// owns 32 rows.  Keys come through LDS in tiles of 64 (four blocks), each wave bringing one block, with one barrier per tile: K
// straight into the tile, one step ahead, V a step earlier into a buffer of the wave's own, from where it is converted into the
// next tile.  Block ids and scales come the same way, 16 tiles at a time, so that no load into registers is ever waited for
// inside the loop.  NG wave groups of 4 waves work on the same rows but on alternating tiles, each with its own
// softmax state, merged through LDS at the end: NG = 2 where there are too few items to give every SIMD two waves.
//
// Products.  S^T = K Q^T takes K as it is, in 8 bits, on v_mfma_scale_f32_32x32x64_f8f6f4, which applies the blocks' scales.  A bf16 q
// has eight significant bits and is the sum of two e4m3 numbers of four: hi = the nearest to q 2^-e, with e from the row's
// largest |q| as in kv8_append.hip, and lo = the rest times 2^4 (exact as long as they stay normal numbers; below that
// off by at most 2^-14 of 2^e, 2^-21.8 of the largest |q|, which is above 224 2^e).  Two products at twice the rate of the bf16 ones take as long as one of those, and K needs no
// conversion and half the LDS reads.  The matrix unit lines up 16 products at a time with 16 bits below the largest and sums these in
// fp32: 8e-6 of sum |q k| on unit-variance numbers, 2^-12 of the largest product at worst.
// O^T += V^T P^T is v_mfma_f32_32x32x16_bf16: each wave turns its block of V into bf16 on the way into LDS (the conversion applies
// the scale; exact), once for all four waves, and stores it in the order in which operands are read.  The probabilities are bf16.
//
// Softmax, masks and the order of keys are those of attn_bf16_kernel: a lane owns one row and 32 of a tile's 64 keys, the
// row's reference exponent is raised only when a tile's probabilities against it sum to more than 2^8.
//
// What bounds it: matrix and vector units, of which the waves of a SIMD use one after the other more than side by side: of a CU's busy time
// the products take 0.52, vector instructions 0.47 (16 ragged requests, 32/8 heads of 128: 233 us, 1034 TFLOP/s of the 1236-1290 that a large bf16
// product reaches; the bf16 cache's kernel takes 289 for such a batch).  4 x (4096+128), 64/8 heads: 66.7 us, 1047 TFLOP/s.  A step of
// eight waves takes 4215 cycles at head_dim 128: 1090 for the scores, 1300 for softmax and V's conversion, 550 for P V as a wave sees them, and 1160 until its
// sister on the SIMD is done; the products of both need 2048.  At head_dim 64 the vector part is twice the products.
// What is brought for later steps is issued under the products: without a branch 71 instead of 77 us (4 x (4096+128)), and
// a wave in its products goes before one in its softmax (s_setprio): 69.  Measured within 2 % or slower: the scores of the next step
// among the softmax of this one, wave groups half a step apart, copies two steps ahead, K or V operands further ahead, row sums by
// fp32 adds or by products with ones.
#include "kv8_attn_common.h"

namespace ragc {
namespace {

constexpr int TM = kKv8TallRows;  // rows per work item
typedef __attribute__((ext_vector_type(8))) int i32x8;

// head_dim 64 stays within 128 registers: four waves to a SIMD, for 256 workgroups of eight waves or more 100.8 -> 84 us (32 x (2000+128),
// 32/8 heads), of four 84.5 -> 81.7.  head_dim 128 holds two.
template <int D, int NG, class Work>
__global__ __launch_bounds__(256 * NG, D == 64 ? 4 : NG == 1 ? 2 : 1) void kv8_attn_kernel(AttnLaunch a, Work wk) {
    constexpr int TILE = kBlock * D;    // bytes of one head's tile of a block
    constexpr int NC = D / 64;          // pieces of 1 KiB per tile
    constexpr int DB = D / 32;          // 32-column tiles of the output
    constexpr int KB = 4 * TILE;        // K of a 64-key tile in LDS
    constexpr int VB = 8 * TILE;        // V, in bf16
    constexpr int WIN = 6 * 256;        // a wave's windows of block ids, K scales and V scales: two of 64 dwords each
    constexpr int OWNB = TILE + WIN;    // what a wave has for itself: its block of V as it comes, its windows
    constexpr int GROUPB = 2 * (KB + VB) + 4 * OWNB;
    constexpr int OROWB = D * 2 + 16;   // a row of the output patch
    constexpr int WSTRIDE = (DB * 4 + 1) * 64 * 16;  // bytes per wave in the merge area: [DB*4 + 1][64 lanes] of 16
    static_assert(NG == 1 ? 4 * 32 * OROWB <= GROUPB : 4 * WSTRIDE <= NG * GROUPB && 32 * OROWB <= WSTRIDE, "merge area and output patches");
    __shared__ __attribute__((aligned(1024))) char smem[NG * GROUPB];
    __shared__ int nan_seen;  // a number that is not finite has been taken out of a V that not every row of the item sees

    touch_args(a, wk);
    const int Hkv = a.kv_heads;
    int g, entry;
    split_block_id(a, blockIdx.x, &g, &entry);
    entry += wk.entry0;
    const int tid = threadIdx.x, lane = tid & 63, kg = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = NG == 1 ? 0 : w >> 2, wq = w & 3;
    const WorkItem it = find_item(wk, entry, a.group, TM);
    const int G = a.group, N = it.new_len, P = it.prefix, s0 = it.new_start, Hq = a.q_heads;
    const uint32_t g_magic = a.group_magic;
    auto div_g = [&](int x) { return g_magic ? (int)__umulhi((uint32_t)x, g_magic) : x; };
    const int rows_total = N * G, tiles = (rows_total + TM - 1) / TM;
    // find_item counts items from the last tile down; here a request has `copies` entries per tile
    const int chunk = wk.splits, copies = copies_of(P + N, chunk);
    const int local = tiles - 1 - it.tile, copy = copies == 1 ? 0 : local % copies;
    const int row0 = (copies == 1 ? it.tile : tiles - 1 - local / copies) * TM;
    const int kv_limit = P + div_g(min(row0 + TM, rows_total) - 1) + 1;  // keys [0, kv_limit) are visible to some row of the item
    const int nblk = (kv_limit + kBlock - 1) / kBlock, all_tiles = (nblk + 3) / 4;
    // a copy may have no tile where this item sees less than the request's last row
    const int t_lo = copies == 1 ? 0 : min(copy * (chunk / 4), all_tiles), t_hi = copies == 1 ? all_tiles : min((copy + 1) * (chunk / 4), all_tiles);
    const int nsteps = (t_hi - t_lo + NG - 1) / NG;  // group grp takes tile t_lo + step*NG + grp
    const int32_t* __restrict__ table = a.block_table + (long long)it.req * a.table_stride;
    const uint8_t* __restrict__ pool_k = static_cast<const uint8_t*>(a.pool_k);
    const uint8_t* __restrict__ pool_v = static_cast<const uint8_t*>(a.pool_v);

    const int wrow0 = row0 + wq * 32;
    const bool wave_active = wrow0 < rows_total;
    const int my_row = min(wrow0 + l32, rows_total - 1), my_tok = div_g(my_row);  // rows past the end repeat the last one
    const int my_vis = P + my_tok + 1;
    const int wave_vis_min = P + div_g(min(wrow0, rows_total - 1)) + 1;
    const int wave_vis_max = P + div_g(min(wrow0 + 31, rows_total - 1)) + 1;

    typedef __attribute__((address_space(3))) char lds_char;
    typedef __attribute__((address_space(3))) uint32_t lds_u32;
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    lds_char* const lds0 = (lds_char*)smem + grp * GROUPB;  // [2][K tile], [2][V tile], then each wave's own
    lds_char* const lds_v = lds0 + 2 * KB;
    lds_char* const raw_v = lds0 + 2 * (KB + VB) + wq * OWNB;
    lds_u32* const win = reinterpret_cast<lds_u32*>(raw_v + TILE);  // [ids, K scales, V scales][2][64]
    auto lds_addr = [&](const __attribute__((address_space(3))) void* p) { return (uint32_t)(uintptr_t)p; };

    // ---- block ids and scales of 16 tiles of four blocks, one block per lane.  A scale comes with its three neighbours, the
    // dword around it.
    const int scales_at = Hkv * TILE + (g & ~3), scale_shift = 8 * (g & 3);
    auto block_of = [&](int step) { return min((t_lo + min(step + (lane >> 2), max(nsteps - 1, 0)) * NG + grp) * 4 + (lane & 3), nblk - 1); };
    const int first_id = table[block_of(0)];

    // ---- Q, elements 64 s + 32 kg .. + 31 of the row, under way with the first block ids
    bf16x8 qv[NC][4];
    {
        const __bf16* const qp = static_cast<const __bf16*>(a.q) + ((long long)(s0 + my_tok) * Hq + g * G + (my_row - my_tok * G)) * D + kg * 32;
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int x = 0; x < 4; ++x) qv[s][x] = *reinterpret_cast<const bf16x8*>(qp + s * 64 + x * 8);
    }
    asm volatile("" ::"v"(first_id));
#pragma unroll
    for (int s = 0; s < NC; ++s)
#pragma unroll
        for (int x = 0; x < 4; ++x) asm volatile("" ::"v"(qv[s][x]));  // here before the first copies, which nothing then waits for but the first step

    // ---- what a wave brings: block wq of a tile
    const uint32_t k_dst = lds_addr(lds0) + wq * TILE;
    const uint32_t run_off[2] = {(uint32_t)lane * 16, (uint32_t)lane * 16};
    auto copy_tile = [&](uint64_t src, uint32_t dst) {
        if constexpr (NC == 2) dma_runs<2>(src, run_off, dst);
        else dma_16B_per_lane(reinterpret_cast<const char*>(src) + lane * 16, dst);
    };
    auto window = [&](int step) { return (step >> 4 & 1) * 64 + 4 * (step & 15); };
    // V of a step's block, two steps ahead of its products; notes where its K is
    uint64_t k_src = 0;
    auto fetch = [&](int id) {
        const long long at = (long long)id * a.block_stride + (long long)g * TILE;
        k_src = uniform_u64(pool_k + at);
        copy_tile(uniform_u64(pool_v + at), lds_addr(raw_v));
    };
    auto id_of = [&](int step) { return __builtin_amdgcn_readfirstlane((int)win[window(step) + wq]); };
    // the next window, where there is a step for it: ids early in this one, scales when those are there.  More steps of this window
    // follow either copy, the first of which waits for it.
    auto next_window = [&](int step) {
        if ((step | 15) + 1 >= nsteps) return;
        const int to = ((step >> 4 & 1) ^ 1) * 64;
        if ((step & 15) == 2) dma_4B_per_lane(table + block_of((step | 15) + 1), lds_addr(win + to));
        if ((step & 15) == 6) {
            const long long scales = (long long)(int)win[to + lane] * a.block_stride + scales_at;
            dma_4B_per_lane(pool_k + scales, lds_addr(win + 128 + to));
            dma_4B_per_lane(pool_v + scales, lds_addr(win + 256 + to));
        }
    };
    // V of `step` from the wave's buffer into tile `slot`.  Lanes take token groups 0, 2, 1, 3, so that half a wave stores a run.
    const int tg_lane = ((lane >> 4) & 1) * 2 + (lane >> 5);
    lds_char* const v_from = raw_v + tg_lane * 256 + (lane & 15) * 16;
    lds_char* const v_dst = lds_v + wq * (2 * TILE) + (tg_lane & 1) * 512 + (lane & 15) * 16 + (tg_lane >> 1) * 8;
    const int vis_min = P + div_g(row0) + 1;
    u32x4 vreg[NC];
    uint32_t v_scale;  // and its neighbours
    auto read_scale = [&](int step) { v_scale = win[256 + window(step) + wq]; };
    auto read_raw = [&]() {
#pragma unroll
        for (int x = 0; x < NC; ++x) vreg[x] = *reinterpret_cast<const lds_u32x4*>(v_from + x * 1024);
    };
    auto check_raw = [&](int step) {
        const int key = (t_lo + step * NG + grp) * 64 + wq * kBlock;
        if (key + kBlock > vis_min) {
            // The frontier: slots behind the last visible key may hold anything and become 0.  What bf16 does not hold, in a key that some
            // rows see and others do not, would reach all through probabilities of 0: it becomes 0, and NaN is given to its rows at the end.
            const uint32_t keep = below(key + tg_lane * 4, kv_limit), to_top = not_finite_from(v_scale >> scale_shift & 255);
            uint32_t nan = 0;
#pragma unroll
            for (int x = 0; x < NC; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    vreg[x][e] &= keep;
                    nan |= nan_bytes(vreg[x][e], to_top);
                    vreg[x][e] = without_nan(vreg[x][e], to_top, below(key + tg_lane * 4, vis_min));
                }
            if (nan != 0) nan_seen = 1;
        }
    };
    auto store_v = [&](int tile, auto c_c) {  // one of the NC pieces; tile: byte offset of the V tile
        constexpr int C = decltype(c_c)::value;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int dt = C * 4 + e;  // elements 16 dt + lane % 16: row (dt / DB) * 16 + lane % 16 of column tile dt % DB
            *reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(v_dst + tile + (dt % DB) * 1024 + (dt / DB) * 256) = widen4(vreg[C][e], scale_of(v_scale >> scale_shift & 255));
        }
    };

    // ---- the first tile, and under it the parts of Q
    int q_scale, q_scale_lo;  // e + 127 and that of the lo part
    i32x8 qhi[NC], qlo[NC];
    {
        const long long at = (long long)first_id * a.block_stride + scales_at;
        const uint32_t ks = *reinterpret_cast<const uint32_t*>(pool_k + at), vs = *reinterpret_cast<const uint32_t*>(pool_v + at);
        win[lane] = (uint32_t)first_id;
        if (tid == 0) nan_seen = 0;
        if (nsteps > 0) {
            fetch(__builtin_amdgcn_readlane(first_id, wq));
            copy_tile(k_src, k_dst);
        }
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t u = __float_as_uint((float)qv[s][x][e]) & 0x7fffffffu;
                    top = max(top, u);
                }
        top = max(top, __float_as_uint(other_half(__uint_as_float(top))));
        const bool bad = top >= 0x7f800000u;
        // 448 = 1.75 * 2^8; a row of numbers below 2^-118 is far from mattering to any score
        q_scale = max(5, (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u));
        q_scale_lo = q_scale - 4;
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                float f[4], r[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = __builtin_ldexpf((float)qv[s][x >> 1][(x & 1) * 4 + e], 127 - q_scale);
                int hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
                hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], hi, true);
                const bf16x4 back = widen4((uint32_t)hi, 1.f);
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = (f[e] - (float)back[e]) * 16.f;  // at most half a step of hi, 16, times 16
                int lo = __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], 0, false);
                lo = __builtin_amdgcn_cvt_pk_fp8_f32(r[2], r[3], lo, true);
                qhi[s][x] = bad ? (int)kNoNan : hi;  // a row with a number that is not finite is NaN: 0x7f four times
                qlo[s][x] = bad ? 0 : lo;
            }
        win[128 + lane] = ks;
        win[256 + lane] = vs;
    }

    f32x16 oacc[DB];
#pragma unroll
    for (int t = 0; t < DB; ++t) oacc[t] = f32x16(0.f);
    float m_run = -INFINITY, l_run = 0.f;
    const float c = a.scale_log2e;
    const int k_lane = (l32 >> 4) * TILE + (l32 & 15) * 16 + kg * 512;

    // One step.  FAST: two more steps follow, every key of this tile and of the next is visible to every row, the wave has rows: no branch
    // stands between the products and what is brought under them (the compiler would move products behind it).
    auto do_step = [&](int step, auto fast_c) {
        constexpr bool FAST = decltype(fast_c)::value;
        const int k_now = (step & 1) * KB, k_next = KB - k_now, v_now = (step & 1) * VB, v_next = VB - v_now;
        wait_vmcnt<0>();  // K of this step, V of the next and what windows were asked for have arrived
        block_barrier();  // every wave's part is in LDS, and every wave is done with the previous step
        next_window(step);
        const bool more = FAST || step + 1 < nsteps;
        const int tg = t_lo + step * NG + grp, key0 = tg * 64;
        if (!FAST) {
            // what the next steps need, before the products: there are one or two such steps in an item
            if (more) {
                copy_tile(k_src, k_dst + k_next);
                read_scale(step + 1);
                read_raw();
                check_raw(step + 1);
                static_for<NC>([&](auto c_c) { store_v(v_next, c_c); });
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read: its buffer is free
                if (step + 2 < nsteps) fetch(id_of(step + 2));
            }
            if (!wave_active || tg >= t_hi || key0 >= wave_vis_max) return;
        }
        lds_char* const kst = lds0 + k_now + k_lane;
        lds_char* const vst = lds_v + v_now + lane * 16;
        // S^T = K Q^T; operands are read a step of the contraction ahead
        f32x16 sacc[2] = {f32x16(0.f), f32x16(0.f)};
        i32x8 kbuf[NC][2];
        auto read_k = [&](int s) {
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                const u32x4 k0 = *reinterpret_cast<const lds_u32x4*>(kst + sub * 2 * TILE + s * 1024);
                const u32x4 k1 = *reinterpret_cast<const lds_u32x4*>(kst + sub * 2 * TILE + s * 1024 + 256);
                if (s == 0) __builtin_amdgcn_sched_barrier(0);  // the first product's operands arrive first
                kbuf[s][sub] = i32x8{(int)k0[0], (int)k0[1], (int)k0[2], (int)k0[3], (int)k1[0], (int)k1[1], (int)k1[2], (int)k1[3]};
            }
        };
        // the small ones first, so that one trip to LDS brings all that the products and V's conversion start from
        uint32_t k_raw[2], id_raw = 0;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) k_raw[sub] = win[128 + window(step) + 2 * sub + (l32 >> 4)];
        if constexpr (FAST) {
            read_scale(step + 1);
            id_raw = win[window(step + 2) + wq];
        }
        __builtin_amdgcn_sched_barrier(0);
        read_k(0);
        if constexpr (FAST) read_raw();
        __builtin_amdgcn_sched_barrier(0);
        int k_scale[2];
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) k_scale[sub] = (int)(k_raw[sub] >> scale_shift);  // byte 0 counts
        __builtin_amdgcn_s_setprio(1);
        static_for<NC>([&](auto s_c) {
            constexpr int S = decltype(s_c)::value;
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (S + 1 < NC) read_k(S + 1);
            if constexpr (FAST && S == 0) copy_tile(k_src, k_dst + k_next);
            sacc[0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kbuf[S][0], qhi[S], sacc[0], 0, 0, 0, k_scale[0], 0, q_scale);
            sacc[1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kbuf[S][1], qhi[S], sacc[1], 0, 0, 0, k_scale[1], 0, q_scale);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (FAST) store_v(v_next, s_c);
            sacc[0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kbuf[S][0], qlo[S], sacc[0], 0, 0, 0, k_scale[0], 0, q_scale_lo);
            sacc[1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kbuf[S][1], qlo[S], sacc[1], 0, 0, 0, k_scale[1], 0, q_scale_lo);
        });
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        // V operands two groups ahead, the first ones under the softmax; at head_dim 64, where four waves share a SIMD, one ahead and none
        // in registers over the softmax
        constexpr int VGROUPS = 4 * DB / 2;
        constexpr int AHEAD = D == 64 ? 1 : 2;
        bf16x8 vbuf[AHEAD + 1][2];
        auto read_v = [&](auto g_c) {
            constexpr int GI = decltype(g_c)::value;
#pragma unroll
            for (int x = 0; x < 2; ++x)
                vbuf[GI % (AHEAD + 1)][x] = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>(vst + (2 * GI + x) / DB * (2 * TILE) + (2 * GI + x) % DB * 1024);
        };
        if constexpr (AHEAD > 1) {
            read_v(std::integral_constant<int, 0>{});
            read_v(std::integral_constant<int, 1>{});
        }
        if constexpr (FAST) {
#pragma unroll
            for (int x = 0; x < NC; ++x) asm volatile("" ::"v"(vreg[x]));  // V has been read: its buffer is free
            fetch(__builtin_amdgcn_readfirstlane((int)id_raw));
        }
        if (!FAST && key0 + 64 > wave_vis_min) {
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + sub * 32 + (i >> 2) * 8 + kg * 4 + (i & 3) >= my_vis) sacc[sub][i] = -INFINITY;
        }
        bf16x8 pb[4];
        float psum;
        auto weigh = [&](float m_sub) {
            psum = 0.f;
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const bf16x2 pp = {(__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(sacc[sub][i], c, -m_sub)),
                                       (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(sacc[sub][i + 1], c, -m_sub))};
                    psum = __builtin_amdgcn_fdot2_f32_bf16(pp, kOnes2, psum, false);
                    pb[sub * 2 + (i >> 3)][i & 7] = pp[0];
                    pb[sub * 2 + (i >> 3)][(i & 7) + 1] = pp[1];
                }
        };
        bool raise_any = step == 0;
        if (!raise_any) {
            weigh(m_run);
            raise_any = __builtin_amdgcn_ballot_w64(!(psum <= kRaiseSum)) != 0;
        }
        if (__builtin_expect(raise_any, false)) {
            float mx = sacc[0][0];
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sacc[sub][i]);
            mx = fmaxf(mx, other_half(mx)) * c;
            const bool raise = mx > m_run;
            const float alpha = raise ? __builtin_amdgcn_exp2f(m_run - mx) : 1.f;  // 0 where the row has no reference yet
            m_run = raise ? mx : m_run;
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < DB; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) oacc[t][i] *= alpha;
            weigh(m_run == -INFINITY ? 0.f : m_run);  // still no visible key: exp2(-inf - 0) = 0
        }
        l_run += psum;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (AHEAD == 1) read_v(std::integral_constant<int, 0>{});
        __builtin_amdgcn_s_setprio(1);
        static_for<VGROUPS>([&](auto g_c) {
            constexpr int GI = decltype(g_c)::value;
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (GI + AHEAD < VGROUPS) read_v(std::integral_constant<int, GI + AHEAD>{});
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                f32x16& o = oacc[(2 * GI + x) % DB];
                o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vbuf[GI % (AHEAD + 1)][x], pb[2 * GI / DB], o, 0, 0, 0);
            }
        });
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
    };

    if (nsteps > 0) {
        wait_vmcnt<0>();
        read_scale(0);
        read_raw();
        block_barrier();  // nan_seen is 0
        check_raw(0);
        static_for<NC>([&](auto c_c) { store_v(0, c_c); });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (nsteps > 1) fetch(__builtin_amdgcn_readlane(first_id, 4 + wq));
        // steps whose tile and the next lie below vis_min, with two more behind them
        const int clear = vis_min / 64 - t_lo - grp;  // tiles of this group from t_lo + grp on, in tiles
        const int fast = wave_active ? max(0, min(nsteps - 2, clear <= 0 ? 0 : (clear + NG - 1) / NG - 1)) : 0;
        int step = 0;
        for (; step < fast; ++step) do_step(step, std::true_type{});
        for (; step < nsteps; ++step) do_step(step, std::false_type{});
    }

    // ---- merge the wave groups through LDS.  The copies' areas are reused: none is under way, as each was asked for by a step before
    // the last; the wait is there for those who change that, and costs nothing.
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    lds_char* const lds = (lds_char*)smem;
    auto piece = [&](int t, int q) { return f32x4{oacc[t][q * 4], oacc[t][q * 4 + 1], oacc[t][q * 4 + 2], oacc[t][q * 4 + 3]}; };
    wait_vmcnt<0>();
    block_barrier();  // every wave is done with the tiles: their memory is reused below
    if (nan_seen) {
        // The keys of the frontier once more: a row that sees what was taken out has NaN in the output.
        for (int key = vis_min; key < my_vis; ++key) {
            const uint8_t* const block = pool_v + (long long)table[key >> 4] * a.block_stride;
            const uint8_t* const tile = block + (long long)g * TILE;
            const uint32_t to_top = not_finite_from(block[(long long)Hkv * TILE + g]);
#pragma unroll
            for (int t = 0; t < DB; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int m = (i >> 2) * 8 + kg * 4 + (i & 3), d = (D / 2) * (m >> 4) + 16 * t + (m & 15);
                    if (nan_bytes(tile[(((d >> 6) * 4 + ((key & 15) >> 2)) * 16 + (d & 15)) * 16 + ((d & 63) >> 4) * 4 + (key & 3)], to_top & 0xff) & 0x80) oacc[t][i] = __builtin_nanf("");
                }
        }
    }
    if (NG > 1) {
        lds_f32x4* const xw = reinterpret_cast<lds_f32x4*>(lds + wq * WSTRIDE) + lane;
        if (grp == 1) {
#pragma unroll
            for (int t = 0; t < DB; ++t)
#pragma unroll
                for (int q = 0; q < 4; ++q) xw[(t * 4 + q) * 64] = piece(t, q);
            xw[DB * 4 * 64] = f32x4{m_run, l_run, 0.f, 0.f};
        }
        block_barrier();
        if (grp == 1) return;
        if (wave_active) {
            const f32x4 ml = xw[DB * 4 * 64];
            // a group may have seen no visible key of a row: weight 0 (which lets NaN through)
            const float m = fmaxf(m_run, ml[0]);
            const float w0 = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m);
            const float w1 = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - m);
            m_run = m;
            l_run = l_run * w0 + ml[1] * w1;
#pragma unroll
            for (int t = 0; t < DB; ++t)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 v = xw[(t * 4 + q) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) oacc[t][q * 4 + e] = oacc[t][q * 4 + e] * w0 + v[e] * w1;
                }
        }
    }

    // ---- normalise and store whole rows, turned around in a patch of LDS that only this wave reads.  A lane holds, of one row, elements
    // D/2 (q/2) + 16 t + 8 (q%2) + 4 kg .. + 3.
    if (!wave_active) return;
    constexpr int CPR = D / 8, RPI = 64 / CPR;  // 16-byte chunks per bf16 row, rows per store instruction
    lds_char* const patch = lds + wq * (NG > 1 ? WSTRIDE : 32 * OROWB);
    const float l_tot = l_run + other_half(l_run);
    if (copies > 1) {
        // O (unnormalised, fp32), max and sum of every row go to the workspace, half of the columns at a time
        float* const part = static_cast<float*>(a.partial) + ((long long)(wk.part_base + entry) * Hkv + g) * (TM * (D + 2));
        if (kg == 0) *reinterpret_cast<float2*>(part + TM * D + (wq * 32 + l32) * 2) = float2{m_run, l_tot};
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
            for (int t = 0; t < DB; ++t)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    *reinterpret_cast<lds_f32x4*>(patch + l32 * OROWB + (16 * t + 8 * q + 4 * kg) * 4) = l_tot == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : piece(t, pass * 2 + q);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int p = 0; p < 32 / RPI; ++p) {
                const int rr = p * RPI + lane / CPR;
                const f32x4 v = *reinterpret_cast<const lds_f32x4*>(patch + rr * OROWB + (lane % CPR) * 16);
                *reinterpret_cast<f32x4*>(part + (wq * 32 + rr) * D + pass * (D / 2) + (lane % CPR) * 4) = v;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the patch is rewritten by the next pass
        }
        return;
    }
    const float inv = 1.f / l_tot;
#pragma unroll
    for (int t = 0; t < DB; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            bf16x4 o4;
#pragma unroll
            for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(oacc[t][q * 4 + e] * inv);
            *reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(patch + l32 * OROWB + ((D / 2) * (q >> 1) + 16 * t + 8 * (q & 1) + 4 * kg) * 2) = o4;
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // other lanes of the wave read them
#pragma unroll
    for (int p = 0; p < 32 / RPI; ++p) {
        const int rr = p * RPI + lane / CPR, row = wrow0 + rr;
        const u32x4 v = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(patch + rr * OROWB + (lane % CPR) * 16);
        if (row < rows_total) {
            const int tok = div_g(row);
            *reinterpret_cast<u32x4*>(static_cast<__bf16*>(a.out) + ((long long)(s0 + tok) * Hq + g * G + (row - tok * G)) * D + (lane % CPR) * 8) = v;
        }
    }
}

template <int D, int NG, class Work>
void launch_one(const AttnLaunch& a, const Work& wk, int entries, hipStream_t s) {
    hipLaunchKernelGGL((kv8_attn_kernel<D, NG, Work>), dim3((unsigned)entries * a.kv_heads), dim3(256 * NG), 0, s, a, wk);
}
template <class Work>
void launch_list(const AttnLaunch& a, const Work& wk, int entries, int waves, hipStream_t s) {
    if (a.head_dim == 64) waves == 8 ? launch_one<64, 2>(a, wk, entries, s) : launch_one<64, 1>(a, wk, entries, s);
    else waves == 8 ? launch_one<128, 2>(a, wk, entries, s) : launch_one<128, 1>(a, wk, entries, s);
}

}  // namespace

hipError_t launch_kv8_attn(const AttnLaunch& a, const AttnWork& wk, int entries, int waves, hipStream_t s) {
    if (entries <= 0) return hipSuccess;
    wk.n_reqs <= kAttnReqStep ? launch_list(a, short_list(wk), entries, waves, s) : launch_list(a, wk, entries, waves, s);
    return hipGetLastError();
}

}  // namespace ragc
