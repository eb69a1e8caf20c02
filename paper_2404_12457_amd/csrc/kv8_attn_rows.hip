// Attention over the 8-bit cache for few rows: decode steps and short questions (plan_kv8 holds the rule).
//
// out[t,h,:] = softmax_j(scale * q[t,h,:].K_j) V_j over j = 0..prefix+i, every key and value from the request's blocks.
//
// Mapping.  One workgroup = (request, kv head, 16 RT rows[, copy]); a row is a (new token, q head of the group) pair, token-major.
// Its NW waves take every NW-th pair of blocks (32 keys) of the copy's range, each with its own online softmax state, and the
// states are combined through LDS at the end; copies of a long range leave theirs in the workspace for kv8_merge_kernel.
//
// What bounds it: the cache's bytes.  Nothing goes through LDS on the way: the pool's layout is the one in which the matrix cores
// take operands, so a wave's loads are runs of 1 KiB straight into the registers they are used from, the next pair of blocks
// under way during the products of this one.  K and V become bf16 by the conversion that applies the block's scale (exact), and the
// products are those of the bf16 kernels, on v_mfma_f32_16x16x32_bf16: S^T = K Q^T, O^T += V^T P^T, a lane has one row
// and four keys of each block, which is also how it holds V.  The probabilities are rounded to bf16 for the product, like those of
// the bf16 kernels, and the row sum is taken over the rounded ones.
//
// Measured over three states in rotation (none stays in a cache): 64 requests of 512-2048 keys, a token each, 64/8 heads of 128, 35.0 us with 4
// waves, two workgroups to a CU, 34.1 with 8 (4.7 and 4.8 TB/s: the longest requests run on when the rest is done; 63 of 2000 keys, 32/8
// heads, 5.2 TB/s); 128 of 200-1000, 32/8 heads, 32.8 and 37.4; the first of head_dim 64 19.0 (4.3 TB/s, the same tail).  Two row tiles (32
// rows), four tokens of each of those requests: 37.9 and 38.3; 512 items of 2064 keys that two share 36.7 and 41.1, 256 of 4320 that four share 34.8
// and 28.1.
// Windows of ids through LDS, or two pairs of blocks under way, changed nothing.
#include "kv8_attn_common.h"

namespace ragc {
namespace {

template <int D, int RT, int NW, class Work>
__global__ __launch_bounds__(64 * NW, 2) void kv8_attn_rows_kernel(AttnLaunch a, Work wk) {
    constexpr int TR = 16 * RT;        // rows per workgroup
    constexpr int TILE = kBlock * D;   // bytes of one head's tile of a block
    constexpr int NC = D / 64;         // 16-byte pieces per lane and tile
    constexpr int DT = D / 16;         // 16-column tiles of the output
    constexpr int OCH = D / 4;         // 16-byte chunks of a fp32 output row
    __shared__ __attribute__((aligned(16))) char smem[NW * TR * D * 4];
    __shared__ float2 MLs[NW][TR];  // (max, sum) of every wave and row

    touch_args(a, wk);
    const int Hkv = a.kv_heads;
    int g, entry;
    split_block_id(a, blockIdx.x, &g, &entry);
    entry += wk.entry0;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, kg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    WorkItem it = find_item(wk, entry, a.group, TR);
    const int G = a.group, N = it.new_len, P = it.prefix, s0 = it.new_start, Hq = a.q_heads;
    const uint32_t g_magic = a.group_magic;
    auto div_g = [&](int x) { return g_magic ? (int)__umulhi((uint32_t)x, g_magic) : x; };
    const int rows_total = N * G;
    // find_item counts items from the last tile down; here a request has `copies` entries per tile
    const int chunk = wk.splits, copies = copies_of(P + N, chunk);
    const int local = (rows_total + TR - 1) / TR - 1 - it.tile, copy = copies == 1 ? 0 : local % copies;
    const int row0 = (copies == 1 ? it.tile : (rows_total + TR - 1) / TR - 1 - local / copies) * TR;
    const int rows_here = min(TR, rows_total - row0);
    const int kv_limit = P + div_g(row0 + rows_here - 1) + 1;  // keys [0, kv_limit) are visible to some row
    const int vis_min = P + div_g(row0) + 1;
    const int nblk = (kv_limit + kBlock - 1) / kBlock;
    // pairs of blocks [lo, hi) of this copy; a copy may have none where the tile's last row sees less than the request's
    const int lo = copy * chunk / 2, hi = chunk == 0 ? (nblk + 1) / 2 : min((copy + 1) * chunk / 2, (nblk + 1) / 2);
    const int nsteps = hi - lo > w ? (hi - lo - w + NW - 1) / NW : 0;

    const int32_t* __restrict__ table = a.block_table + (long long)it.req * a.table_stride;
    const uint8_t* __restrict__ pool_k = static_cast<const uint8_t*>(a.pool_k);
    const uint8_t* __restrict__ pool_v = static_cast<const uint8_t*>(a.pool_v);
    const int scales_at = Hkv * TILE + g;

    // block ids and scale bytes of this wave's pairs, 32 steps of two at a time, one per lane
    int base = 0, ids = 0, sk = 0, sv = 0;
    auto block_at = [&](int step) { return min((lo + w + (step + (lane >> 1)) * NW) * 2 + (lane & 1), nblk - 1); };
    auto window = [&](int step) {
        base = step;
        ids = table[block_at(step)];
        const long long at = (long long)ids * a.block_stride + scales_at;
        sk = pool_k[at];
        sv = pool_v[at];
    };

    // Q, B operand of S^T: row l16, elements 16 (kg + 4 c) + 8 h .. + 7
    bf16x8 qreg[RT][NC][2];
    int vis[RT];
    if (nsteps > 0) ids = table[block_at(0)];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = row0 + min(rt * 16 + l16, rows_here - 1), tok = div_g(row);  // rows past the end repeat the last one
        vis[rt] = P + tok + 1;
        const __bf16* const qp = static_cast<const __bf16*>(a.q) + ((long long)(s0 + tok) * Hq + g * G + (row - tok * G)) * D + kg * 16;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) qreg[rt][c][h] = *reinterpret_cast<const bf16x8*>(qp + c * 64 + h * 8);
    }

    struct Pair {
        u32x4 k[2][NC], v[2][NC];
    };
    auto load = [&](int step, Pair* p) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int id = __builtin_amdgcn_readlane(ids, 2 * (step - base) + b);
            const long long at = (long long)id * a.block_stride + (long long)g * TILE;
            const u32x4* const pk = reinterpret_cast<const u32x4*>(pool_k + at);
            const u32x4* const pv = reinterpret_cast<const u32x4*>(pool_v + at);
#pragma unroll
            for (int c = 0; c < NC; ++c) p->k[b][c] = pk[c * 64 + lane];
#pragma unroll
            for (int c = 0; c < NC; ++c) p->v[b][c] = pv[c * 64 + lane];
        }
    };

    f32x4 oacc[RT][DT];
    float m_run[RT], l_run[RT];  // as in attn_bf16_rows_kernel
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m_run[rt] = -INFINITY;
        l_run[rt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) oacc[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float c = a.scale_log2e;

    auto work = [&](int step, Pair& p, int sk_now, int sv_now) {
        const int key0 = (lo + w + step * NW) * 32;
        float scale_v[2];
        f32x4 s[RT][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const float scale_k = scale_of(b ? sk_now >> 8 : sk_now & 255);
            scale_v[b] = scale_of(b ? sv_now >> 8 : sv_now & 255);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int cc = 0; cc < NC; ++cc)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bf16x8 kk = join(widen4(p.k[b][cc][2 * h], scale_k), widen4(p.k[b][cc][2 * h + 1], scale_k));
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) s[rt][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qreg[rt][cc][h], s[rt][b], 0, 0, 0);
                }
        }
        if (key0 + 32 > vis_min) {
            // The frontier.  What a row does not see weighs nothing, whatever the bytes there are: scores are replaced, V behind the
            // last visible key becomes 0, and what bf16 does not hold in a V that some rows see and others do not goes to the former as NaN, by a
            // product of where such numbers are with who sees them.
            uint32_t nan = 0;
            const uint32_t to_top[2] = {not_finite_from(sv_now & 255), not_finite_from(sv_now >> 8)};
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int key = key0 + 16 * b + 4 * kg;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (key + r >= vis[rt]) s[rt][b][r] = -INFINITY;
                const uint32_t keep = below(key, kv_limit);
#pragma unroll
                for (int cc = 0; cc < NC; ++cc)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p.v[b][cc][e] &= keep;
                        nan |= nan_bytes(p.v[b][cc][e], to_top[b]);
                    }
            }
            if (kv_limit > vis_min && __builtin_amdgcn_ballot_w64(nan != 0) != 0) {
                bf16x8 sees[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sees[rt][e] = key0 + 16 * (e >> 2) + 4 * kg + (e & 3) < vis[rt] ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll
                for (int cc = 0; cc < NC; ++cc)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bf16x8 at = join(widen4(where_nan(p.v[0][cc][e], to_top[0]), 1.f), widen4(where_nan(p.v[1][cc][e], to_top[1]), 1.f));
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(at, sees[rt], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (n[r] > 0.f) oacc[rt][cc * 4 + e][r] = __builtin_nanf("");
                        }
                        p.v[0][cc][e] = without_nan(p.v[0][cc][e], to_top[0]);
                        p.v[1][cc][e] = without_nan(p.v[1][cc][e], to_top[1]);
                    }
            }
        }
        bf16x8 pb[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float mx = s[rt][0][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[rt][e >> 2][e & 3]);
            if (__builtin_amdgcn_ballot_w64(mx * c > m_run[rt] + kRescaleThreshold) != 0) {
                mx = fmaxf(mx, other_half(mx));
                mx = fmaxf(mx, other_quarter(mx)) * c;
                const bool raise = mx > m_run[rt] + kRescaleThreshold;  // true on a row's first visible pair (m_run = -inf)
                const float alpha = raise ? __builtin_amdgcn_exp2f(m_run[rt] - mx) : 1.f;
                m_run[rt] = raise ? mx : m_run[rt];
                l_run[rt] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) oacc[rt][dt][r] *= alpha;
            }
            const float m_sub = m_run[rt] == -INFINITY ? 0.f : m_run[rt];  // a row without a visible key yet: exp2(-inf - 0) = 0
            float psum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const bf16x2 pp = {(__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e >> 2][e & 3], c, -m_sub)),
                                   (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e >> 2][(e & 3) + 1], c, -m_sub))};
                psum = __builtin_amdgcn_fdot2_f32_bf16(pp, kOnes2, psum, false);
                pb[rt][e] = pp[0];
                pb[rt][e + 1] = pp[1];
            }
            l_run[rt] += psum;
        }
#pragma unroll
        for (int cc = 0; cc < NC; ++cc)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bf16x8 vv = join(widen4(p.v[0][cc][e], scale_v[0]), widen4(p.v[1][cc][e], scale_v[1]));
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) oacc[rt][cc * 4 + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pb[rt], oacc[rt][cc * 4 + e], 0, 0, 0);
            }
    };

    if (nsteps > 0) {
        {
            const long long at = (long long)ids * a.block_stride + scales_at;
            Pair p[2];
            load(0, &p[0]);
            sk = pool_k[at];
            sv = pool_v[at];
            auto bytes = [&](int x, int step) {  // both blocks' bytes of a step
                return __builtin_amdgcn_readlane(x, 2 * (step - base)) | __builtin_amdgcn_readlane(x, 2 * (step - base) + 1) << 8;
            };
            auto turn = [&](int step, Pair& now, Pair& next) {
                const int sk_now = bytes(sk, step), sv_now = bytes(sv, step);
                if (step + 1 < nsteps) {
                    if (step + 1 - base >= 32) window(step + 1);
                    load(step + 1, &next);
                }
                work(step, now, sk_now, sv_now);
            };
            for (int step = 0; step < nsteps; step += 2) {
                turn(step, p[0], p[1]);
                if (step + 1 < nsteps) turn(step + 1, p[1], p[0]);
            }
        }
    }

    // ---- combine the waves' states, as attn_bf16_rows_kernel does: a wave that has seen no key of a row has l = 0 there and
    // counts nothing; one whose scores were NaN has l = NaN next to m = -inf, which must reach the output
    typedef __attribute__((address_space(3))) char lds_char;
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    lds_char* const own = (lds_char*)smem + w * (TR * D * 4);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float l = l_run[rt];
        l += other_half(l);
        l += other_quarter(l);
        const int r = rt * 16 + l16;
        if (kg == 0) MLs[w][r] = float2{m_run[rt], l};
        if (r < rows_here) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const f32x4 o = l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : oacc[rt][dt];
                *reinterpret_cast<lds_f32x4*>(own + r * (D * 4) + (((dt * 4 + kg) ^ (r & (OCH - 1))) << 4)) = o;
            }
        }
    }
    __syncthreads();
    constexpr int TPR = D / 8;  // threads per row: 8 columns each
    for (int idx = tid; idx < rows_here * TPR; idx += 64 * NW) {
        const int r = idx / TPR, c8 = idx % TPR;
        float2 ml[NW];
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            ml[x] = MLs[x][r];
            m = fmaxf(m, ml[x].x);
        }
        f32x4 o[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            const float wgt = ml[x].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[x].x - m);
            l += ml[x].y * wgt;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 v = *reinterpret_cast<const lds_f32x4*>((lds_char*)smem + x * (TR * D * 4) + r * (D * 4) + (((2 * c8 + h) ^ (r & (OCH - 1))) << 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) o[h][e] += v[e] * wgt;
            }
        }
        if (copies > 1) {
            float* const part = static_cast<float*>(a.partial) + ((long long)(wk.part_base + entry) * Hkv + g) * (TR * (D + 2));
            if (c8 == 0) *reinterpret_cast<float2*>(part + TR * D + r * 2) = float2{m, l};
            *reinterpret_cast<f32x4*>(part + r * D + c8 * 8) = o[0];
            *reinterpret_cast<f32x4*>(part + r * D + c8 * 8 + 4) = o[1];
        } else {
            const float inv = 1.f / l;
            const int row = row0 + r, tok = div_g(row);
            bf16x8 ob;
#pragma unroll
            for (int e = 0; e < 8; ++e) ob[e] = (__bf16)(o[e >> 2][e & 3] * inv);
            *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(a.out) + ((long long)(s0 + tok) * Hq + g * G + (row - tok * G)) * D + c8 * 8) = ob;
        }
    }
}

// Combines the copies' states of every row: out = sum_c O_c 2^(m_c - m) / sum_c l_c 2^(m_c - m), m = max_c m_c.  The list holds the
// requests that have more than one copy, an item per row tile, and in place of a request's number the slot of its first
// entry.  A thread has four columns of a row and every SHARE-th copy; a workgroup 256 / SHARE of these, of the rows of one (tile, kv
// head).  Few rows have many copies (decode steps), where many rows share the work there are few.
// Bounded by the trips to memory: one step of 100003 keys in 31 copies, 64/8 heads, 4.7 us after 40.4 of the products' kernel.
template <int D, int TR, int SHARE, class Work>
__global__ __launch_bounds__(256) void kv8_merge_kernel(AttnLaunch a, Work wk, int row_groups) {
    constexpr int TPR = D / 4, RPW = 256 / (TPR * SHARE);
    __shared__ f32x4 os[SHARE][RPW][TPR];
    __shared__ float2 mls[SHARE][RPW];
    const int Hkv = a.kv_heads;
    const int item = blockIdx.x / (row_groups * Hkv) + wk.entry0, g = blockIdx.x / row_groups % Hkv;
    const WorkItem it = find_item(wk, item, a.group, TR);
    const int G = a.group, rows_total = it.new_len * G, tiles = (rows_total + TR - 1) / TR;
    const int copies = copies_of(it.prefix + it.new_len, wk.splits);
    // entries go from the last tile down, a tile's copies in a row
    const int slot = it.req + (tiles - 1 - it.tile) * copies;
    const int grp = threadIdx.x / (TPR * RPW), rr = threadIdx.x / TPR % RPW, d4 = threadIdx.x % TPR;
    const int r = blockIdx.x % row_groups * RPW + rr, row = it.tile * TR + r;
    if (row - rr >= rows_total) return;
    constexpr int PART = TR * (D + 2);
    const float* const part0 = static_cast<const float*>(a.partial) + ((long long)slot * Hkv + g) * PART;
    const long long copy_stride = (long long)Hkv * PART;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float m1, float l1, f32x4 o1) {
        const float top = fmaxf(m, m1);
        const float w0 = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top), w1 = l1 == 0.f ? 0.f : __builtin_amdgcn_exp2f(m1 - top);
        l = l * w0 + l1 * w1;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * w0 + o1[e] * w1;
        m = top;
    };
    constexpr int AHEAD = 4;
    if (row < rows_total) {  // rows behind the last were not written
        for (int c0 = grp; c0 < copies; c0 += SHARE * AHEAD) {
            float2 ml[AHEAD];
            f32x4 oc[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const float* const pc = part0 + min(c0 + u * SHARE, copies - 1) * copy_stride;
                ml[u] = *reinterpret_cast<const float2*>(pc + TR * D + r * 2);
                oc[u] = *reinterpret_cast<const f32x4*>(pc + r * D + d4 * 4);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (c0 + u * SHARE < copies) add(ml[u].x, ml[u].y, oc[u]);
        }
    }
    if (SHARE > 1) {
        os[grp][rr][d4] = o;
        if (d4 == 0) mls[grp][rr] = float2{m, l};
        __syncthreads();
        if (grp != 0) return;
#pragma unroll
        for (int x = 1; x < SHARE; ++x) add(mls[x][rr].x, mls[x][rr].y, os[x][rr][d4]);
    }
    if (row >= rows_total) return;
    const float inv = 1.f / l;
    const int tok = row / G;
    bf16x4 o4;
#pragma unroll
    for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(o[e] * inv);
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.out) + ((long long)(it.new_start + tok) * a.q_heads + g * G + (row - tok * G)) * D + d4 * 4) = o4;
}

template <int D, int RT, int NW, class Work>
void launch_one(const AttnLaunch& a, const Work& wk, int entries, hipStream_t s) {
    hipLaunchKernelGGL((kv8_attn_rows_kernel<D, RT, NW, Work>), dim3((unsigned)entries * a.kv_heads), dim3(64 * NW), 0, s, a, wk);
}
template <int D, class Work>
void launch_waves(const AttnLaunch& a, const Work& wk, int entries, int rows, int waves, hipStream_t s) {
    if (waves == 4) rows == kKv8Rows ? launch_one<D, 1, 4>(a, wk, entries, s) : launch_one<D, 2, 4>(a, wk, entries, s);
    else rows == kKv8Rows ? launch_one<D, 1, 8>(a, wk, entries, s) : launch_one<D, 2, 8>(a, wk, entries, s);
}
template <class Work>
void launch_list(const AttnLaunch& a, const Work& wk, int entries, int rows, int waves, hipStream_t s) {
    a.head_dim == 64 ? launch_waves<64>(a, wk, entries, rows, waves, s) : launch_waves<128>(a, wk, entries, rows, waves, s);
}
template <int D, int TR, class Work>
void merge_one(const AttnLaunch& a, const Work& wk, int items, int max_rows, hipStream_t s) {
    constexpr int SHARE = TR == kKv8TallRows ? 1 : TR == kKv8WideRows ? 4 : 8, RPW = 1024 / (D * SHARE);
    const int row_groups = ((max_rows < TR ? max_rows : TR) + RPW - 1) / RPW;
    hipLaunchKernelGGL((kv8_merge_kernel<D, TR, SHARE, Work>), dim3((unsigned)items * a.kv_heads * row_groups), dim3(256), 0, s, a, wk, row_groups);
}
template <class Work>
void merge_list(const AttnLaunch& a, const Work& wk, int items, int rows, int max_rows, hipStream_t s) {
    const bool d64 = a.head_dim == 64;
    if (rows == kKv8Rows) d64 ? merge_one<64, kKv8Rows>(a, wk, items, max_rows, s) : merge_one<128, kKv8Rows>(a, wk, items, max_rows, s);
    else if (rows == kKv8WideRows) d64 ? merge_one<64, kKv8WideRows>(a, wk, items, max_rows, s) : merge_one<128, kKv8WideRows>(a, wk, items, max_rows, s);
    else d64 ? merge_one<64, kKv8TallRows>(a, wk, items, max_rows, s) : merge_one<128, kKv8TallRows>(a, wk, items, max_rows, s);
}

}  // namespace

hipError_t launch_kv8_attn_rows(const AttnLaunch& a, const AttnWork& wk, int entries, int rows, int waves, hipStream_t s) {
    if (entries <= 0) return hipSuccess;
    wk.n_reqs <= kAttnReqStep ? launch_list(a, short_list(wk), entries, rows, waves, s) : launch_list(a, wk, entries, rows, waves, s);
    return hipGetLastError();
}

hipError_t launch_kv8_merge(const AttnLaunch& a, const AttnWork& wk, int items, int rows, int max_rows, hipStream_t s) {
    if (items <= 0) return hipSuccess;
    wk.n_reqs <= kAttnReqStep ? merge_list(a, short_list(wk), items, rows, max_rows, s) : merge_list(a, wk, items, rows, max_rows, s);
    return hipGetLastError();
}

}  // namespace ragc
