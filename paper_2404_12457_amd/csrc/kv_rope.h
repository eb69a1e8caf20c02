// Position rotation of packed rows (gfx950 device code of kv_rope.hip and kv8_append.hip).
//
// Pair i of a head turns by the angle of its row's position, angle row p of cos_sin = cos of the rot_dim/2 angles, then
// their sin:  (a, b) -> (a cos - b sin, a sin + b cos), in fp32 (one fma and one product of exact bf16 or fp32 factors: off by
// at most 2^-24 of each product), rounded once to the type.  The pairs are elements i and i + rot_dim/2, or 2i and 2i + 1;
// elements from rot_dim on stay.
//
// A thread owns one task of a head: two 16-byte chunks that hold both ends of its pairs, so that an array may be turned in
// place.  Task t of a head takes the angles from t * E on (E elements per chunk), whichever the pairs: chunks t and t + half as
// many as turn, or 2t and 2t + 1; behind the turned chunks tasks are two chunks in a row.  The task and its angles are the same for
// all heads of a row, so the angles are read once for HG heads.
#pragma once
#include "kv_rows.h"

namespace ragc {
namespace {

template <class T>
struct RopeTask {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef __attribute__((ext_vector_type(E))) T chunk;
    int c0, c1;  // the two chunks of the head
    bool turns;
    float cs[E], sn[E];

    __device__ __forceinline__ RopeTask(const RopeArgs& rope, int t, long long pos) {
        const int rc = rope.rot_dim / E, hc = rc / 2;
        turns = t < hc;
        c0 = turns ? (rope.interleaved ? 2 * t : t) : rc + 2 * (t - hc);
        c1 = turns && !rope.interleaved ? t + hc : c0 + 1;
        const float* const at = rope.cos_sin + pos * rope.rot_dim + (turns ? t * E : 0);
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const float4 c = *reinterpret_cast<const float4*>(at + i), s = *reinterpret_cast<const float4*>(at + rope.rot_dim / 2 + i);
            cs[i] = c.x, cs[i + 1] = c.y, cs[i + 2] = c.z, cs[i + 3] = c.w;
            sn[i] = s.x, sn[i + 1] = s.y, sn[i + 2] = s.z, sn[i + 3] = s.w;
        }
    }
    static __device__ __forceinline__ void pair(T& a, T& b, float c, float s) {
        const float x = (float)a, y = (float)b;
        a = (T)__builtin_fmaf(x, c, -(y * s));
        b = (T)__builtin_fmaf(x, s, y * c);
    }
    __device__ __forceinline__ void turn(chunk& a, chunk& b, bool interleaved) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            T x, y;
            if (interleaved) {
                const int f = 2 * e % E;
                x = 2 * e < E ? a[f] : b[f];
                y = 2 * e < E ? a[f + 1] : b[f + 1];
                pair(x, y, cs[e], sn[e]);
                if (2 * e < E) a[f] = x, a[f + 1] = y; else b[f] = x, b[f + 1] = y;
            } else {
                x = a[e];
                y = b[e];
                pair(x, y, cs[e], sn[e]);
                a[e] = x;
                b[e] = y;
            }
        }
    }
};

// One workgroup of 256 threads: HG heads, from number hg * HG on, of the 256 / (tasks per head) packed rows from row0 on.  Heads are
// numbered K first, then V, then Q; `kv` = 0 leaves K and V out.  All loads are under way before the first store.
template <class T, int HG>
__device__ __forceinline__ void rope_rows(const PagedBatch& b, const RopeArgs& rope, const RopeRows& x, int kv, int row0, int hg) {
    typedef typename RopeTask<T>::chunk chunk;
    const int D = b.head_dim;
    const int tasks_shift = __ffs(D * (int)sizeof(T) >> 5) - 1;
    const int first_row = b.new_start[0];
    const int mine = row0 + ((int)threadIdx.x >> tasks_shift);
    const int t = first_row + min(mine, x.total_new - 1);
    const RowAt at = locate_row(b, t);
    const int pos = at.prefix + (t - at.start);
    const RopeTask<T> task(rope, threadIdx.x & ((1 << tasks_shift) - 1), pos);
    const int heads = 2 * kv + x.q_heads, h0 = hg * HG;
    const T* const src_k = static_cast<const T*>(x.k_new) + (long long)t * kv * D;
    const T* const src_v = static_cast<const T*>(x.v_new) + (long long)t * kv * D;
    const T* const src_q = static_cast<const T*>(x.q) + (long long)t * x.q_heads * D;
    chunk a[HG], c[HG];
#pragma unroll
    for (int u = 0; u < HG; ++u) {
        const int h = min(h0 + u, heads - 1);
        const chunk* const p = reinterpret_cast<const chunk*>(h < kv ? src_k + h * D : h < 2 * kv ? src_v + (h - kv) * D : src_q + (h - 2 * kv) * D);
        a[u] = p[task.c0];
        c[u] = p[task.c1];
    }
    long long slot = 0;
    if (h0 < 2 * kv) {
        const int blk = b.block_table[(long long)at.req * b.table_stride + (pos >> 4)];
        slot = (long long)blk * b.block_stride + (long long)(pos & 15) * D;
    }
    if (mine >= x.total_new) return;
#pragma unroll
    for (int u = 0; u < HG; ++u) {
        const int h = h0 + u;
        if (h >= heads) return;
        const bool is_v = h >= kv && h < 2 * kv;
        if (task.turns && !is_v) task.turn(a[u], c[u], rope.interleaved);
        if (h < 2 * kv) {
            chunk* const p = reinterpret_cast<chunk*>(static_cast<T*>(is_v ? x.pool_v : x.pool_k) + slot + (long long)(is_v ? h - kv : h) * (kBlock * D));
            p[task.c0] = a[u];
            p[task.c1] = c[u];
        }
        T* const copy = static_cast<T*>(h >= 2 * kv ? x.q_out : x.k_out);
        if (!is_v && copy) {
            chunk* const p = reinterpret_cast<chunk*>(copy + ((long long)t * (h >= 2 * kv ? x.q_heads : kv) + (h >= 2 * kv ? h - 2 * kv : h)) * D);
            p[task.c0] = a[u];
            p[task.c1] = c[u];
        }
    }
}

}  // namespace
}  // namespace ragc
