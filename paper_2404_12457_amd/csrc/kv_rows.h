// Where a packed row of new tokens belongs (gfx950 device code, shared by the kernels that write the paged K/V store).
#pragma once
#include "ragc_internal.h"

namespace ragc {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Request that owns packed row t: largest r with new_start[r] <= t (new_start is
// increasing and new_start[0] <= t < new_start[num_reqs]).
__device__ __forceinline__ int find_request(const int32_t* __restrict__ new_start, int num_reqs, int t) {
    int lo = 0, hi = num_reqs;  // invariant: new_start[lo] <= t < new_start[hi]
    while (hi - lo > 1) {
        int mid = (lo + hi) >> 1;
        if (new_start[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

struct RowAt {
    int req, start, prefix;  // request, its first packed row and its cached length
};

// The request of row t, a row per lane; every lane of the wave takes part.  Up to 64 requests are searched among the lanes
// after one trip to memory, more in memory.
__device__ __forceinline__ RowAt locate_row(const PagedBatch& b, int t) {
    const int lane = threadIdx.x & 63;
    RowAt at;
    if (b.num_reqs <= 64) {  // one request per lane, then find_request among the lanes
        const int mine = min(lane, b.num_reqs - 1);
        const int starts = b.new_start[mine], prefixes = b.prefix_len[mine];
        at.req = 0;
#pragma unroll
        for (int step = 32; step > 0; step >>= 1) {
            const int s = __shfl(starts, at.req + step, 64);  // req + step <= 63
            if (at.req + step < b.num_reqs && s <= t) at.req += step;
        }
        at.start = __shfl(starts, at.req, 64);
        at.prefix = __shfl(prefixes, at.req, 64);
    } else {
        at.req = find_request(b.new_start, b.num_reqs, t);
        at.start = b.new_start[at.req];
        at.prefix = b.prefix_len[at.req];
    }
    return at;
}

}  // namespace
}  // namespace ragc
