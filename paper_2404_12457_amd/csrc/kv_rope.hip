// Append with the position rotation on the way: K of the new tokens is turned by the angles of its positions and stored with V
// in their paged slots, Q is turned by the same launch (paper Sec. 4: the tensors of the accessed documents are cached after the
// first token; cached keys have their positions in them).
//
// What bounds it: HBM on large calls (every row read once and written once), the trips to memory in a row on small ones (lengths, then
// the table and the angles' rows, with the sources under way).  Four heads per workgroup and row keep 128 bytes per thread in flight and
// share the angles.  16 requests of 7.4k tokens in all, 32/8 heads of 128 in bf16, Q turned too, 185 MB moved: 39.2 us, 4.7 TB/s
// (a large copy runs at 5.05 on the same card); a step of 64 requests, 64/8 heads, 5.3 us.
#include "kv_rope.h"

namespace ragc {
namespace {

template <class T, int HG>
__global__ __launch_bounds__(256) void append_rope_kernel(PagedBatch b, RopeArgs rope, RopeRows x, int rows, int head_groups) {
    // the head group varies fastest, so workgroups that run together cover whole source rows
    rope_rows<T, HG>(b, rope, x, b.kv_heads, blockIdx.x / head_groups * rows, blockIdx.x % head_groups);
}

template <class T, int HG>
hipError_t launch_one(const PagedBatch& b, const RopeArgs& rope, const RopeRows& x, hipStream_t s) {
    const int rows = 256 / (b.head_dim * (int)sizeof(T) / 32);
    const int head_groups = (2 * b.kv_heads + x.q_heads + HG - 1) / HG;
    const long long grid = (long long)((x.total_new + rows - 1) / rows) * head_groups;
    if (grid > 0xffffff) return hipErrorInvalidValue;  // grid times workgroup size stays below 2^32 threads
    hipLaunchKernelGGL((append_rope_kernel<T, HG>), dim3((unsigned)grid), dim3(256), 0, s, b, rope, x, rows, head_groups);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append_rope(const PagedBatch& b, const RopeArgs& rope, const RopeRows& x, int esize, hipStream_t s) {
    return esize == 2 ? launch_one<__bf16, 4>(b, rope, x, s) : launch_one<float, 4>(b, rope, x, s);
}

}  // namespace ragc
