// Attention of trees of drafted tokens over a paged cache: decode_wide.h's kernel
// with every row's own set of keys behind the context.
#include "decode_wide.h"

namespace mla {
namespace {

template <int KIND>
void launch_kind(const TreeArgs& a, hipStream_t stream) {
    const int64_t blocks = tree_workgroups(a.num_work, static_cast<int64_t>(a.s_q) * a.H, a.shape.rows);
    const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
    if (a.shape.rows == rows_per_block(2)) hipLaunchKernelGGL((decode_kernel<KIND, false, 2, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((decode_kernel<KIND, false, 1, true>), grid, block, 0, stream, a);
}

}  // namespace

hipError_t launch_tree_attn(CacheKind kind, const TreeArgs& a, hipStream_t stream) {
    if (a.num_work == 0) return hipSuccess;
    if (a.shape.waves != kWaves || (a.shape.rows != rows_per_block(1) && a.shape.rows != rows_per_block(2)))
        return hipErrorInvalidValue;
    switch (kind) {
        case KIND_C4R4: launch_kind<KIND_C4R4>(a, stream); break;
        case KIND_C2R4: launch_kind<KIND_C2R4>(a, stream); break;
        case KIND_C4R4P: launch_kind<KIND_C4R4P>(a, stream); break;
        case KIND_C2R4P: launch_kind<KIND_C2R4P>(a, stream); break;
        case KIND_BF16: launch_kind<KIND_BF16>(a, stream); break;
    }
    return hipGetLastError();
}

}  // namespace mla
