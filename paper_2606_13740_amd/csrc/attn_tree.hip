// libdllm: the paged attention's kernels whose rows have masks.
#include <hip/hip_runtime.h>

#include "attn_launch.hpp"

namespace dllm {

void launch_attn_tree(int dtype, const PagedArgs& a, const AttnPlan& p, int Dh, hipStream_t s) {
    launch_attn<true>(dtype, a, p, Dh, s);
}

}  // namespace dllm
