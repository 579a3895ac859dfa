// Instantiates the attention of drafted tokens for element type __bf16.
#include "tree_attn.hpp"

namespace depsync {
hipError_t launch_tree_attn_bf16(const TreeAttnArgs& a, int head_dim, hipStream_t stream) {
    return launch_tree_attn_type<__bf16>(a, head_dim, stream);
}
}  // namespace depsync
