// Instantiates the attention of drafted tokens for element type _Float16.
#include "tree_attn.hpp"

namespace depsync {
hipError_t launch_tree_attn_f16(const TreeAttnArgs& a, int head_dim, hipStream_t stream) {
    return launch_tree_attn_type<_Float16>(a, head_dim, stream);
}
}  // namespace depsync
