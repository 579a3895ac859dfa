// Instantiates the attention of drafted tokens over a cache of 8 bits for element type __bf16.
#include "tree_attn8.hpp"

namespace depsync {
hipError_t launch_tree_attn8_bf16(const TreeAttn8Args& a, int head_dim, hipStream_t stream) {
    return launch_tree_attn8_type<__bf16>(a, head_dim, stream);
}
}  // namespace depsync
