// Kernel arguments and launchers of the cache operators (attention of drafted tokens, append, weights, eviction).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace depsync {

// Elements from one sequence, token and head to the next.
struct Strides { int64_t batch, token, head; };

struct TreeAttnArgs {
    const void *q, *k_new, *v_new, *k_cache, *v_cache;
    const int32_t *cached, *drafted;      // drafted may be null
    const uint64_t* tree;                 // may be null: token t sees 0..t
    void* out;
    float* lse;                           // may be null
    float* parts;                         // slots > batch: partial results (see tree_attn.hpp)
    Strides q_s, new_s, cache_s, out_s;
    int64_t tree_batch;
    uint32_t batch, tokens, heads, kv_heads, group, capacity;
    uint32_t rows;                        // tokens * group: query rows of one key and value head
    uint32_t few;                         // 1: the form for few rows
    uint32_t slots;                       // the most parts that all sequences' key axes are cut into (batch: none is cut)
    uint32_t part_slots, part_blocks;     // of a sequence where each has as many: its parts, blocks of keys in one
    uint32_t part_least;                  // blocks of keys in a part at least, where all share the slots
    float scale;                          // scores to base-2 exponents
};

struct CacheAppendArgs {
    const void *k_new, *v_new;
    void *k_cache, *v_cache;
    const int32_t* cached;
    int32_t* cached_out;
    const int32_t *accepted, *n_accepted, *start;
    float* weights;
    int32_t* pos;
    int32_t* n_out;                       // may be null
    Strides new_s, cache_s;
    uint32_t batch, tokens, kv_heads, capacity, n_max;
};

struct CacheWeightsArgs {
    const void *q, *k_cache;
    const float* lse;
    const int32_t *cached, *accepted, *n_accepted;
    float* weights;
    Strides q_s, cache_s;
    uint32_t batch, tokens, heads, kv_heads, group, capacity, n_max;
    uint32_t few;                         // 1: the form for few rows
    uint32_t n_parts, part_blocks;        // workgroups along the keys, and (few rows) blocks of 128 keys in each
    uint32_t keys;                        // (many rows) keys of a workgroup: 32, in eight waves, or 64, in four
    float scale;                          // scores to base-2 exponents
};

struct CacheEvictArgs {
    void *k_cache, *v_cache, *k_out, *v_out;       // (k_out = k_cache where the rows move in place)
    float *weights, *weights_out;
    int32_t *pos, *pos_out;
    const int32_t* cached;
    int32_t* cached_out;
    uint32_t* moves;                      // workspace: per sequence and head the number of moves, then their rows
    Strides cache_s, out_s;
    uint32_t batch, kv_heads, capacity, capacity_out, budget, recent, max_cached;
    uint32_t max_moves;
    uint32_t in_place;
    uint32_t fused, lanes;                // the rows move in the same launch; threads to a row
};

// The attention kernel's two forms: query rows of a workgroup and keys of a block.
constexpr uint32_t TREE_FEW_ROWS = 32, TREE_FEW_KEYS = 128, TREE_MANY_ROWS = 128, TREE_MANY_KEYS = 32;

hipError_t launch_tree_attn(const TreeAttnArgs& a, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_tree_attn_bf16(const TreeAttnArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_tree_attn_f16(const TreeAttnArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_cache_append(const CacheAppendArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_cache_weights(const CacheWeightsArgs& a, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_cache_evict(const CacheEvictArgs& a, int head_dim, hipStream_t stream);

template <class F, class A>
inline hipError_t launch_one(F* kernel, uint32_t n_blocks, uint32_t threads, hipStream_t stream, const A& a) {
    void* args[] = {const_cast<A*>(&a)};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(n_blocks), dim3(threads), args, 0, stream);
}

}  // namespace depsync
