// C-ABI layer of the cache operators (declarations in include/depsync.h): checks of arguments, division of the work.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/depsync.h"
#include "cache_ops.h"
#include "launch.h"

using namespace depsync;

namespace {

constexpr int64_t MAX_TOKEN_STRIDE = 1 << 24;     // 64 rows of a cache, as far as a workgroup reaches from one base, stay below 2 GiB
constexpr int64_t MAX_BLOCKS = 1 << 23;           // workgroups of a launch (HIP counts threads in 32 bits)

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool operand(const void* p) { return p && aligned(p, 16); }
bool array(const void* p) { return p && aligned(p, 4); }
bool optional(const void* p) { return aligned(p, 4); }
int64_t cdiv64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Strides of [batch][token][head][head_dim].  Those of dimensions of size one are not read: kernels get what a dense row has.
// Where rows are written, or read by the bounds of a run of rows, they must not overlap.
bool strides(Strides& s, int64_t batch, int64_t token, int64_t head, int64_t n_batch, int64_t n_token, int64_t n_head, int dim, bool written, bool run) {
    s = {n_batch > 1 ? batch : dim, n_token > 1 ? token : dim, n_head > 1 ? head : dim};
    for (int64_t x : {s.batch, s.token, s.head})
        if (x < 0 || x % 8 != 0 || x > (int64_t)1 << 40 || (written && x < dim)) return false;
    return !run || (s.token >= dim && s.token <= MAX_TOKEN_STRIDE);
}

// What the descriptors share.  head_dim and element types this build does not have: DEPSYNC_ENOTIMPL.
int common(int batch, int tokens, int heads, int kv_heads, int head_dim, int dtype, int capacity) {
    if (batch < 1 || batch > 1 << 20 || tokens < 1 || tokens > 65536 || kv_heads < 1 || heads < kv_heads || heads > 65536 || heads % kv_heads != 0 ||
        capacity < 0 || capacity > 1 << 30 || head_dim < 1 || (dtype != DEPSYNC_BF16 && dtype != DEPSYNC_FP16))
        return DEPSYNC_EINVAL;
    return head_dim == 64 || head_dim == 128 ? DEPSYNC_OK : DEPSYNC_ENOTIMPL;
}

bool base2_scale(float given, int head_dim, float& out) {
    if (!std::isfinite(given) || given < 0.0f) return false;
    out = (given == 0.0f ? 1.0f / std::sqrt((float)head_dim) : given) * 1.4426950408889634f;
    return true;
}

int rows_hint(int max_cached, int capacity) { return max_cached == 0 ? capacity : std::min(max_cached, capacity); }

int cu_count(int& n_cu) {
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return hip_fail(e);
    const hipError_t e = hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, dev);
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

int tree_check(const depsync_tree_attn_desc* d) {
    if (!d) return DEPSYNC_EINVAL;
    if (int rc = common(d->batch, d->tokens, d->heads, d->kv_heads, d->head_dim, d->dtype, d->capacity); rc != DEPSYNC_OK) return rc;
    return d->max_cached < 0 ? DEPSYNC_EINVAL : DEPSYNC_OK;
}

// How the key axis of dep_tree_attn is cut: few (sequence, head) pairs and row blocks leave CUs idle unless it is, but parts leave results of
// 4 (head_dim + 2) bytes a row in memory, which a second kernel reads.  The model, in microseconds, fitted to times of 27 shapes under
// up to 28 cuts each (1 to 2048 rows, caches of 0 to 120000; its choice is 4 % behind the best cut in the mean, in the worst case 21 %):
// a workgroup's start, a block of keys where its workgroup is alone on the CU and where two share it, the keys' way from HBM, the
// second kernel and the results' way there and back.  5.9 is what a second launch costs a program that waits for the host (one token of 12 heads over 500
// rows 12.4 us in one launch, 15.5 in two); captured into a graph it is about 4 (12.1 and 11.6).  The lengths are the longest sequence's; the
// kernels then share out the parts by the real ones.
double tree_cost(int64_t base, int64_t part, int64_t blocks, int64_t pairs, int64_t rows, int64_t row_blocks, int head_dim, int n_cu, bool few) {
    const int64_t parts = cdiv64(blocks, part), groups = base * parts, slots = 2 * (int64_t)n_cu;
    const double at_once = (double)std::min(groups, slots), wide = head_dim / 128.0;
    const double step = few ? 0.13 + 1.32 * wide : (at_once > n_cu ? 1.0 : at_once > n_cu / 2 ? 0.8 : 0.55) * (0.3 + 0.7 * wide);
    const double hbm = at_once / row_blocks * (few ? TREE_FEW_KEYS : TREE_MANY_KEYS) * 4.0 * head_dim / 5.2e6;
    const double join = parts > 1 ? 5.9 + (double)parts * pairs * rows * (head_dim + 2) * 8.0 / 4e6 : 0.0;
    return (double)cdiv64(groups, slots) * (3.0 + part * std::cbrt(step * step * step + hbm * hbm * hbm)) + join;   // (between the larger and the sum)
}

int tree_plan(const depsync_tree_attn_desc* d, int n_cu, TreeAttnArgs& a, size_t& bytes) {
    if (n_cu <= 0)
        if (int rc = cu_count(n_cu); rc != DEPSYNC_OK) return rc;
    a.batch = d->batch; a.tokens = d->tokens; a.heads = d->heads; a.kv_heads = d->kv_heads; a.capacity = d->capacity;
    a.group = d->heads / d->kv_heads;
    const int64_t rows = (int64_t)d->tokens * a.group;
    if (rows > 1 << 24) return DEPSYNC_ENOTIMPL;
    a.rows = (uint32_t)rows;
    // From 33 to 64 rows two workgroups of 32 walk the same keys, the second from L2; that is ahead of one of 128 rows until the caches are larger than
    // what L2 and the Infinity Cache keep between the two.  Inputs that change from call to call, us for 32 and for 128 rows: 16 x 40 rows over 1000 keys of 8
    // heads, 66 MB, 21 and 30; 32 x 40 over 1000, 131 MB, 38 and 35; 64 x 64 over 1000, 262 MB, 73 and 63; 64 x 40 over 4000, 1 GB, 223 and 201; 52 rows of one
    // head of 64 over 120000, 73 and 62.  Between 100 and 270 MB it depends on how many sequences share them: 8 x 48 over 8000 67 and 64, but 16 x 64
    // over 4000 64 and 68, 4 x 52 over 8000 40 and 42, 16 x 40 over 2000 36 and 49.
    const int64_t cache_bytes = (int64_t)d->batch * d->kv_heads * rows_hint(d->max_cached, d->capacity) * d->head_dim * 4;
    a.few = rows <= (cache_bytes < 100000000 ? 64 : 32);
    const int64_t keys = a.few ? TREE_FEW_KEYS : TREE_MANY_KEYS, row_blocks = cdiv64(rows, a.few ? TREE_FEW_ROWS : TREE_MANY_ROWS);
    const int64_t pairs = (int64_t)d->batch * d->kv_heads, base = pairs * row_blocks;
    const int64_t blocks = cdiv64(rows_hint(d->max_cached, d->capacity), keys) + cdiv64(d->tokens, keys);
    int64_t part = blocks;
    double best = tree_cost(base, part, blocks, pairs, rows, row_blocks, d->head_dim, n_cu, a.few);
    for (int64_t rounds = 1; rounds <= 4; ++rounds) {             // parts that fill the chip a whole number of times
        const int64_t parts = std::min(blocks, std::max<int64_t>(1, rounds * 2 * n_cu / base)), p = cdiv64(blocks, parts);
        const double t = tree_cost(base, p, blocks, pairs, rows, row_blocks, d->head_dim, n_cu, a.few);
        if (t < best) { best = t; part = p; }
        if (p + 1 > blocks) continue;
        for (int64_t q : {2 * p, 4 * p}) {                         // or fewer, where their results cost more
            const double u = tree_cost(base, std::min(q, blocks), blocks, pairs, rows, row_blocks, d->head_dim, n_cu, a.few);
            if (u < best) { best = u; part = std::min(q, blocks); }
        }
    }
    // (the kernels add up all sequences' blocks in 32 bits)
    const int64_t parts = d->batch * (cdiv64(d->capacity, keys) + cdiv64(d->tokens, keys)) < 1ll << 32 ? cdiv64(blocks, part) : 1;
    if (cdiv64(pairs * parts, 8) * 8 * row_blocks > MAX_BLOCKS || cdiv64(pairs * rows, 4) > MAX_BLOCKS) return DEPSYNC_ENOTIMPL;
    a.slots = (uint32_t)(d->batch * parts);
    a.part_slots = (uint32_t)parts;
    a.part_blocks = (uint32_t)part;
    a.part_least = (uint32_t)std::min<int64_t>(part, a.few ? 1 : 4);
    bytes = parts > 1 ? (size_t)pairs * parts * rows * (d->head_dim + 2) * sizeof(float) : 0;
    return DEPSYNC_OK;
}

int64_t evict_moves(const depsync_cache_evict_desc* d) {
    return d->k_out ? d->budget : std::max(0, std::min(d->budget, d->capacity - d->budget));
}

int evict_check(const depsync_cache_evict_desc* d) {
    if (!d) return DEPSYNC_EINVAL;
    if (int rc = common(d->batch, 1, d->kv_heads, d->kv_heads, d->head_dim, d->dtype, d->capacity); rc != DEPSYNC_OK) return rc;
    if (d->capacity < 1 || d->max_cached < 0 || d->budget < 1 || d->recent < 0 || d->recent > d->budget) return DEPSYNC_EINVAL;
    return (int64_t)d->batch * d->kv_heads > MAX_BLOCKS / 4 ? DEPSYNC_ENOTIMPL : DEPSYNC_OK;   // (1024 threads each)
}

}  // namespace

extern "C" {

int depsync_tree_attn_workspace(const depsync_tree_attn_desc* d, int n_cu, size_t* bytes) {
    if (!bytes) return DEPSYNC_EINVAL;
    if (int rc = tree_check(d); rc != DEPSYNC_OK) return rc;
    TreeAttnArgs a = {};
    return tree_plan(d, n_cu, a, *bytes);
}

int dep_tree_attn(const depsync_tree_attn_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = tree_check(d); rc != DEPSYNC_OK) return rc;
    TreeAttnArgs a = {};
    size_t need = 0;
    const int D = d->head_dim;
    if (!operand(d->q) || !operand(d->k_new) || !operand(d->v_new) || !operand(d->out) || !optional(d->drafted) || !optional(d->lse) ||
        (d->capacity > 0 && (!operand(d->k_cache) || !operand(d->v_cache) || !array(d->cached))) || !aligned(d->tree, 8))
        return DEPSYNC_EINVAL;
    if (!strides(a.q_s, d->q_batch, d->q_token, d->q_head, d->batch, d->tokens, d->heads, D, false, false) ||
        !strides(a.new_s, d->new_batch, d->new_token, d->new_head, d->batch, d->tokens, d->kv_heads, D, false, true) ||
        !strides(a.out_s, d->out_batch, d->out_token, d->out_head, d->batch, d->tokens, d->heads, D, true, false))
        return DEPSYNC_EINVAL;
    if (d->capacity > 0 && !strides(a.cache_s, d->cache_batch, d->cache_token, d->cache_head, d->batch, d->capacity, d->kv_heads, D, false, true))
        return DEPSYNC_EINVAL;
    if (d->tree && d->tree_batch != 0 && d->tree_batch < (int64_t)d->tokens * cdiv64(d->tokens, 64)) return DEPSYNC_EINVAL;
    if (!base2_scale(d->scale, D, a.scale)) return DEPSYNC_EINVAL;
    if (int rc = tree_plan(d, 0, a, need); rc != DEPSYNC_OK) return rc;
    if (need > 0 && (!operand(workspace) || workspace_bytes < need)) return DEPSYNC_EINVAL;
    a.q = d->q; a.k_new = d->k_new; a.v_new = d->v_new; a.k_cache = d->k_cache; a.v_cache = d->v_cache;
    a.cached = d->cached; a.drafted = d->drafted; a.tree = d->tree; a.tree_batch = d->tree_batch;
    a.out = d->out; a.lse = d->lse; a.parts = static_cast<float*>(workspace);
    const hipError_t e = launch_tree_attn(a, d->dtype, D, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

int dep_cache_append(const depsync_cache_append_desc* d, void* stream) {
    if (!d) return DEPSYNC_EINVAL;
    if (int rc = common(d->batch, d->tokens, d->kv_heads, d->kv_heads, d->head_dim, d->dtype, d->capacity); rc != DEPSYNC_OK) return rc;
    CacheAppendArgs a = {};
    const int D = d->head_dim;
    if (d->capacity < 1 || d->n_max < 1 || d->n_max > 65536 || (!d->accepted && d->n_max > d->tokens)) return DEPSYNC_EINVAL;
    if (!operand(d->k_new) || !operand(d->v_new) || !operand(d->k_cache) || !operand(d->v_cache) || !array(d->cached) || !array(d->cached_out) ||
        d->cached == d->cached_out || !optional(d->accepted) || !optional(d->n_accepted) || !optional(d->weights) || !optional(d->pos) ||
        (d->pos && !array(d->start)) || !optional(d->n_out))
        return DEPSYNC_EINVAL;
    if (d->n_out && (d->n_out == d->cached || d->n_out == d->cached_out || d->n_out == d->n_accepted)) return DEPSYNC_EINVAL;
    if (!strides(a.new_s, d->new_batch, d->new_token, d->new_head, d->batch, d->tokens, d->kv_heads, D, false, false) ||
        !strides(a.cache_s, d->cache_batch, d->cache_token, d->cache_head, d->batch, d->capacity, d->kv_heads, D, true, true))
        return DEPSYNC_EINVAL;
    const int64_t rows = 256 / (D / 8);
    if (d->batch * cdiv64((int64_t)d->n_max * d->kv_heads, rows) > MAX_BLOCKS) return DEPSYNC_ENOTIMPL;
    a.k_new = d->k_new; a.v_new = d->v_new; a.k_cache = d->k_cache; a.v_cache = d->v_cache;
    a.cached = d->cached; a.cached_out = d->cached_out; a.accepted = d->accepted; a.n_accepted = d->n_accepted;
    a.weights = d->weights; a.pos = d->pos; a.start = d->start; a.n_out = d->n_out;
    a.batch = d->batch; a.tokens = d->tokens; a.kv_heads = d->kv_heads; a.capacity = d->capacity; a.n_max = d->n_max;
    const hipError_t e = launch_cache_append(a, D, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

int dep_cache_weights(const depsync_cache_weights_desc* d, void* stream) {
    if (!d) return DEPSYNC_EINVAL;
    if (int rc = common(d->batch, d->tokens, d->heads, d->kv_heads, d->head_dim, d->dtype, d->capacity); rc != DEPSYNC_OK) return rc;
    CacheWeightsArgs a = {};
    const int D = d->head_dim;
    if (d->capacity < 1 || d->max_cached < 0 || d->n_max < 1 || d->n_max > 65536 || (!d->accepted && d->n_max > d->tokens)) return DEPSYNC_EINVAL;
    if (!operand(d->q) || !array(d->lse) || !operand(d->k_cache) || !array(d->cached) || !optional(d->accepted) || !optional(d->n_accepted) || !array(d->weights))
        return DEPSYNC_EINVAL;
    if (!strides(a.q_s, d->q_batch, d->q_token, d->q_head, d->batch, d->tokens, d->heads, D, false, true) ||
        !strides(a.cache_s, d->cache_batch, d->cache_token, d->cache_head, d->batch, d->capacity, d->kv_heads, D, false, true))
        return DEPSYNC_EINVAL;
    if (!base2_scale(d->scale, D, a.scale)) return DEPSYNC_EINVAL;
    a.q = d->q; a.lse = d->lse; a.k_cache = d->k_cache; a.cached = d->cached; a.accepted = d->accepted; a.n_accepted = d->n_accepted; a.weights = d->weights;
    a.batch = d->batch; a.tokens = d->tokens; a.heads = d->heads; a.kv_heads = d->kv_heads; a.group = d->heads / d->kv_heads; a.capacity = d->capacity; a.n_max = d->n_max;
    const int64_t keys = rows_hint(d->max_cached, d->capacity), pairs = (int64_t)d->batch * d->kv_heads;
    if ((int64_t)d->n_max * a.group > 1 << 24 || pairs * cdiv64(keys, 32) > MAX_BLOCKS) return DEPSYNC_ENOTIMPL;
    a.few = (int64_t)d->n_max * a.group <= 64;       // (what LDS keeps beside the keys on their way)
    int n_cu = 0;
    if (int rc = cu_count(n_cu); rc != DEPSYNC_OK) return rc;
    if (a.few) {
        // Three workgroups share a CU.  Where each would have 8 blocks or more, twice as many even out sequences of different lengths (8 of 500 to
        // 20000 rows: 36 and 30 us, 2 of 20000 and 39000: 35 and 33); with fewer they cost more than that (4 of 4000 to 8000, 3 blocks: 12.7 and 13.7).
        const int64_t blocks = cdiv64(keys, 128) * pairs, share = cdiv64(blocks, 3 * (int64_t)n_cu);
        a.part_blocks = (uint32_t)std::max<int64_t>(1, share < 8 ? share : cdiv64(blocks, 6 * (int64_t)n_cu));
        a.n_parts = (uint32_t)cdiv64(cdiv64(keys, 128), a.part_blocks);
    } else {
        // 64 keys to a workgroup read the queries half as often as 32 (4 x 1500 tokens of 32 heads: 69 us, 88 with 32), but the first keys' have all rows to
        // walk and the last ones' few: where workgroups are not many, twice as many of twice the waves even that out (2048 tokens of 12 heads: 21 us with 64
        // and 18 with 32; of 32 heads on 4: 133 and 69).  3 x 1500 tokens of 12 heads, 864 workgroups of 64: 27 us, 30 with 32.
        a.keys = pairs * cdiv64(keys, 64) < 2 * (int64_t)n_cu ? 32 : 64;
        a.n_parts = (uint32_t)cdiv64(keys, a.keys);
    }
    const hipError_t e = launch_cache_weights(a, d->dtype, D, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

int depsync_cache_evict_workspace(const depsync_cache_evict_desc* d, size_t* bytes) {
    if (!bytes) return DEPSYNC_EINVAL;
    if (int rc = evict_check(d); rc != DEPSYNC_OK) return rc;
    *bytes = (size_t)d->batch * d->kv_heads * (1 + 2 * (size_t)evict_moves(d)) * sizeof(uint32_t);
    return DEPSYNC_OK;
}

int dep_cache_evict(const depsync_cache_evict_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    if (int rc = depsync_cache_evict_workspace(d, &need); rc != DEPSYNC_OK) return rc;
    CacheEvictArgs a = {};
    const int D = d->head_dim;
    const bool other = d->k_out != nullptr;
    if (!operand(d->k_cache) || !operand(d->v_cache) || !array(d->weights) || !array(d->pos) || !array(d->cached) || !array(d->cached_out) ||
        d->cached == d->cached_out || !operand(workspace) || workspace_bytes < need)
        return DEPSYNC_EINVAL;
    if ((d->v_out != nullptr) != other || (d->weights_out != nullptr) != other || (d->pos_out != nullptr) != other) return DEPSYNC_EINVAL;
    if (!strides(a.cache_s, d->cache_batch, d->cache_token, d->cache_head, d->batch, d->capacity, d->kv_heads, D, !other, true)) return DEPSYNC_EINVAL;
    if (other) {
        if (!operand(d->k_out) || !operand(d->v_out) || !array(d->weights_out) || !array(d->pos_out) || d->capacity_out < d->budget || d->capacity_out > 1 << 30 ||
            d->k_out == d->k_cache || d->v_out == d->v_cache || d->weights_out == d->weights || d->pos_out == d->pos ||
            !strides(a.out_s, d->out_batch, d->out_token, d->out_head, d->batch, d->capacity_out, d->kv_heads, D, true, true))
            return DEPSYNC_EINVAL;
    } else {
        a.out_s = a.cache_s;
    }
    a.k_cache = d->k_cache; a.v_cache = d->v_cache; a.weights = d->weights; a.pos = d->pos;
    a.k_out = other ? d->k_out : d->k_cache; a.v_out = other ? d->v_out : d->v_cache;
    a.weights_out = other ? d->weights_out : d->weights; a.pos_out = other ? d->pos_out : d->pos;
    a.cached = d->cached; a.cached_out = d->cached_out; a.moves = static_cast<uint32_t*>(workspace);
    a.batch = d->batch; a.kv_heads = d->kv_heads; a.capacity = d->capacity; a.capacity_out = other ? d->capacity_out : d->capacity;
    a.budget = d->budget; a.recent = d->recent; a.max_cached = rows_hint(d->max_cached, d->capacity);
    a.max_moves = (uint32_t)evict_moves(d);
    a.in_place = other ? 0 : 1;
    const hipError_t e = launch_cache_evict(a, D, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

}  // extern "C"
