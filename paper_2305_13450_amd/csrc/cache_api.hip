// C-ABI layer of the cache operators (declarations in include/depsync.h): checks of arguments, division of the work.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "../../include/depsync.h"
#include "cache_ops.h"
#include "launch.h"

using namespace depsync;

namespace {

constexpr int64_t MAX_TOKEN_STRIDE = 1 << 24;     // 64 rows of a cache, as far as a workgroup reaches from one base, stay below 2 GiB
constexpr int64_t L2_BYTES = 32 << 20;            // of the eight XCDs together
constexpr int64_t MAX_BLOCKS = 1 << 23;           // workgroups of a launch (HIP counts threads in 32 bits)

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool operand(const void* p) { return p && aligned(p, 16); }
bool array(const void* p) { return p && aligned(p, 4); }
bool optional(const void* p) { return aligned(p, 4); }
// Arrays that a call writes are neither one another nor any that it reads (some workgroups read while others write).
bool apart(std::initializer_list<const void*> written, std::initializer_list<const void*> read) {
    for (auto w = written.begin(); w != written.end(); ++w)
        if (*w && (std::count(written.begin(), w, *w) || std::count(read.begin(), read.end(), *w))) return false;
    return true;
}
int64_t cdiv64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Strides of [batch][token][head][head_dim].  Those of dimensions of size one are not read: kernels get what a dense row has.
// Where rows are written, or read by the bounds of a run of rows, they must not overlap.
bool strides(Strides& s, int64_t batch, int64_t token, int64_t head, int64_t n_batch, int64_t n_token, int64_t n_head, int dim, bool written, bool run, int multiple = 8) {
    s = {n_batch > 1 ? batch : dim, n_token > 1 ? token : dim, n_head > 1 ? head : dim};
    for (int64_t x : {s.batch, s.token, s.head})
        if (x < 0 || x % multiple != 0 || x > (int64_t)1 << 40 || (written && x < dim)) return false;
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
    static std::atomic<int> known[64];               // of a device, once asked for (0: not yet)
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return hip_fail(e);
    if (dev >= 0 && dev < 64 && (n_cu = known[dev].load(std::memory_order_relaxed)) > 0) return DEPSYNC_OK;
    const hipError_t e = hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, dev);
    if (e != hipSuccess) return hip_fail(e);
    if (dev >= 0 && dev < 64) known[dev].store(n_cu, std::memory_order_relaxed);
    return DEPSYNC_OK;
}

int tree_check(const depsync_tree_attn_desc* d) {
    if (!d) return DEPSYNC_EINVAL;
    if (int rc = common(d->batch, d->tokens, d->heads, d->kv_heads, d->head_dim, d->dtype, d->capacity); rc != DEPSYNC_OK) return rc;
    return d->max_cached < 0 ? DEPSYNC_EINVAL : DEPSYNC_OK;
}

// Checks the operands and fills in what does not depend on the division of the work.  multiple: of the cache's strides.
int tree_operands(const depsync_tree_attn_desc* d, TreeAttnArgs& a, int multiple) {
    const int D = d->head_dim;
    if (!operand(d->q) || !operand(d->k_new) || !operand(d->v_new) || !operand(d->out) || !optional(d->drafted) || !optional(d->lse) ||
        (d->capacity > 0 && (!operand(d->k_cache) || !operand(d->v_cache) || !array(d->cached))) || !aligned(d->tree, 8))
        return DEPSYNC_EINVAL;
    if (!strides(a.q_s, d->q_batch, d->q_token, d->q_head, d->batch, d->tokens, d->heads, D, false, false) ||
        !strides(a.new_s, d->new_batch, d->new_token, d->new_head, d->batch, d->tokens, d->kv_heads, D, false, true) ||
        !strides(a.out_s, d->out_batch, d->out_token, d->out_head, d->batch, d->tokens, d->heads, D, true, false))
        return DEPSYNC_EINVAL;
    if (d->capacity > 0 && !strides(a.cache_s, d->cache_batch, d->cache_token, d->cache_head, d->batch, d->capacity, d->kv_heads, D, false, true, multiple))
        return DEPSYNC_EINVAL;
    if (d->tree && d->tree_batch != 0 && d->tree_batch < (int64_t)d->tokens * cdiv64(d->tokens, 64)) return DEPSYNC_EINVAL;
    if (!base2_scale(d->scale, D, a.scale)) return DEPSYNC_EINVAL;
    a.q = d->q; a.k_new = d->k_new; a.v_new = d->v_new; a.k_cache = d->k_cache; a.v_cache = d->v_cache;
    a.cached = d->cached; a.drafted = d->drafted; a.tree = d->tree; a.tree_batch = d->tree_batch;
    a.out = d->out; a.lse = d->lse;
    return DEPSYNC_OK;
}

// How the key axis of dep_tree_attn is cut: few (sequence, head) pairs and row blocks leave CUs idle unless it is, but parts leave results of
// 4 (head_dim + 2) bytes a row in memory, which a second kernel reads.  The model, in microseconds, fitted to times of 27 shapes under
// up to 28 cuts each (1 to 2048 rows, caches of 0 to 120000; its choice is 4 % behind the best cut in the mean, in the worst case 21 %):
// a workgroup's start, a block of keys where its workgroup is alone on the CU and where two share it, the keys' way from HBM, the
// second kernel and the results' way there and back.  5.9 is what a second launch costs a program that waits for the host (one token of 12 heads over 500
// rows 12.4 us in one launch, 15.5 in two); captured into a graph it is about 4 (12.1 and 11.6).  The lengths are the longest sequence's; the
// kernels then share out the parts by the real ones.
// Over a cache of 8 bits the form for few rows has constants of its own, fitted to 46 shapes of 1 to 64 rows and both head sizes: a block takes 0.75 us for up to 16 rows of 128 and
// 1.3 for 32 (0.62 and 1.0 with 64) while its workgroup is alone on a CU, 1.4 times as long where two share it, or what HBM lets through, a quarter less to two. Several
// sequences count as three quarters of the longest: parts divide the real lengths between them, so cutting evens them out, and uncut ones leave HBM to the longest in the end (12 sequences of 1000 to
// 4000 rows, 25 query rows: 46 us uncut, as taking all for the longest has it, and 35; 8 of 500 to 4096, 64 rows: 30 and 26). The cut taken is on average 2.7 % behind the best, 4.3 % without that.
// The form for many rows (28 shapes): a block as below, never HBM; 0.5 % behind the best cut, 3 % with the constants over 16 bits (8 sequences of 2300 rows, 252 query rows: 66 us uncut, and 48).
double tree_cost(int64_t base, int64_t part, int64_t blocks, int64_t pairs, int64_t rows, int64_t row_blocks, int head_dim, int n_cu, bool few, bool held, int64_t batch) {
    const int64_t parts = cdiv64(blocks, part), groups = base * parts, slots = 2 * (int64_t)n_cu;
    const double at_once = (double)std::min(groups, slots), wide = head_dim / 128.0;
    double step = few ? 0.13 + 1.32 * wide : (at_once > n_cu ? 1.0 : at_once > n_cu / 2 ? 0.8 : 0.55) * (0.3 + 0.7 * wide);
    double rate = 5.2e6, start = 5.9, results = 4e6;               // of a cached row's 4 bytes a dimension; of a second launch, and of what it reads
    double mean = 1.0, late = 1.0;                                 // of the longest sequence: what a part has, and what HBM has to bring while that is walked
    if (few && held) {
        step = (0.25 + 0.25 * wide + (rows <= 16 ? 0.25 : 0.4) * (1.0 + wide)) * (at_once > n_cu ? 1.4 : 1.0);
        rate = at_once > n_cu ? 9.8e6 : 13e6;
        start = 5.5;
        if (batch > 1) (parts > 1 ? mean : late) = 0.75;
    } else if (held) {
        step = (at_once > n_cu ? 1.07 : at_once > n_cu / 2 ? 0.82 : 0.76) * (0.5 + 0.5 * wide);
        late = 0.0;
        start = 8.0;
        results = 6e6;
    }
    const double hbm = at_once / row_blocks * (few ? TREE_FEW_KEYS : TREE_MANY_KEYS) * 4.0 * head_dim / rate * late;
    const double join = parts > 1 ? start + (double)parts * pairs * rows * (head_dim + 2) * 8.0 / results : 0.0;
    return (double)cdiv64(groups, slots) * (3.0 + mean * part * std::cbrt(step * step * step + hbm * hbm * hbm)) + join;   // (between the larger and the sum)
}

int tree_plan(const depsync_tree_attn_desc* d, int n_cu, TreeAttnArgs& a, size_t& bytes, int held = 0) {   // held: rows of a block of a cache of 8 bits
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
    // Over a cache of 8 bits the form for few rows is ahead up to 64 rows at all sizes but one of 30 measured: its tiles are converted in each of two workgroups of 32 rows, but in
    // step with what HBM brings, and those of one of 128 rows behind barriers.  In us: 64 x 64 rows over 4000 keys of 8 heads, 524 MB, 147 and 169 us; 32 x 64 over 4000,
    // 262 MB, 76 and 96; 64 x 40 over 1000, 131 MB, 51 and 54; 52 rows of 8 heads of 64 over 120001 51 and 62; 16 x 33 over 2000 27 and 38; many short sequences last: 128 x 48 over
    // 500 67 and 71, 256 x 64 over 300 (4 heads) 57 and 54.
    const int64_t cache_bytes = (int64_t)d->batch * d->kv_heads * rows_hint(d->max_cached, d->capacity) * d->head_dim * 4;
    a.few = rows <= (held || cache_bytes < 100000000 ? 64 : 32);
    const int64_t keys = a.few ? TREE_FEW_KEYS : TREE_MANY_KEYS, row_blocks = cdiv64(rows, a.few ? TREE_FEW_ROWS : TREE_MANY_ROWS);
    const int64_t pairs = (int64_t)d->batch * d->kv_heads, base = pairs * row_blocks;
    const int64_t wide = d->tokens + held;                         // rows of 16 bits behind those of full blocks (and room up to a tile)
    const int64_t blocks = cdiv64(rows_hint(d->max_cached, d->capacity), keys) + cdiv64(wide, keys);
    int64_t part = blocks;
    double best = tree_cost(base, part, blocks, pairs, rows, row_blocks, d->head_dim, n_cu, a.few, held != 0, d->batch);
    for (int64_t rounds = 1, before = 0, p; rounds <= 4; ++rounds, before = p) {   // parts that fill the chip a whole number of times
        const int64_t parts = std::min(blocks, std::max<int64_t>(1, rounds * 2 * n_cu / base));
        p = cdiv64(blocks, parts);
        if (p == before) continue;
        const double t = tree_cost(base, p, blocks, pairs, rows, row_blocks, d->head_dim, n_cu, a.few, held != 0, d->batch);
        if (t < best) { best = t; part = p; }
        if (p + 1 > blocks) continue;
        for (int64_t q : {2 * p, 4 * p}) {                         // or fewer, where their results cost more
            const double u = tree_cost(base, std::min(q, blocks), blocks, pairs, rows, row_blocks, d->head_dim, n_cu, a.few, held != 0, d->batch);
            if (u < best) { best = u; part = std::min(q, blocks); }
        }
    }
    // (the kernels add up all sequences' blocks in 32 bits)
    const int64_t parts = d->batch * (cdiv64(d->capacity, keys) + cdiv64(wide, keys)) < 1ll << 32 ? cdiv64(blocks, part) : 1;
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

bool cache8_block(int block, int capacity) { return (block == 32 || block == 64 || block == 128) && capacity >= block && capacity % block == 0; }

// The children refused at one node are listed in LDS, so tokens are limited to what a draft may have.
int verify_check(const depsync_verify_drafts_desc* d) {
    if (!d || d->batch < 1 || d->batch > 1 << 20 || d->tokens < 1 || d->tokens > 65536 || d->vocab < 1 || d->vocab > 1 << 24) return DEPSYNC_EINVAL;
    return d->tokens > (int32_t)VERIFY_TOKENS ? DEPSYNC_ENOTIMPL : DEPSYNC_OK;
}

// How dep_verify_drafts spreads its rows.  One workgroup to a sequence has some 32 KB of reads on their way, 30 to 80 GB/s (32 chains of 6 over 50257 tokens: 43 us, 18 with
// rows over 32 workgroups each; 16 trees of 32 over 32000 without draft probabilities: 17.6 and 16.3, each before the sums went by DPP); below 16384 numbers a second launch
// costs what it saves.
// A tree whose tokens were drawn needs a pass over a row for each refusal that another child follows: so many launches go on where the one before stopped, and
// the last does the rest itself, 25 us a pass over 128000 numbers.  A launch that finds everything done costs 2.7.  Trees of 64 tokens, 8 at a time, need 3 to 6 passes mostly and 11 at
// times: 162 us without further launches, and on average over their inputs 58 with four, 38 with six, 41 with nine (one tree of 16: 24, 28 and 36).
void verify_plan(const depsync_verify_drafts_desc* d, VerifyArgs& a, size_t& bytes) {
    a.launches = 0;
    a.pieces = (uint32_t)std::min<int64_t>(VERIFY_PIECES, std::min<int64_t>(cdiv64(d->vocab, 1024), 1024 / d->batch));
    if (a.pieces >= 2 && d->vocab >= 16384) a.launches = d->q && d->parents ? std::min(1 + (uint32_t)std::max(d->tokens - 2, 0), VERIFY_LAUNCHES) : 1;
    if (!a.launches) a.pieces = 1;
    a.piece = (uint32_t)cdiv64(cdiv64(d->vocab, a.pieces), 256) * 256;
    bytes = (size_t)a.launches * d->batch * (sizeof(VerifyState) + a.pieces * sizeof(double)) + (a.launches > 1 ? (size_t)d->batch * d->tokens * 8 : 0);
}

// Strides of [batch][tokens][vocab] numbers, those of dimensions of size one not read.
bool rows(int64_t& batch, int64_t& token, int64_t given_batch, int64_t given_token, const depsync_verify_drafts_desc* d) {
    batch = d->batch > 1 ? given_batch : 0;
    token = d->tokens > 1 ? given_token : 0;
    return batch >= 0 && token >= 0 && batch <= (int64_t)1 << 40 && token <= (int64_t)1 << 40;
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
    if (int rc = tree_operands(d, a, 8); rc != DEPSYNC_OK) return rc;
    if (int rc = tree_plan(d, 0, a, need); rc != DEPSYNC_OK) return rc;
    if (need > 0 && (!operand(workspace) || workspace_bytes < need)) return DEPSYNC_EINVAL;
    a.parts = static_cast<float*>(workspace);
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
        !optional(d->accepted) || !optional(d->n_accepted) || !optional(d->weights) || !optional(d->pos) || (d->pos && !array(d->start)) || !optional(d->n_out) ||
        !apart({d->cached_out, d->n_out, d->weights, d->pos}, {d->cached, d->accepted, d->n_accepted, d->pos ? d->start : nullptr}))
        return DEPSYNC_EINVAL;
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

int depsync_tree_attn8_workspace(const depsync_tree_attn8_desc* d, int n_cu, size_t* bytes) {
    if (!bytes || !d) return DEPSYNC_EINVAL;
    if (int rc = tree_check(&d->attn); rc != DEPSYNC_OK) return rc;
    if (!cache8_block(d->block, d->attn.capacity)) return DEPSYNC_EINVAL;
    TreeAttn8Args a = {};
    return tree_plan(&d->attn, n_cu, a, *bytes, d->block);
}

int dep_tree_attn8(const depsync_tree_attn8_desc* d8, void* workspace, size_t workspace_bytes, void* stream) {
    if (!d8) return DEPSYNC_EINVAL;
    const depsync_tree_attn_desc* const d = &d8->attn;
    if (int rc = tree_check(d); rc != DEPSYNC_OK) return rc;
    if (!cache8_block(d8->block, d->capacity)) return DEPSYNC_EINVAL;
    TreeAttn8Args a = {};
    size_t need = 0;
    const int D = d->head_dim;
    if (!operand(d8->k_tail) || !operand(d8->v_tail) || !array(d8->k_scale) || !array(d8->v_scale)) return DEPSYNC_EINVAL;
    if (int rc = tree_operands(d, a, 16); rc != DEPSYNC_OK) return rc;
    if (!strides(a.tail_s, d8->tail_batch, d8->tail_token, d8->tail_head, d->batch, d8->block, d->kv_heads, D, false, true)) return DEPSYNC_EINVAL;
    if (int rc = tree_plan(d, 0, a, need, d8->block); rc != DEPSYNC_OK) return rc;
    if (need > 0 && (!operand(workspace) || workspace_bytes < need)) return DEPSYNC_EINVAL;
    a.k_scale = d8->k_scale; a.v_scale = d8->v_scale; a.k_tail = d8->k_tail; a.v_tail = d8->v_tail;
    a.block_log2 = d8->block == 32 ? 5 : d8->block == 64 ? 6 : 7;
    a.n_blocks = (uint32_t)(d->capacity / d8->block);
    a.together = d->kv_heads > 1 && a.cache_s.head < 128 ? 1 : 0;
    a.parts = static_cast<float*>(workspace);
    const hipError_t e = d->dtype == DEPSYNC_BF16 ? launch_tree_attn8_bf16(a, D, static_cast<hipStream_t>(stream)) : launch_tree_attn8_f16(a, D, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

int dep_cache_append8(const depsync_cache_append8_desc* d, void* stream) {
    if (!d) return DEPSYNC_EINVAL;
    if (int rc = common(d->batch, d->tokens, d->kv_heads, d->kv_heads, d->head_dim, d->dtype, d->capacity); rc != DEPSYNC_OK) return rc;
    CacheAppend8Args a = {};
    const int D = d->head_dim;
    if (!cache8_block(d->block, d->capacity) || d->n_max < 1 || d->n_max > 65536 || (!d->accepted && d->n_max > d->tokens)) return DEPSYNC_EINVAL;
    if (!operand(d->k_new) || !operand(d->v_new) || !operand(d->k_cache) || !operand(d->v_cache) || !operand(d->k_tail) || !operand(d->v_tail) ||
        !array(d->k_scale) || !array(d->v_scale) || !array(d->cached) || !array(d->cached_out) || !optional(d->accepted) || !optional(d->n_accepted) ||
        !optional(d->n_out) || !apart({d->cached_out, d->n_out}, {d->cached, d->accepted, d->n_accepted}))
        return DEPSYNC_EINVAL;
    if (!strides(a.new_s, d->new_batch, d->new_token, d->new_head, d->batch, d->tokens, d->kv_heads, D, false, false) ||
        !strides(a.cache_s, d->cache_batch, d->cache_token, d->cache_head, d->batch, d->capacity, d->kv_heads, D, true, true, 16) ||
        !strides(a.tail_s, d->tail_batch, d->tail_token, d->tail_head, d->batch, d->block, d->kv_heads, D, true, true))
        return DEPSYNC_EINVAL;
    a.n_blocks = (uint32_t)(d->capacity / d->block);
    a.most_full = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(a.n_blocks, ((int64_t)d->block - 1 + d->n_max) / d->block));
    if ((int64_t)d->batch * d->kv_heads * 2 * a.most_full > MAX_BLOCKS) return DEPSYNC_ENOTIMPL;
    a.k_new = d->k_new; a.v_new = d->v_new; a.k_cache = d->k_cache; a.v_cache = d->v_cache; a.k_tail = d->k_tail; a.v_tail = d->v_tail;
    a.k_scale = d->k_scale; a.v_scale = d->v_scale;
    a.cached = d->cached; a.cached_out = d->cached_out; a.accepted = d->accepted; a.n_accepted = d->n_accepted; a.n_out = d->n_out;
    a.batch = d->batch; a.tokens = d->tokens; a.kv_heads = d->kv_heads; a.capacity = d->capacity; a.n_max = d->n_max;
    const hipError_t e = launch_cache_append8(a, d->dtype, D, d->block, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

int dep_qk_norm_rope(const depsync_qk_norm_rope_desc* d, void* stream) {
    if (!d) return DEPSYNC_EINVAL;
    if (int rc = common(d->batch, d->tokens, d->heads, d->kv_heads, d->head_dim, d->dtype, 0); rc != DEPSYNC_OK) return rc;
    QkNormArgs a = {};
    const int D = d->head_dim, R = d->rotary_dim;
    if (R < 0 || R > D || R % 16 != 0 || (d->interleaved & ~1) || (d->norm & ~1) || !std::isfinite(d->eps) || d->eps < 0.0f) return DEPSYNC_EINVAL;
    if (!operand(d->q) || !operand(d->k) || !operand(d->q_out) || !operand(d->k_out) || !aligned(d->q_gain, 16) || !aligned(d->k_gain, 16) ||
        (R > 0 && !operand(d->freq)) || !optional(d->start) || !optional(d->depth) || !optional(d->drafted))
        return DEPSYNC_EINVAL;
    if (!strides(a.q_s, d->q_batch, d->q_token, d->q_head, d->batch, d->tokens, d->heads, D, false, false) ||
        !strides(a.k_s, d->k_batch, d->k_token, d->k_head, d->batch, d->tokens, d->kv_heads, D, false, false) ||
        !strides(a.q_out_s, d->q_out_batch, d->q_out_token, d->q_out_head, d->batch, d->tokens, d->heads, D, true, false) ||
        !strides(a.k_out_s, d->k_out_batch, d->k_out_token, d->k_out_head, d->batch, d->tokens, d->kv_heads, D, true, false))
        return DEPSYNC_EINVAL;
    auto same = [](const Strides& x, const Strides& y) { return x.batch == y.batch && x.token == y.token && x.head == y.head; };
    if ((d->q == d->q_out && !same(a.q_s, a.q_out_s)) || (d->k == d->k_out && !same(a.k_s, a.k_out_s))) return DEPSYNC_EINVAL;
    if (d->depth && d->depth_batch != 0 && d->depth_batch < d->tokens) return DEPSYNC_EINVAL;
    a.q = d->q; a.k = d->k; a.q_out = d->q_out; a.k_out = d->k_out; a.q_gain = d->q_gain; a.k_gain = d->k_gain; a.freq = d->freq;
    a.start = d->start; a.depth = d->depth; a.depth_batch = d->depth_batch; a.drafted = d->drafted;
    a.batch = d->batch; a.tokens = d->tokens; a.heads = d->heads; a.kv_heads = d->kv_heads; a.rotary_dim = R; a.eps = d->eps;
    const int64_t tokens = (int64_t)d->batch * d->tokens, at_once = 64 / (D / 16);
    a.q_waves = (uint32_t)cdiv64(d->heads, at_once);
    a.k_waves = (uint32_t)cdiv64(d->kv_heads, at_once);
    const bool streams = tokens * (d->heads + d->kv_heads) * D * 2 > L2_BYTES;
    if (cdiv64(tokens * (a.q_waves + a.k_waves), 4) > MAX_BLOCKS) return DEPSYNC_ENOTIMPL;
    const hipError_t e = launch_qk_norm_rope(a, d->dtype, D, d->interleaved != 0, d->norm != 0, streams, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

int depsync_verify_drafts_workspace(const depsync_verify_drafts_desc* d, size_t* bytes) {
    if (!bytes) return DEPSYNC_EINVAL;
    if (int rc = verify_check(d); rc != DEPSYNC_OK) return rc;
    VerifyArgs a = {};
    verify_plan(d, a, *bytes);
    return DEPSYNC_OK;
}

int dep_verify_drafts(const depsync_verify_drafts_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    if (int rc = depsync_verify_drafts_workspace(d, &need); rc != DEPSYNC_OK) return rc;
    VerifyArgs a = {};
    if (!array(d->p) || !optional(d->q) || !array(d->ids) || !optional(d->parents) || !optional(d->drafted) || !array(d->u) || !array(d->accepted) ||
        !array(d->n_accepted) || !array(d->next) || !apart({d->accepted, d->n_accepted, d->next}, {d->p, d->q, d->ids, d->parents, d->drafted, d->u}) || (d->parents && d->parents_batch != 0 && d->parents_batch < d->tokens))
        return DEPSYNC_EINVAL;
    if (!rows(a.p_batch, a.p_token, d->p_batch, d->p_token, d) || (d->q && !rows(a.q_batch, a.q_token, d->q_batch, d->q_token, d))) return DEPSYNC_EINVAL;
    if (need > 0 && (!operand(workspace) || workspace_bytes < need)) return DEPSYNC_EINVAL;
    a.p = d->p; a.q = d->q; a.ids = d->ids; a.parents = d->parents; a.parents_batch = d->parents_batch; a.drafted = d->drafted; a.u = d->u;
    a.accepted = d->accepted; a.n_accepted = d->n_accepted; a.next = d->next;
    a.batch = d->batch; a.tokens = d->tokens; a.vocab = d->vocab;
    verify_plan(d, a, need);
    a.sums = static_cast<double*>(workspace);
    a.states = reinterpret_cast<VerifyState*>(a.sums + (size_t)a.launches * d->batch * a.pieces);
    a.kept = reinterpret_cast<VerifyToken*>(a.states + (size_t)a.launches * d->batch);
    const hipError_t e = launch_verify_drafts(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DEPSYNC_OK : hip_fail(e);
}

}  // extern "C"
