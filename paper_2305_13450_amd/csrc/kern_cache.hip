// The cache beside attention: accepted keys and values appended, attention weights added up, rows of least weight evicted.
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "tree_attn.hpp"

namespace depsync {

namespace {

// ---- append ----------------------------------------------------------------------------------------------------------------
// A copy of n rows per sequence and head, D / 8 lanes to a row and 16 bytes to a lane, K and V alike.  Bound by launch latency for
// a tree's accepted path (32 sequences of up to 6 tokens: 3.0 us), by HBM for a prompt (4 x 1024 tokens of 8 heads, 34 MB read and written: 6.5 us).
template <int D>
__global__ __launch_bounds__(256) void cache_append_kernel(const CacheAppendArgs a) {
    constexpr uint32_t LANES = D / 8, ROWS = 256 / LANES;
    const uint32_t blocks = (a.n_max * a.kv_heads + ROWS - 1) / ROWS;
    const uint32_t b = blockIdx.x / blocks, blk = blockIdx.x % blocks;
    const uint32_t cached = clamp_count(a.cached[b], a.capacity);
    const uint32_t n = min(a.n_accepted ? clamp_count(a.n_accepted[b], a.n_max) : a.n_max, a.capacity - cached);
    if (blk == 0 && threadIdx.x == 0) {
        a.cached_out[b] = (int32_t)(cached + n);
        if (a.n_out) a.n_out[b] = (int32_t)n;
    }
    const uint32_t item = blk * ROWS + threadIdx.x / LANES, unit = threadIdx.x % LANES;
    const uint32_t i = item / a.kv_heads, h = item % a.kv_heads;
    if (i >= n) return;
    const uint32_t t = a.accepted ? clamp_count(a.accepted[(size_t)b * a.n_max + i], a.tokens - 1) : i;
    const int64_t from = (int64_t)b * a.new_s.batch + (int64_t)t * a.new_s.token + (int64_t)h * a.new_s.head;
    const int64_t to = (int64_t)b * a.cache_s.batch + (int64_t)(cached + i) * a.cache_s.token + (int64_t)h * a.cache_s.head;
    const u32x4 k = ((const u32x4*)((const uint16_t*)a.k_new + from))[unit];
    const u32x4 v = ((const u32x4*)((const uint16_t*)a.v_new + from))[unit];
    ((u32x4*)((uint16_t*)a.k_cache + to))[unit] = k;
    ((u32x4*)((uint16_t*)a.v_cache + to))[unit] = v;
    if (unit == 0) {
        const size_t at = ((size_t)b * a.kv_heads + h) * a.capacity + cached + i;
        if (a.weights) a.weights[at] = 0.0f;
        if (a.pos) a.pos[at] = a.start[b] + (int32_t)i;
    }
}

// ---- weights ---------------------------------------------------------------------------------------------------------------
// W_k += sum_r exp2(s_rk - lse_r): no running maximum is needed, as the sums are known, so every key is one workgroup's own and the
// sum over rows needs no atomics.  S = Q K^T this time: a lane owns one key, and its 16 accumulators are 16 of 32 rows.

// The accepted token i of a sequence.
__device__ __forceinline__ uint32_t accepted_token(const CacheWeightsArgs& a, uint32_t b, uint32_t i) {
    return a.accepted ? clamp_count(a.accepted[(size_t)b * a.n_max + i], a.tokens - 1) : i;
}
// In the place of its sum a row that is not there, and one that saw nothing, has this.  It makes the weights of finite scores 0; those of a key that is
// not finite are NaN (a row that is not there is zeros, and 0 x inf no number) and have to be set to 0.
constexpr float NO_ROW = 0x1.fffffep127f;
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
// A row's sum, base 2.
__device__ __forceinline__ float row_sum(const CacheWeightsArgs& a, uint32_t b, uint32_t token, uint32_t hq) {
    const float x = a.lse[((size_t)b * a.tokens + token) * a.heads + hq];
    return x == -INFINITY ? NO_ROW : x * 1.4426950408889634f;
}
// Sum over 16 rows of a lane's weights for its key: scores st, sums in LDS, and the last key that each row sees (-1 where its sum is NO_ROW), which
// is asked for where `masked`: where a row does not see all keys.
__device__ __forceinline__ float rows_weight(const f32x16& st, const float* lse, const int32_t* last, uint32_t h2, float sc, bool masked, int32_t key) {
    float p[16], part[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 l4 = *(const f32x4*)(lse + 8 * g + 4 * h2);
#pragma unroll
        for (int e = 0; e < 4; ++e) p[4 * g + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[4 * g + e], sc, -l4[e]));
    }
    if (masked) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const i32x4 last4 = *(const i32x4*)(last + 8 * g + 4 * h2);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (key > last4[e]) p[4 * g + e] = 0.0f;
        }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) part[g] = (p[4 * g] + p[4 * g + 1]) + (p[4 * g + 2] + p[4 * g + 3]);
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// At most 64 rows, those of an accepted path: the time is that of reading K once (16 sequences of 2500 to 4096 rows, 8 heads: 112 MB in
// 21.7 us, the rate of a copy).  The rows stay in LDS; each wave walks 32 of a block's
// 128 keys, the next ones on their way into registers meanwhile, and no wave waits for another.
template <typename T, int D>
__global__ __launch_bounds__(256, 3) void cache_weights_few_kernel(const CacheWeightsArgs a) {
    using Tile = KeyTile<T, D>;
    using M = Mma<T>;
    using V8 = typename M::V8;
    __shared__ __align__(16) char ldsQ[2 * Tile::BYTES];
    __shared__ __align__(16) char ldsK[4][Tile::BYTES];
    __shared__ __align__(16) float lse[64];
    __shared__ __align__(16) int32_t last[64];                     // the last key that the row sees
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uni(tid >> 6), h2 = lane >> 5;
    const uint32_t h = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, part = rest % a.n_parts, b = rest / a.n_parts;
    const uint32_t cached = uni(clamp_count(a.cached[b], a.capacity));
    const uint32_t n = uni(a.n_accepted ? clamp_count(a.n_accepted[b], a.n_max) : a.n_max);
    const uint32_t blocks = (cached + 127) / 128, begin = part * a.part_blocks;
    const uint32_t end = part + 1 == a.n_parts ? blocks : min(blocks, begin + a.part_blocks);
    if (begin >= end || n == 0) return;
    const uint32_t pitch = (uint32_t)a.cache_s.token * 2u, lrow = lane / Tile::CHUNKS, chunk = lane % Tile::CHUNKS;
    const char* const keys = (const char*)a.k_cache + ((int64_t)b * a.cache_s.batch + (int64_t)h * a.cache_s.head) * 2;
    float* const weights = a.weights + ((size_t)b * a.kv_heads + h) * a.capacity;
    u32x4 kreg[Tile::NI];
    float old = 0.0f;
    auto fetch = [&](uint32_t blk) __attribute__((always_inline)) {
        const uint32_t first = blk * 128 + wave * 32, have = first < cached ? min(32u, cached - first) : 0u;
        const OperandBuf K(uni_ptr(keys + (int64_t)first * pitch), uni(have ? (have - 1) * pitch + D * 2u : 0u));   // (rows that are not there: zeros)
        const uint32_t off = lrow * pitch + chunk * 16;
#pragma unroll
        for (uint32_t i = 0; i < Tile::NI; ++i) kreg[i] = K.load16(off, i * Tile::RPI * pitch);
        if (lane < have) old = weights[first + lane];
    };
    fetch(begin);
    const int32_t base = (int32_t)cached - (int32_t)n;             // row i sees keys 0..base + i
    const uint32_t rows = n * a.group;
    for (uint32_t x = tid; x < 64 * Tile::CHUNKS; x += 256) {
        const uint32_t r = x / Tile::CHUNKS, c = x % Tile::CHUNKS, i = r / a.group, g = r - i * a.group;
        u32x4 q = {0, 0, 0, 0};
        if (r < rows) q = ((const u32x4*)((const T*)a.q + (int64_t)b * a.q_s.batch + (int64_t)accepted_token(a, b, i) * a.q_s.token + (int64_t)(h * a.group + g) * a.q_s.head))[c];
        *(u32x4*)(ldsQ + r * Tile::PITCH + ((c ^ Tile::kswz(r)) << 4)) = q;
    }
    if (tid < 64) {
        const uint32_t i = tid / a.group, g = tid - i * a.group;
        const float sum = tid < rows ? row_sum(a, b, accepted_token(a, b, i), h * a.group + g) : NO_ROW;
        lse[tid] = sum;
        last[tid] = sum == NO_ROW ? -1 : base + (int32_t)i;
    }
    __syncthreads();
    const uint64_t none = __ballot(lse[lane] == NO_ROW);
    char* const mine = ldsK[wave];
    const uint32_t koff = Tile::koff(lane), kput = lrow * Tile::PITCH + ((chunk ^ Tile::kswz(lrow)) << 4);
    for (uint32_t blk = begin; blk < end; ++blk) {
        const uint32_t kp = opaque(kput);
#pragma unroll
        for (uint32_t i = 0; i < Tile::NI; ++i) *(u32x4*)(mine + (kp ^ ((Tile::kswz(i * Tile::RPI)) << 4)) + i * Tile::RPI * Tile::PITCH) = kreg[i];
        const float before = old;
        if (blk + 1 < end) fetch(blk + 1);
        asm volatile("" ::: "memory");                             // (a wave's LDS accesses keep their order)
        __builtin_amdgcn_wave_barrier();
        V8 kf[D / 16];
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) kf[kk] = *(const V8*)(mine + (koff ^ (kk * 32u)));
        const int32_t first = (int32_t)(blk * 128 + wave * 32), key = first + (int32_t)(lane & 31u);
        float w = 0.0f;
        for (uint32_t u = 0; u * 32 < rows; ++u) {
            f32x16 st;
#pragma unroll
            for (int v = 0; v < 16; ++v) st[v] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) st = M::mma(*(const V8*)(ldsQ + u * Tile::BYTES + (koff ^ (kk * 32u))), kf[kk], st);
            w += rows_weight(st, lse + 32 * u, last + 32 * u, h2, a.scale, (uint32_t)(none >> (32 * u)) != 0 || first + 31 > base, key);
        }
        w += __shfl_xor(w, 32);
        if (lane < 32 && key < (int32_t)cached) weights[key] = before + w;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

// More rows, those of a prompt: the time is that of the matrix cores and the exponentials (2048 tokens of 12 heads: 6.4 GFLOP and 25 million
// exponentials in 18.6 us; the first keys' workgroups walk 2048 rows, and every walk ends in a sum over eight waves).  A workgroup keeps 32 KT keys' fragments in
// registers, in every wave, and its waves walk the rows, 32 tokens of one query head at a time each, the next ones on their way into
// registers meanwhile.  (Rows by head and not by token: their addresses are a line then, and the last key they see as well.)
template <typename T, int D, int KT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES / 2) void cache_weights_many_kernel(const CacheWeightsArgs a) {
    using Tile = KeyTile<T, D>;
    using M = Mma<T>;
    using V8 = typename M::V8;
    constexpr uint32_t KEYS = 32 * KT, COPIES = Tile::NI * KT, NK = (COPIES + WAVES - 1) / WAVES;   // 1 KB copies of keys, a wave's
    __shared__ __align__(16) char lds[WAVES][Tile::BYTES];         // the keys, then each wave's rows
    __shared__ __align__(16) float lse[WAVES][32];
    __shared__ __align__(16) int32_t last[WAVES][32];              // the last key that the row sees
    __shared__ float joined[WAVES][KEYS];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uni(tid >> 6), h2 = lane >> 5;
    const uint32_t h = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, part = rest % a.n_parts, b = rest / a.n_parts;
    const uint32_t cached = uni(clamp_count(a.cached[b], a.capacity));
    const uint32_t n = uni(a.n_accepted ? clamp_count(a.n_accepted[b], a.n_max) : a.n_max);
    if (n == 0) return;
    const uint32_t lrow = lane / Tile::CHUNKS, chunk = lane % Tile::CHUNKS;
    const uint32_t koff = Tile::koff(lane), put = lrow * Tile::PITCH + ((chunk ^ Tile::kswz(lrow)) << 4);
    char* const mine = lds[wave];
    const uint32_t q_pitch = (uint32_t)a.q_s.token * 2u;
    const int32_t base = (int32_t)cached - (int32_t)n;             // row i sees keys 0..base + i
    for (uint32_t k0 = part * KEYS; k0 < cached; k0 += a.n_parts * KEYS) {   // (once, unless max_cached is less than a sequence has)
        V8 kf[KT][D / 16];
        {
            const uint32_t pitch = (uint32_t)a.cache_s.token * 2u, have = min(KEYS, cached - k0);
            const char* p = (const char*)a.k_cache + ((int64_t)b * a.cache_s.batch + (int64_t)k0 * a.cache_s.token + (int64_t)h * a.cache_s.head) * 2;
            const OperandBuf K(uni_ptr(p), uni((have - 1) * pitch + D * 2u));   // (rows that are not there: zeros)
            u32x4 reg[NK];                                         // (tiles of 32 keys behind one another)
#pragma unroll
            for (uint32_t i = 0; i < NK; ++i) reg[i] = K.load16(lrow * pitch + chunk * 16, (wave * NK + i) * Tile::RPI * pitch);
            __syncthreads();                                       // (the rows of the keys before are done with)
#pragma unroll
            for (uint32_t i = 0; i < NK; ++i) {
                const uint32_t rr = (wave * NK + i) * Tile::RPI + lrow;
                if (COPIES % WAVES == 0 || wave * NK + i < COPIES) *(u32x4*)(lds[0] + rr * Tile::PITCH + ((chunk ^ Tile::kswz(rr & 31u)) << 4)) = reg[i];
            }
            __syncthreads();
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) kf[t][kk] = *(const V8*)(lds[t] + (koff ^ (kk * 32u)));
            __syncthreads();
        }
        const uint32_t i_first = (int32_t)k0 > base ? (uint32_t)((int32_t)k0 - base) & ~31u : 0u;   // rows before see none of these keys
        const uint32_t i_end = i_first < n ? i_first + ((n - i_first + 31) & ~31u) : i_first;
        struct Place { uint32_t g, i; };                           // a step's query head and first token
        auto onward = [&](Place& x) __attribute__((always_inline)) {   // the wave's next step
            x.i += 32 * WAVES;
            while (x.i >= i_end && x.g < a.group) { x.i -= i_end - i_first; ++x.g; }
        };
        u32x4 qreg[Tile::NI];
        float sum = NO_ROW;
        auto fetch = [&](const Place& at) __attribute__((always_inline)) {
            const uint32_t hq = h * a.group + at.g, mine = at.i + (lane & 31u);
            const T* const q = (const T*)a.q + (int64_t)b * a.q_s.batch + (int64_t)hq * a.q_s.head;
            if (!a.accepted) {                                     // (rows that are not there: zeros)
                const OperandBuf Q(uni_ptr(q + (int64_t)at.i * a.q_s.token), uni((min(32u, n - at.i) - 1) * q_pitch + D * 2u));
#pragma unroll
                for (uint32_t i = 0; i < Tile::NI; ++i) qreg[i] = Q.load16(lrow * q_pitch + chunk * 16, i * Tile::RPI * q_pitch);
            } else {                                               // (the last one)
#pragma unroll
                for (uint32_t i = 0; i < Tile::NI; ++i)
                    qreg[i] = *(const u32x4*)(q + (int64_t)accepted_token(a, b, min(at.i + i * Tile::RPI + lrow, n - 1)) * a.q_s.token + chunk * 8);
            }
            const float x = row_sum(a, b, accepted_token(a, b, min(mine, n - 1)), hq);
            sum = mine < n ? x : NO_ROW;
        };
        float w[KT] = {};
        const int32_t key = (int32_t)(k0 + (lane & 31u));
        Place now = {0, i_first + wave * 32};
        while (now.i >= i_end && now.g < a.group && i_end > i_first) { now.i -= i_end - i_first; ++now.g; }
        if (i_end == i_first) now.g = a.group;                     // (no row sees these keys)
        if (now.g < a.group) fetch(now);
        while (now.g < a.group) {
            const uint32_t p = opaque(put);
#pragma unroll
            for (uint32_t i = 0; i < Tile::NI; ++i) *(u32x4*)(mine + (p ^ ((Tile::kswz(i * Tile::RPI)) << 4)) + i * Tile::RPI * Tile::PITCH) = qreg[i];
            const int32_t see = base + (int32_t)now.i;             // the last key that the first of these rows sees
            const bool none = __ballot(sum == NO_ROW) != 0;
            if (lane < 32) { lse[wave][lane] = sum; last[wave][lane] = sum == NO_ROW ? -1 : see + (int32_t)lane; }
            onward(now);
            if (WAVES == 4 && now.g < a.group) fetch(now);
            asm volatile("" ::: "memory");                         // (a wave's LDS accesses keep their order)
            __builtin_amdgcn_wave_barrier();
            V8 q[D / 16];
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) q[kk] = *(const V8*)(mine + (koff ^ (kk * 32u)));
            f32x16 st[KT];
#pragma unroll
            for (int t = 0; t < KT; ++t) {                         // (one tile's scores beside the other's exponentials)
#pragma unroll
                for (int v = 0; v < 16; ++v) st[t][v] = 0.0f;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) st[t] = M::mma(q[kk], kf[t][kk], st[t]);
            }
            if (WAVES == 8) {                                      // (into the registers that the fragments have left: 128 are there)
                __builtin_amdgcn_sched_barrier(0);
                if (now.g < a.group) fetch(now);
            }
#pragma unroll
            for (int t = 0; t < KT; ++t)
                w[t] += rows_weight(st[t], lse[wave], last[wave], h2, a.scale, none || (int32_t)k0 + 32 * t + 31 > see, key + 32 * t);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            w[t] += __shfl_xor(w[t], 32);
            if (lane < 32) joined[wave][32 * t + lane] = w[t];
        }
        __syncthreads();
        if (tid < KEYS && k0 + tid < cached) {
            float x = (joined[0][tid] + joined[1][tid]) + (joined[2][tid] + joined[3][tid]);
            if (WAVES == 8) x += (joined[4][tid] + joined[5][tid]) + (joined[6][tid] + joined[7][tid]);
            a.weights[((size_t)b * a.kv_heads + h) * a.capacity + k0 + tid] += x;
        }
    }
}

// ---- evict -----------------------------------------------------------------------------------------------------------------
// The rows that stay are those with the `budget` largest 32-bit keys (weight as an ordered integer; the newest above all), the
// lowest rows among equal ones: four passes over 8 bits each find the smallest key that stays and how many of its equals do, a
// walk in row order then lists the moves.  One workgroup per sequence and head; the keys stay in LDS where they fit.  A few rows' worth of
// arithmetic on 8 bytes a row: bound by the latencies of its steps (2053 rows of 256 heads 10.8 us, 16384 of 32 heads 29 us), so loads go out eight to
// a thread at once, and a step that appended few rows moves them in the same launch (a separate one: 15.2 us and 3).
constexpr uint32_t EVICT_LDS_KEYS = 32768, EVICT_LOADS = 8, EVICT_FUSED = 256, EVICT_FEW = 16;

// Larger float, larger integer; NaN is the least.  Infinity is below 0xffffffff, the key of the newest rows.
__device__ __forceinline__ uint32_t evict_key(float w) {
    const uint32_t x = __builtin_bit_cast(uint32_t, w + 0.0f);       // (-0 counts as 0)
    return w == w ? (x & 0x80000000u ? ~x : x | 0x80000000u) : 0u;
}
__device__ __forceinline__ bool evict_new(int32_t pos, int32_t newest, uint32_t recent) { return (int64_t)pos > (int64_t)newest - (int64_t)recent; }

// Exclusive sum over the threads of the workgroup, and the total.
template <uint32_t THREADS>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* wave_sums, uint32_t& total) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t x = wave_sums_to(v);
    __syncthreads();                                                 // (the sums of the scan before are read)
    if (lane == 63) wave_sums[wave] = x;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (uint32_t i = 0; i < THREADS / 64; ++i) {
        const uint32_t s = wave_sums[i];
        before += i < wave ? s : 0u;
        all += s;
    }
    total = all;
    return before + x - v;
}

// Row src of the cache to row dst, 16 bytes to each of `lanes` threads.
__device__ __forceinline__ void move_row(const CacheEvictArgs& a, uint32_t pair, uint32_t src, uint32_t dst, uint32_t unit) {
    const uint32_t b = pair / a.kv_heads, h = pair % a.kv_heads;
    const int64_t from = (int64_t)b * a.cache_s.batch + (int64_t)src * a.cache_s.token + (int64_t)h * a.cache_s.head;
    const int64_t to = (int64_t)b * a.out_s.batch + (int64_t)dst * a.out_s.token + (int64_t)h * a.out_s.head;
    const u32x4 k = ((const u32x4*)((const uint16_t*)a.k_cache + from))[unit];
    const u32x4 v = ((const u32x4*)((const uint16_t*)a.v_cache + from))[unit];
    ((u32x4*)((uint16_t*)a.k_out + to))[unit] = k;
    ((u32x4*)((uint16_t*)a.v_out + to))[unit] = v;
    if (unit == 0) {
        const size_t f = (size_t)pair * a.capacity + src, t = (size_t)pair * a.capacity_out + dst;
        a.weights_out[t] = a.weights[f];
        a.pos_out[t] = a.pos[f];
    }
}

template <uint32_t THREADS, uint32_t LDS_KEYS>
__global__ __launch_bounds__(THREADS) void cache_evict_select_kernel(const CacheEvictArgs a) {
    __shared__ uint32_t keys[LDS_KEYS];
    __shared__ uint32_t hist[2][256], wave_sums[THREADS / 64], found[3];
    __shared__ int32_t newest_of[THREADS / 64];
    __shared__ uint64_t least_of[2][THREADS / 64];
    __shared__ uint32_t gone[EVICT_FEW];
    __shared__ uint32_t moved[2][EVICT_FUSED];                       // the first moves: where from, where to
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const uint32_t b = blockIdx.x / a.kv_heads, h = blockIdx.x % a.kv_heads;
    const uint32_t n = uni(clamp_count(a.cached[b], a.capacity));
    uint32_t* const list = a.moves + (size_t)blockIdx.x * (1 + 2 * (size_t)a.max_moves);
    if (h == 0 && tid == 0) a.cached_out[b] = (int32_t)min(n, a.budget);
    const uint32_t unit = tid % a.lanes;
    if (n <= a.budget) {
        const uint32_t moves = a.in_place ? 0u : n;
        if (tid == 0) list[0] = moves;
        if (a.fused)
            for (uint32_t i = tid / a.lanes; i < moves; i += THREADS / a.lanes) move_row(a, blockIdx.x, i, i, unit);
        else
            for (uint32_t i = tid; i < moves; i += THREADS) list[1 + i] = i;
        return;
    }
    const float* const w = a.weights + (size_t)blockIdx.x * a.capacity;
    const int32_t* const pos = a.pos + (size_t)blockIdx.x * a.capacity;
    const bool in_lds = n <= LDS_KEYS, at_once = n <= THREADS * EVICT_LOADS;
    if (tid < 256) hist[0][tid] = 0;
    int32_t newest = INT32_MIN, y[EVICT_LOADS];
    for (uint32_t i0 = 0; i0 < n; i0 += THREADS * EVICT_LOADS) {
        float x[EVICT_LOADS];
#pragma unroll
        for (uint32_t e = 0; e < EVICT_LOADS; ++e) {
            const uint32_t i = min(i0 + e * THREADS + tid, n - 1);    // (the last row again and again: the same key)
            x[e] = w[i]; y[e] = pos[i];
        }
#pragma unroll
        for (uint32_t e = 0; e < EVICT_LOADS; ++e) {
            if (in_lds) keys[min(i0 + e * THREADS + tid, n - 1)] = evict_key(x[e]);
            newest = max(newest, y[e]);
        }
    }
    // (positions as unsigned numbers in the same order)
    newest = (int32_t)(last_lane(wave_prefix((uint32_t)newest ^ 0x80000000u, 0u, [](uint32_t p, uint32_t q) { return max(p, q); })) ^ 0x80000000u);
    if (lane == 0) newest_of[wave] = newest;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < THREADS / 64; ++i) newest = max(newest, newest_of[i]);
    if (in_lds && a.recent) {
        for (uint32_t i0 = 0; i0 < n; i0 += THREADS * EVICT_LOADS) {
            if (!at_once) {
#pragma unroll
                for (uint32_t e = 0; e < EVICT_LOADS; ++e) y[e] = pos[min(i0 + e * THREADS + tid, n - 1)];
            }
#pragma unroll
            for (uint32_t e = 0; e < EVICT_LOADS; ++e)
                if (evict_new(y[e], newest, a.recent)) keys[min(i0 + e * THREADS + tid, n - 1)] = 0xffffffffu;
        }
        __syncthreads();
    }
    auto key = [&](uint32_t i) __attribute__((always_inline)) { return in_lds ? keys[i] : evict_new(pos[i], newest, a.recent) ? 0xffffffffu : evict_key(w[i]); };
    uint32_t sources = 0;
    const uint32_t leaving = n - a.budget;
    if (a.in_place && leaving <= EVICT_FEW) {
        // A step's few: the least key (of equal ones the highest row) is looked for as often as rows have to go.
        uint64_t least = 0;
        for (uint32_t m = 0; m < leaving; ++m) {
            uint64_t mine = ~0ull;
            for (uint32_t i0 = 0; i0 < n; i0 += THREADS * 4) {
                uint32_t k[4];
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) k[e] = key(min(i0 + e * THREADS + tid, n - 1));
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) {
                    const uint64_t c = (uint64_t)k[e] << 32 | ~min(i0 + e * THREADS + tid, n - 1);
                    if (c > least && c < mine) mine = c;
                }
            }
            const uint32_t hi = last_lane(wave_prefix((uint32_t)(mine >> 32), ~0u, [](uint32_t p, uint32_t q) { return min(p, q); }));
            const uint32_t lo = last_lane(wave_prefix((uint32_t)(mine >> 32) == hi ? (uint32_t)mine : ~0u, ~0u, [](uint32_t p, uint32_t q) { return min(p, q); }));
            if (lane == 0) least_of[m & 1][wave] = (uint64_t)hi << 32 | lo;
            __syncthreads();
            least = ~0ull;
#pragma unroll
            for (uint32_t i = 0; i < THREADS / 64; ++i) least = min(least, least_of[m & 1][i]);
            if (tid == 0) gone[m] = ~(uint32_t)least;
        }
        __syncthreads();
        if (wave == 0) {                                             // lane l < leaving: the row gone[l], and row budget + l
            const uint32_t g = lane < leaving ? gone[lane] : ~0u, r = a.budget + lane;
            uint32_t at = 0;
            bool stays = lane < leaving;
            for (uint32_t m = 0; m < leaving; ++m) { at += gone[m] < g ? 1u : 0u; stays = stays && gone[m] != r; }
            if (g < a.budget) { moved[1][at] = g; list[1 + a.max_moves + at] = g; }
            const uint64_t all = __ballot(stays);
            const uint32_t si = (uint32_t)__popcll(all & ((1ull << lane) - 1));
            if (stays) { moved[0][si] = r; list[1 + si] = r; }
            if (lane == 0) found[0] = (uint32_t)__popcll(all);
        }
        __syncthreads();
        sources = found[0];
    } else {
    // The smallest key that stays, from its highest 8 bits down; `need` keys with these bits stay.  Where all of them do, the rest is zeros.
    uint32_t prefix = 0, need = a.budget;
    for (int shift = 24, buf = 0; shift >= 0; shift -= 8, buf ^= 1) {
        for (uint32_t i0 = 0; i0 < n; i0 += THREADS * 4) {
            uint32_t k[4];
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) k[e] = key(min(i0 + e * THREADS + tid, n - 1));
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                bool todo = i0 + e * THREADS + tid < n && (shift == 24 || k[e] >> (shift + 8) == prefix);
                const uint32_t bin = (k[e] >> shift) & 255u;
                // Many keys share a bin (weights of one magnitude, rows that nothing attended to): a wave adds its first bins at once while that is
                // worth it.
#pragma unroll
                for (int peel = 0; peel < 2; ++peel) {
                    const uint64_t left = __ballot(todo);
                    if (__popcll(left) < 24) break;
                    const uint32_t bin0 = (uint32_t)__builtin_amdgcn_readlane((int)bin, (int)__builtin_ctzll(left));
                    const uint64_t same = __ballot(todo && bin == bin0);
                    if (lane == 0) atomicAdd(&hist[buf][bin0], (uint32_t)__popcll(same));
                    todo = todo && bin != bin0;
                }
                if (todo) atomicAdd(&hist[buf][bin], 1u);
            }
        }
        __syncthreads();
        if (wave == 0) {                                             // lane l: bins 255 - 4 l .. 252 - 4 l, from the top
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) { c[e] = hist[buf][255 - 4 * lane - e]; sum += c[e]; }
            uint32_t above = wave_sums_to(sum) - sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (above < need && need <= above + c[e]) { found[0] = 255 - 4 * lane - e; found[1] = need - above; found[2] = need == above + c[e]; }
                above += c[e];
            }
        } else if (wave < 5) {
            hist[buf ^ 1][tid - 64] = 0;
        }
        __syncthreads();
        prefix = prefix << 8 | found[0];
        need = found[1];
        if (found[2]) { prefix <<= shift; need = 0xffffffffu; break; }   // (uniform)
    }
    // in row order: of the rows with that key the first `need` stay
    uint32_t equal = 0, holes = 0;
    for (uint32_t i0 = 0; i0 < n; i0 += THREADS * EVICT_LOADS) {
        const uint32_t first = i0 + tid * EVICT_LOADS;
        uint32_t k[EVICT_LOADS], eq = 0;
#pragma unroll
        for (uint32_t e = 0; e < EVICT_LOADS; ++e) {
            k[e] = first + e < n ? key(first + e) : 0u;
            eq += first + e < n && k[e] == prefix;
        }
        uint32_t all, rank = 0;
        if (need != 0xffffffffu) {
            rank = equal + block_scan<THREADS>(eq, wave_sums, all);
            equal += all;
        }
        uint32_t hole = 0, source = 0;                               // one bit a row
#pragma unroll
        for (uint32_t e = 0; e < EVICT_LOADS; ++e) {
            const bool there = first + e < n, is = there && k[e] == prefix;
            const bool stays = there && (k[e] > prefix || (is && rank < need));
            rank += is;
            hole |= (a.in_place && there && !stays && first + e < a.budget ? 1u : 0u) << e;
            source |= (stays && (!a.in_place || first + e >= a.budget) ? 1u : 0u) << e;
        }
        // holes in the low half, sources in the high (at most 8192 of each)
        const uint32_t at = block_scan<THREADS>(__popc(hole) | __popc(source) << 16, wave_sums, all);
        uint32_t hi = holes + (at & 0xffffu), si = sources + (at >> 16);
#pragma unroll
        for (uint32_t e = 0; e < EVICT_LOADS; ++e) {
            if (source >> e & 1u) {
                list[1 + si] = first + e;
                if (si < EVICT_FUSED) moved[0][si] = first + e;
                ++si;
            }
            if (hole >> e & 1u) {
                list[1 + a.max_moves + hi] = first + e;
                if (hi < EVICT_FUSED) moved[1][hi] = first + e;
                ++hi;
            }
        }
        holes += all & 0xffffu;
        sources += all >> 16;
    }
    }
    if (!a.fused) {
        if (tid == 0) list[0] = sources;
        return;
    }
    __syncthreads();
    for (uint32_t m = tid / a.lanes; m < sources; m += THREADS / a.lanes) {
        const uint32_t src = m < EVICT_FUSED ? moved[0][m] : list[1 + m];
        const uint32_t dst = !a.in_place ? m : m < EVICT_FUSED ? moved[1][m] : list[1 + a.max_moves + m];
        move_row(a, blockIdx.x, src, dst, unit);
    }
}

// The listed rows moved.  In place sources lie behind the budget and their places before it, so no row is both.  Bound by HBM, on rows of 256 bytes
// (4 x 2000 rows of 8 heads, 66 MB read and written: 12 us, 5.4 TB/s).
__global__ __launch_bounds__(256) void cache_evict_move_kernel(const CacheEvictArgs a, uint32_t blocks) {
    const uint32_t pair = blockIdx.x / blocks, blk = blockIdx.x % blocks, rows = 256 / a.lanes;
    const uint32_t* const list = a.moves + (size_t)pair * (1 + 2 * (size_t)a.max_moves);
    const uint32_t n = list[0];
    for (uint32_t m = blk * rows + threadIdx.x / a.lanes; m < n; m += blocks * rows)
        move_row(a, pair, list[1 + m], a.in_place ? list[1 + a.max_moves + m] : m, threadIdx.x % a.lanes);
}

template <typename T, int D>
hipError_t launch_weights_of(const CacheWeightsArgs& a, hipStream_t stream) {
    const uint32_t blocks = a.batch * a.kv_heads * a.n_parts;
    if (a.few) return launch_one(cache_weights_few_kernel<T, D>, blocks, 256, stream, a);
    if (a.keys == 64) return launch_one(cache_weights_many_kernel<T, D, 2, 4>, blocks, 256, stream, a);
    return launch_one(cache_weights_many_kernel<T, D, 1, 8>, blocks, 512, stream, a);
}

}  // namespace

hipError_t launch_cache_append(const CacheAppendArgs& a, int head_dim, hipStream_t stream) {
    const uint32_t rows = 256 / (head_dim / 8);
    const uint32_t blocks = a.batch * ((a.n_max * a.kv_heads + rows - 1) / rows);
    return head_dim == 128 ? launch_one(cache_append_kernel<128>, blocks, 256, stream, a) : launch_one(cache_append_kernel<64>, blocks, 256, stream, a);
}

hipError_t launch_cache_weights(const CacheWeightsArgs& a, int dtype, int head_dim, hipStream_t stream) {
    if (dtype == 0) return head_dim == 128 ? launch_weights_of<__bf16, 128>(a, stream) : launch_weights_of<__bf16, 64>(a, stream);
    return head_dim == 128 ? launch_weights_of<_Float16, 128>(a, stream) : launch_weights_of<_Float16, 64>(a, stream);
}

hipError_t launch_cache_evict(const CacheEvictArgs& given, int head_dim, hipStream_t stream) {
    CacheEvictArgs a = given;
    const uint32_t pairs = a.batch * a.kv_heads;
    a.lanes = head_dim / 8;
    // As many moves as a sequence of max_cached rows makes (the kernels walk any number).  A workgroup moves 64 or 128 rows at a time, so up to
    // EVICT_FUSED they are not worth another launch.
    const uint32_t most = a.in_place ? (a.max_cached > a.budget ? a.max_cached - a.budget : 0u) : a.budget;
    a.fused = most <= EVICT_FUSED;
    // Half the waves have half the way to a barrier, and less LDS leaves room for other workgroups (2053 rows of 256 heads 14.1 and 10.6 us)
    const hipError_t e = a.max_cached <= 512 * EVICT_LOADS ? launch_one(cache_evict_select_kernel<512, 8192>, pairs, 512, stream, a)
                                                           : launch_one(cache_evict_select_kernel<1024, EVICT_LDS_KEYS>, pairs, 1024, stream, a);
    if (e != hipSuccess || a.fused) return e;
    uint32_t blocks = (most < a.max_moves ? most : a.max_moves) / (256 / a.lanes) + 1;
    blocks = min(blocks, max(1u, min(256u, (1u << 23) / pairs)));
    void* args[] = {&a, &blocks};
    return hipLaunchKernel(reinterpret_cast<const void*>(cache_evict_move_kernel), dim3(pairs * blocks), dim3(256), args, 0, stream);
}

hipError_t launch_tree_attn(const TreeAttnArgs& a, int dtype, int head_dim, hipStream_t stream) {
    return dtype == 0 ? launch_tree_attn_bf16(a, head_dim, stream) : launch_tree_attn_f16(a, head_dim, stream);
}

}  // namespace depsync
