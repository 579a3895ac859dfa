// The cache beside attention: accepted keys and values appended, attention weights added up, rows of least weight evicted.
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "tree_attn.hpp"

namespace depsync {

namespace {

// ---- append ----------------------------------------------------------------------------------------------------------------
// A copy of n rows per sequence and head, D / 8 lanes to a row and 16 bytes to a lane, K and V alike.  Bound by launch latency for
// a tree's accepted path, by HBM for a prompt.
template <int D>
__global__ __launch_bounds__(256) void cache_append_kernel(const CacheAppendArgs a) {
    constexpr uint32_t LANES = D / 8, ROWS = 256 / LANES;
    const uint32_t blocks = (a.n_max * a.kv_heads + ROWS - 1) / ROWS;
    const uint32_t b = blockIdx.x / blocks, blk = blockIdx.x % blocks;
    const uint32_t cached = clamp_count(a.cached[b], a.capacity);
    const uint32_t n = min(a.n_accepted ? clamp_count(a.n_accepted[b], a.n_max) : a.n_max, a.capacity - cached);
    if (blk == 0 && threadIdx.x == 0) a.cached_out[b] = (int32_t)(cached + n);
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
// sum over rows needs no atomics.  S = Q K^T this time: a lane owns one key, and its 16 accumulators are 16 of 32 rows.  A wave
// keeps its 32 keys' fragments in registers and walks the rows, which the workgroup copies to LDS 64 at a time, two stages in turn.
// Few rows (an accepted path): the time is that of reading K once.  Many (a prompt): the matrix cores' and the exponentials'.
// KW waves lie along the keys and 4 / KW along the rows.
template <typename T, int D, int KW>
__global__ __launch_bounds__(256) void cache_weights_kernel(const CacheWeightsArgs a) {
    using Tile = KeyTile<T, D>;
    using M = Mma<T>;
    using V8 = typename M::V8;
    constexpr uint32_t KEYS = 32 * KW, STAGE = 2 * Tile::BYTES;
    __shared__ __align__(16) char lds[2 * STAGE];                  // first the keys, then two stages of 64 query rows
    __shared__ __align__(16) float lse[2][64];                     // base 2
    __shared__ __align__(16) int32_t last[2][64];                  // the last key that the row sees
    __shared__ float joined[2][64];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uni(tid >> 6), h2 = lane >> 5;
    const uint32_t blocks = (a.max_cached + KEYS - 1) / KEYS;
    const uint32_t pair = blockIdx.x / blocks, b = pair / a.kv_heads, h = pair % a.kv_heads;
    const uint32_t cached = uni(clamp_count(a.cached[b], a.capacity));
    const uint32_t n = uni(a.n_accepted ? clamp_count(a.n_accepted[b], a.n_max) : a.n_max);
    if (n == 0) return;
    for (uint32_t k0 = (blockIdx.x % blocks) * KEYS; k0 < cached; k0 += blocks * KEYS) {   // (once, unless max_cached is less than a sequence has)
    const int32_t base = (int32_t)cached - (int32_t)n;             // row i sees keys 0..base + i
    const uint32_t i_first = (int32_t)k0 > base ? (uint32_t)((int32_t)k0 - base) : 0u;   // the first row that sees one of these keys
    const uint32_t rows = n * a.group, r_first = i_first * a.group / 64 * 64;
    const uint32_t lrow = lane / Tile::CHUNKS, chunk = lane % Tile::CHUNKS;
    V8 kf[D / 16];
    const uint32_t kw = wave % KW, rw = wave / KW;
    {
        const uint32_t first = k0 + kw * 32, have = first < cached ? min(32u, cached - first) : 0u;
        const uint32_t pitch = (uint32_t)a.cache_s.token * 2u;
        const char* p = (const char*)a.k_cache + ((int64_t)b * a.cache_s.batch + (int64_t)first * a.cache_s.token + (int64_t)h * a.cache_s.head) * 2;
        const OperandBuf K(uni_ptr(p), uni(have ? (have - 1) * pitch + D * 2u : 0u));
        char* const mine = lds + wave * Tile::BYTES;
        u32x4 reg[Tile::NI];
#pragma unroll
        for (uint32_t i = 0; i < Tile::NI; ++i) reg[i] = K.load16((i * Tile::RPI + lrow) * pitch + chunk * 16, 0);
#pragma unroll
        for (uint32_t i = 0; i < Tile::NI; ++i) {
            const uint32_t rr = i * Tile::RPI + lrow;
            *(u32x4*)(mine + rr * Tile::PITCH + ((chunk ^ Tile::kswz(rr)) << 4)) = reg[i];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        const uint32_t koff = Tile::koff(lane);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) kf[kk] = *(const V8*)(mine + (koff ^ (kk * 32u)));
    }
    // 64 rows of Q: each thread copies 16 bytes of every fourth 1 KB, and one of 64 rows' sum
    constexpr uint32_t NI = Tile::NI / 2;
    const uint32_t qrow = wave * (Tile::RPI * NI) + lrow;
    u32x4 qreg[NI];
    float lse_reg = INFINITY;
    int32_t last_reg = -1;
    auto token = [&](uint32_t i) __attribute__((always_inline)) {
        return a.accepted ? clamp_count(a.accepted[(size_t)b * a.n_max + i], a.tokens - 1) : i;
    };
    auto fetch = [&](uint32_t r0) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) {
            const uint32_t r = r0 + i * Tile::RPI + qrow;
            qreg[i] = u32x4{0, 0, 0, 0};
            if (r < rows) {
                const uint32_t at = r / a.group, g = r - at * a.group;
                const T* p = (const T*)a.q + (int64_t)b * a.q_s.batch + (int64_t)token(at) * a.q_s.token + (int64_t)(h * a.group + g) * a.q_s.head;
                qreg[i] = ((const u32x4*)p)[chunk];
            }
        }
        if (tid < 64) {
            const uint32_t r = r0 + tid;
            lse_reg = INFINITY; last_reg = -1;                     // no such row: no weight
            if (r < rows) {
                const uint32_t at = r / a.group, g = r - at * a.group;
                const float x = a.lse[((size_t)b * a.tokens + token(at)) * a.heads + h * a.group + g];
                lse_reg = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;   // (a row that saw nothing gives none)
                last_reg = base + (int32_t)at;
            }
        }
    };
    auto put = [&](uint32_t s) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) {
            const uint32_t rr = i * Tile::RPI + qrow;
            *(u32x4*)(lds + s * STAGE + rr * Tile::PITCH + ((chunk ^ Tile::kswz(rr)) << 4)) = qreg[i];
        }
        if (tid < 64) { lse[s][tid] = lse_reg; last[s][tid] = last_reg; }
    };
    float w = 0.0f;
    const int32_t key = (int32_t)(k0 + kw * 32 + (lane & 31u));
    const uint32_t koff = Tile::koff(lane);
    fetch(r_first);
    __syncthreads();                                               // every wave has its keys: the stages may be written
    put(0);
    if (r_first + 64 < rows) fetch(r_first + 64);
    __syncthreads();
    for (uint32_t r0 = r_first, s = 0; r0 < rows; r0 += 64, s ^= 1u) {
#pragma unroll
        for (uint32_t u = 0; u < 2; ++u) {
            if (KW < 4 && u != rw) continue;
            f32x16 st;
#pragma unroll
            for (int v = 0; v < 16; ++v) st[v] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const V8 qf = *(const V8*)(lds + s * STAGE + u * Tile::BYTES + (koff ^ (kk * 32u)));
                st = M::mma(qf, kf[kk], st);
            }
            const bool cut = base + (int32_t)((r0 + 32 * u) / a.group) < (int32_t)(k0 + KEYS - 1);
            float part = 0.0f;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 l4 = *(const f32x4*)(&lse[s][32 * u + 8 * g + 4 * h2]);
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[4 * g + e], a.scale, -l4[e]));
                if (cut) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key > last[s][32 * u + 8 * g + 4 * h2 + e]) p[e] = 0.0f;
                }
                part += (p[0] + p[1]) + (p[2] + p[3]);
            }
            w += part;
        }
        if (r0 + 64 < rows) {
            put(s ^ 1u);
            if (r0 + 128 < rows) fetch(r0 + 128);
        }
        __syncthreads();
    }
    w += __shfl_xor(w, 32);
    if constexpr (KW < 4) {
        if (rw == 1 && lane < 32) joined[kw][lane] = w;
        __syncthreads();
        if (rw == 0 && lane < 32) w += joined[kw][lane];
    }
    if (rw == 0 && lane < 32 && key < (int32_t)cached) a.weights[((size_t)b * a.kv_heads + h) * a.capacity + key] += w;
    __syncthreads();                                               // the stages are done with
    }
}

// ---- evict -----------------------------------------------------------------------------------------------------------------
// The rows that stay are those with the `budget` largest 32-bit keys (weight as an ordered integer; the newest above all), the
// lowest rows among equal ones: four passes over 8 bits each find the smallest key that stays and how many of its equals do, a
// walk in row order then lists the moves.  One workgroup per sequence and head; the keys stay in LDS where they fit.
constexpr uint32_t EVICT_THREADS = 1024, EVICT_LDS_KEYS = 32768, EVICT_VPT = 4;

__device__ __forceinline__ uint32_t evict_key(float w, int32_t pos, int32_t newest, int32_t recent) {
    if ((int64_t)pos > (int64_t)newest - recent) return 0xffffffffu;
    if (!(w == w)) return 0u;
    const uint32_t x = __builtin_bit_cast(uint32_t, w + 0.0f);       // (-0 counts as 0)
    const uint32_t k = x & 0x80000000u ? ~x : x | 0x80000000u;       // larger float, larger integer; infinity is below the newest
    return k;
}

// Exclusive sum over the threads of the workgroup, and the total.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* wave_sums, uint32_t& total) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(x, d);
        if (lane >= (uint32_t)d) x += y;
    }
    __syncthreads();                                                 // (the sums of the scan before are read)
    if (lane == 63) wave_sums[wave] = x;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (uint32_t i = 0; i < EVICT_THREADS / 64; ++i) {
        const uint32_t s = wave_sums[i];
        before += i < wave ? s : 0u;
        all += s;
    }
    total = all;
    return before + x - v;
}

__global__ __launch_bounds__(1024) void cache_evict_select_kernel(const CacheEvictArgs a) {
    __shared__ uint32_t keys[EVICT_LDS_KEYS];
    __shared__ uint32_t hist[256], wave_sums[EVICT_THREADS / 64], found[2];
    __shared__ int32_t newest_of[EVICT_THREADS / 64];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const uint32_t b = blockIdx.x / a.kv_heads, h = blockIdx.x % a.kv_heads;
    const uint32_t n = uni(clamp_count(a.cached[b], a.capacity));
    uint32_t* const list = a.moves + (size_t)blockIdx.x * (1 + 2 * (size_t)a.max_moves);
    if (h == 0 && tid == 0) a.cached_out[b] = (int32_t)min(n, a.budget);
    if (n <= a.budget) {
        const uint32_t moves = a.in_place ? 0u : n;
        if (tid == 0) list[0] = moves;
        for (uint32_t i = tid; i < moves; i += EVICT_THREADS) list[1 + i] = i;
        return;
    }
    const float* const w = a.weights + (size_t)blockIdx.x * a.capacity;
    const int32_t* const pos = a.pos + (size_t)blockIdx.x * a.capacity;
    int32_t newest = INT32_MIN;
    for (uint32_t i = tid; i < n; i += EVICT_THREADS) newest = max(newest, pos[i]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) newest = max(newest, __shfl_xor(newest, d));
    if (lane == 0) newest_of[wave] = newest;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < EVICT_THREADS / 64; ++i) newest = max(newest, newest_of[i]);
    const bool in_lds = n <= EVICT_LDS_KEYS;
    if (in_lds)
        for (uint32_t i = tid; i < n; i += EVICT_THREADS) keys[i] = evict_key(w[i], pos[i], newest, (int32_t)a.recent);
    auto key = [&](uint32_t i) __attribute__((always_inline)) { return in_lds ? keys[i] : evict_key(w[i], pos[i], newest, (int32_t)a.recent); };
    // the smallest key that stays, from its highest 8 bits down; `need` keys with these bits stay
    uint32_t prefix = 0, need = a.budget;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (uint32_t i = tid; i < 256; i += EVICT_THREADS) hist[i] = 0;
        __syncthreads();
        for (uint32_t i0 = 0; i0 < n; i0 += EVICT_THREADS) {
            const uint32_t i = i0 + tid;
            const uint32_t k = i < n ? key(i) : 0u;
            bool todo = i < n && (shift == 24 || k >> (shift + 8) == prefix);
            const uint32_t bin = (k >> shift) & 255u;
            // many keys share a bin (weights of one magnitude, rows that nothing attended to): a wave adds its first two bins at once
#pragma unroll
            for (int peel = 0; peel < 2; ++peel) {
                const uint64_t left = __ballot(todo);
                if (!left) break;
                const uint32_t lead = (uint32_t)__builtin_ctzll(left), bin0 = __shfl(bin, lead);
                const uint64_t same = __ballot(todo && bin == bin0);
                if (lane == lead) atomicAdd(&hist[bin0], (uint32_t)__popcll(same));
                todo = todo && bin != bin0;
            }
            if (todo) atomicAdd(&hist[bin], 1u);
        }
        __syncthreads();
        if (wave == 0) {                                             // lane l: bins 255 - 4 l .. 252 - 4 l, from the top
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) { c[e] = hist[255 - 4 * lane - e]; sum += c[e]; }
            uint32_t x = sum;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t y = __shfl_up(x, d);
                if (lane >= (uint32_t)d) x += y;
            }
            uint32_t above = x - sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (above < need && need <= above + c[e]) { found[0] = 255 - 4 * lane - e; found[1] = need - above; }
                above += c[e];
            }
        }
        __syncthreads();
        prefix = prefix << 8 | found[0];
        need = found[1];
    }
    // in row order: of the rows with that key the first `need` stay
    uint32_t equal = 0, holes = 0, sources = 0;
    for (uint32_t i0 = 0; i0 < n; i0 += EVICT_THREADS * EVICT_VPT) {
        const uint32_t first = i0 + tid * EVICT_VPT;
        uint32_t k[EVICT_VPT], eq = 0;
#pragma unroll
        for (uint32_t e = 0; e < EVICT_VPT; ++e) {
            k[e] = first + e < n ? key(first + e) : 0u;
            eq += first + e < n && k[e] == prefix;
        }
        uint32_t all, rank = equal + block_scan(eq, wave_sums, all);
        equal += all;
        bool hole[EVICT_VPT], source[EVICT_VPT];
        uint32_t both = 0;                                           // holes in the low half, sources in the high (at most 4096 of each)
#pragma unroll
        for (uint32_t e = 0; e < EVICT_VPT; ++e) {
            const bool there = first + e < n, is = there && k[e] == prefix;
            const bool stays = there && (k[e] > prefix || (is && rank < need));
            rank += is;
            hole[e] = a.in_place && there && !stays && first + e < a.budget;
            source[e] = stays && (!a.in_place || first + e >= a.budget);
            both += (hole[e] ? 1u : 0u) + (source[e] ? 0x10000u : 0u);
        }
        const uint32_t at = block_scan(both, wave_sums, all);
        uint32_t hi = holes + (at & 0xffffu), si = sources + (at >> 16);
#pragma unroll
        for (uint32_t e = 0; e < EVICT_VPT; ++e) {
            if (source[e]) list[1 + si++] = first + e;
            if (hole[e]) list[1 + a.max_moves + hi++] = first + e;
        }
        holes += all & 0xffffu;
        sources += all >> 16;
    }
    if (tid == 0) list[0] = sources;
}

// The listed rows moved, D / 8 lanes to a row.  In place sources lie behind the budget and their places before it, so no row is both.
template <int D>
__global__ __launch_bounds__(256) void cache_evict_move_kernel(const CacheEvictArgs a, uint32_t blocks) {
    constexpr uint32_t LANES = D / 8, ROWS = 256 / LANES;
    const uint32_t pair = blockIdx.x / blocks, blk = blockIdx.x % blocks;
    const uint32_t b = pair / a.kv_heads, h = pair % a.kv_heads, unit = threadIdx.x % LANES;
    const uint32_t* const list = a.moves + (size_t)pair * (1 + 2 * (size_t)a.max_moves);
    const uint32_t n = list[0];
    for (uint32_t m = blk * ROWS + threadIdx.x / LANES; m < n; m += blocks * ROWS) {
        const uint32_t src = list[1 + m], dst = a.in_place ? list[1 + a.max_moves + m] : m;
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
}

template <typename T, int D>
hipError_t launch_weights_of(const CacheWeightsArgs& a, hipStream_t stream) {
    const uint64_t pairs = (uint64_t)a.batch * a.kv_heads, wide = pairs * ((a.max_cached + 127) / 128);
    // Few workgroups and many rows: half the keys to a workgroup, its waves two by two
    if (wide < 512 && a.n_max * a.group > 64) return launch_one(cache_weights_kernel<T, D, 2>, (uint32_t)(pairs * ((a.max_cached + 63) / 64)), 256, stream, a);
    return launch_one(cache_weights_kernel<T, D, 4>, (uint32_t)wide, 256, stream, a);
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

hipError_t launch_cache_evict(const CacheEvictArgs& a, int head_dim, hipStream_t stream) {
    const uint32_t pairs = a.batch * a.kv_heads, rows = 256 / (head_dim / 8);
    hipError_t e = launch_one(cache_evict_select_kernel, pairs, EVICT_THREADS, stream, a);
    if (e != hipSuccess) return e;
    // as many moves as a sequence of max_cached rows makes; the kernel walks any number
    const uint32_t most = a.in_place ? (a.max_cached > a.budget ? a.max_cached - a.budget : 1u) : a.budget;
    uint32_t blocks = (most < a.max_moves ? most : a.max_moves) / rows + 1;
    if (blocks > 256) blocks = 256;
    CacheEvictArgs x = a;
    void* args[] = {&x, &blocks};
    const void* move = head_dim == 128 ? reinterpret_cast<const void*>(cache_evict_move_kernel<128>) : reinterpret_cast<const void*>(cache_evict_move_kernel<64>);
    return hipLaunchKernel(move, dim3(pairs * blocks), dim3(256), args, 0, stream);
}

hipError_t launch_tree_attn(const TreeAttnArgs& a, int dtype, int head_dim, hipStream_t stream) {
    return dtype == 0 ? launch_tree_attn_bf16(a, head_dim, stream) : launch_tree_attn_f16(a, head_dim, stream);
}

}  // namespace depsync
