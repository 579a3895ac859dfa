// Accepted keys and values appended to a cache of 8 bits.
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "tree_attn.hpp"

namespace depsync {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// The scale of a block by the bits of its largest finite magnitude: 2^e, the smallest from 2^-126 on with magnitude <= 448 2^e = 1.75 2^(e + 8).  A power
// of two, as the numbers are floating point ones: none loses bits to the division, and quantising gives the same numbers however it is computed.
struct BlockScale {
    float scale, inverse;
    __device__ __forceinline__ explicit BlockScale(float largest) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, largest);
        const int32_t e = max((int32_t)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
        scale = bits ? __builtin_bit_cast(float, (uint32_t)(e + 127) << 23) : 0.0f;
        inverse = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
    }
};

// Four numbers in 8 bits, to nearest, ties to even.  What is not finite: the largest number of its sign, and NaN.
__device__ __forceinline__ float within(float y) { return fabsf(y) == INFINITY ? copysignf(448.0f, y) : y; }
__device__ __forceinline__ uint32_t e4m3_of(float a, float b, float c, float d) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(within(a), within(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(within(c), within(d), x, true);
}

// A workgroup to a sequence, head, K or V, and a block that the call can fill.  Bound by latency: lengths, the row's number, the row and the search are behind one another (one to
// six accepted rows of 32 sequences: 4.6 us; 4 x 1024 tokens of 8 heads in blocks of 32, 26 MB: 8.3, 3.1 TB/s, 2048 workgroups that all start at once).  Its rows stay in registers between the search for the largest magnitude
// and the conversion, so they are read once.  The workgroup of the first block reads the rows held in 16 bits, which the rows behind the last full block
// overwrite: that workgroup writes these too, afterwards.
template <typename T, int D, int BLOCK>
__global__ __launch_bounds__(256) void cache_append8_kernel(const CacheAppend8Args a) {
    constexpr uint32_t LANES = D / 8, RPP = 256 / LANES, PASSES = (BLOCK + RPP - 1) / RPP;
    constexpr uint16_t INF = __is_same(T, __bf16) ? 0x7f80 : 0x7c00;
    __shared__ uint32_t largest[4];
    uint32_t x = blockIdx.x;
    const uint32_t i = x % a.most_full; x /= a.most_full;
    const uint32_t is_v = x & 1u; x >>= 1;
    const uint32_t h = x % a.kv_heads, b = x / a.kv_heads;
    const uint32_t cached = clamp_count(a.cached[b], a.capacity);
    const uint32_t n = min(a.n_accepted ? clamp_count(a.n_accepted[b], a.n_max) : a.n_max, a.capacity - cached);
    const uint32_t end = cached + n, first = cached / BLOCK, last = end / BLOCK;
    if (blockIdx.x % (a.most_full * a.kv_heads * 2) == 0 && threadIdx.x == 0) {
        a.cached_out[b] = (int32_t)end;
        if (a.n_out) a.n_out[b] = (int32_t)n;
    }
    const uint32_t row0 = threadIdx.x / LANES, unit = threadIdx.x % LANES;
    const uint16_t* const fresh = (const uint16_t*)(is_v ? a.v_new : a.k_new) + (int64_t)b * a.new_s.batch + (int64_t)h * a.new_s.head;
    uint16_t* const held = (uint16_t*)(is_v ? a.v_tail : a.k_tail) + (int64_t)b * a.tail_s.batch + (int64_t)h * a.tail_s.head;
    auto new_row = [&](uint32_t r) __attribute__((always_inline)) {      // of the sequence's row r
        const uint32_t at = r - cached, t = a.accepted ? clamp_count(a.accepted[(size_t)b * a.n_max + at], a.tokens - 1) : at;
        return ((const u32x4*)(fresh + (int64_t)t * a.new_s.token))[unit];
    };
    const uint32_t blk = first + i;
    if (blk < last) {
        u32x4 raw[PASSES];
        uint32_t top = 0;                                                // bits of the largest finite magnitude
#pragma unroll
        for (uint32_t p = 0; p < PASSES; ++p) {
            const uint32_t slot = p * RPP + row0, r = blk * BLOCK + slot;
            raw[p] = slot >= BLOCK ? u32x4{0, 0, 0, 0} : r < cached ? ((const u32x4*)(held + (int64_t)slot * a.tail_s.token))[unit] : new_row(r);
        }
#pragma unroll
        for (uint32_t p = 0; p < PASSES; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = (raw[p][e >> 1] >> (16 * (e & 1))) & 0x7fffu;
                top = max(top, m < INF ? m : 0u);
            }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
        if ((threadIdx.x & 63u) == 0) largest[threadIdx.x >> 6] = top;
        __syncthreads();
        top = max(max(largest[0], largest[1]), max(largest[2], largest[3]));
        const BlockScale s((float)__builtin_bit_cast(T, (uint16_t)top));
        if (threadIdx.x == 0) (is_v ? a.v_scale : a.k_scale)[((size_t)b * a.kv_heads + h) * a.n_blocks + blk] = s.scale;
        uint8_t* const to = (uint8_t*)(is_v ? a.v_cache : a.k_cache) + (int64_t)b * a.cache_s.batch + (int64_t)h * a.cache_s.head;
#pragma unroll
        for (uint32_t p = 0; p < PASSES; ++p) {
            const uint32_t slot = p * RPP + row0;
            if (slot >= BLOCK) continue;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (float)__builtin_bit_cast(T, (uint16_t)(raw[p][e >> 1] >> (16 * (e & 1)))) * s.inverse;
            const u32x2 bits = {e4m3_of(y[0], y[1], y[2], y[3]), e4m3_of(y[4], y[5], y[6], y[7])};
            ((u32x2*)(to + (int64_t)(blk * BLOCK + slot) * a.cache_s.token))[unit] = bits;
        }
    }
    if (i != 0) return;
    for (uint32_t r = max(cached, last * BLOCK) + row0; r < end; r += RPP) {
        const u32x4 bits = new_row(r);
        ((u32x4*)(held + (int64_t)(r - last * BLOCK) * a.tail_s.token))[unit] = bits;
    }
}

template <typename T, int D>
hipError_t launch_append8_of(const CacheAppend8Args& a, int block, hipStream_t stream) {
    const uint32_t n = a.batch * a.kv_heads * 2 * a.most_full;
    if (block == 32) return launch_one(cache_append8_kernel<T, D, 32>, n, 256, stream, a);
    if (block == 64) return launch_one(cache_append8_kernel<T, D, 64>, n, 256, stream, a);
    return launch_one(cache_append8_kernel<T, D, 128>, n, 256, stream, a);
}

}  // namespace

hipError_t launch_cache_append8(const CacheAppend8Args& a, int dtype, int head_dim, int block, hipStream_t stream) {
    if (dtype == 0) return head_dim == 128 ? launch_append8_of<__bf16, 128>(a, block, stream) : launch_append8_of<__bf16, 64>(a, block, stream);
    return head_dim == 128 ? launch_append8_of<_Float16, 128>(a, block, stream) : launch_append8_of<_Float16, 64>(a, block, stream);
}

}  // namespace depsync
