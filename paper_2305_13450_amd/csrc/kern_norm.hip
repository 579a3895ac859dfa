// Norms of queries and keys for each head, with the rotation by their positions.
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "tree_attn.hpp"

namespace depsync {

namespace {

// cos and sin of a turn's fraction x / 2^32.  The nearest quarter is taken off in whole numbers; what is left, |z| <= pi / 4, goes into the
// series of both up to z^8 and z^9, whose first terms left out are below 2.5e-8 and 2e-9.
__device__ __forceinline__ void turn(uint32_t x, float& c, float& s) {
    const uint32_t quarter = (x + 0x20000000u) >> 30;
    const float z = (float)(int32_t)(x - (quarter << 30)) * (6.2831853071795865f / 4294967296.0f), w = z * z;
    float p = __builtin_fmaf(w, 1.0f / 362880.0f, -1.0f / 5040.0f), q = __builtin_fmaf(w, 1.0f / 40320.0f, -1.0f / 720.0f);
    p = __builtin_fmaf(w, p, 1.0f / 120.0f);
    p = __builtin_fmaf(w, p, -1.0f / 6.0f);
    p = __builtin_fmaf(w * p, z, z);
    q = __builtin_fmaf(w, q, 1.0f / 24.0f);
    q = __builtin_fmaf(w, q, -0.5f);
    q = __builtin_fmaf(w, q, 1.0f);
    c = quarter & 1u ? p : q;
    s = quarter & 1u ? q : p;
    if (quarter == 1u || quarter == 2u) c = -c;
    if (quarter & 2u) s = -s;
}

// Sum over the LANES lanes (a power of two up to 8) that hold a row, in all of them.
template <int LANES> __device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

// A wave takes 8 heads of 128 numbers (16 of 64) of one token, queries or keys.  A lane holds two runs of 8 numbers of a head that are each other's partners
// (8 u and 8 u + rotary_dim / 2; interleaved, and behind rotary_dim: 16 u and 16 u + 8), D / 16 lanes to a head, so no number crosses lanes but the sum of
// squares.  Bound by HBM, read and written once: 4 x 2048 tokens of 64 + 8 heads of 128, 302 MB, in 53 us warm and 57 to 62 in turn with others, 5 TB/s as a copy; the eight angles of a lane are worked
// out anew by each of a token's 9 waves meanwhile.  What L2 cannot hold for the next kernel is stored past it (inputs that change, 302 MB: 68 and 66 us, 84 MB: 22 and 20).  One token of 32 sequences: 4.4 us, four loads behind one another.
template <typename T, int D, bool INTERLEAVED, bool NORM, bool STREAMS>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const QkNormArgs a) {
    constexpr uint32_t LANES = D / 16, HEADS = 64 / LANES;
    typedef T T8 __attribute__((ext_vector_type(8)));
    const uint32_t lane = threadIdx.x & 63u, unit = lane % LANES;
    const uint32_t waves = a.q_waves + a.k_waves;
    const uint64_t wave = (uint64_t)blockIdx.x * 4 + uni(threadIdx.x >> 6);
    const uint32_t token = (uint32_t)(wave / waves), part = (uint32_t)(wave % waves);
    const uint32_t b = token / a.tokens, t = token % a.tokens;
    if (b >= a.batch || (a.drafted && t >= clamp_count(a.drafted[b], a.tokens))) return;
    const bool keys = part >= a.q_waves;
    const uint32_t heads = keys ? a.kv_heads : a.heads;
    const Strides &from_s = keys ? a.k_s : a.q_s, &to_s = keys ? a.k_out_s : a.q_out_s;
    const T* const from = (const T*)(keys ? a.k : a.q) + (int64_t)b * from_s.batch + (int64_t)t * from_s.token;
    T* const to = (T*)(keys ? a.k_out : a.q_out) + (int64_t)b * to_s.batch + (int64_t)t * to_s.token;
    const bool rotated = unit < a.rotary_dim / 16;
    const uint32_t e0 = !INTERLEAVED && rotated ? 8 * unit : 16 * unit, e1 = !INTERLEAVED && rotated ? e0 + a.rotary_dim / 2 : e0 + 8;
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { cs[i] = 1.0f; sn[i] = 0.0f; }
    if (rotated) {
        const int64_t pos = (int64_t)(a.start ? a.start[b] : 0) + (a.depth ? a.depth[(int64_t)b * a.depth_batch + t] : (int32_t)t);
#pragma unroll
        for (int i = 0; i < 8; ++i) turn((uint32_t)(((uint64_t)pos * a.freq[8 * unit + i]) >> 32), cs[i], sn[i]);
    }
    float gain[2][8];
    const float* const g = keys ? a.k_gain : a.q_gain;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const f32x4 x = g ? *(const f32x4*)(g + (c ? e1 : e0) + 4 * v) : f32x4{1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i) gain[c][4 * v + i] = x[i];
        }
    const uint32_t h = (keys ? part - a.q_waves : part) * HEADS + lane / LANES;
    T8 in[2] = {};
    if (h < heads) {
        in[0] = *(const T8*)(from + (int64_t)h * from_s.head + e0);
        in[1] = *(const T8*)(from + (int64_t)h * from_s.head + e1);
    }
    float x[2][8], sum = 0.0f;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[c][i] = (float)in[c][i];
            sum = __builtin_fmaf(x[c][i], x[c][i], sum);
        }
    float f = 1.0f;
    if constexpr (NORM) f = 1.0f / sqrtf(__builtin_fmaf(row_sum<LANES>(sum), 1.0f / D, a.eps));
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] *= f * gain[c][i];
    T8 out[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int ca = INTERLEAVED ? i / 4 : 0, ia = INTERLEAVED ? 2 * (i % 4) : i, cb = INTERLEAVED ? ca : 1, ib = INTERLEAVED ? ia + 1 : i;
        const float u = x[ca][ia], v = x[cb][ib];
        out[ca][ia] = (T)__builtin_fmaf(u, cs[i], rotated ? -v * sn[i] : 0.0f);   // (numbers behind rotary_dim are no pairs: one that is not finite stays alone)
        out[cb][ib] = (T)__builtin_fmaf(v, cs[i], rotated ? u * sn[i] : 0.0f);
    }
    if (h >= heads) return;
    T8 *const to0 = (T8*)(to + (int64_t)h * to_s.head + e0), *const to1 = (T8*)(to + (int64_t)h * to_s.head + e1);
    if constexpr (STREAMS) {                                           // (two branches' stores, alike but for their way, would become one)
        __builtin_nontemporal_store(out[0], to0);
        __builtin_nontemporal_store(out[1], to1);
    } else {
        *to0 = out[0];
        *to1 = out[1];
    }
}

template <typename T, int D, bool INTERLEAVED, bool NORM>
hipError_t launch_norm_with(const QkNormArgs& a, bool streams, hipStream_t stream) {
    const uint64_t waves = (uint64_t)a.batch * a.tokens * (a.q_waves + a.k_waves);
    const uint32_t n = (uint32_t)((waves + 3) / 4);
    return streams ? launch_one(qk_norm_rope_kernel<T, D, INTERLEAVED, NORM, true>, n, 256, stream, a) : launch_one(qk_norm_rope_kernel<T, D, INTERLEAVED, NORM, false>, n, 256, stream, a);
}
template <typename T, int D>
hipError_t launch_norm_of(const QkNormArgs& a, bool interleaved, bool norm, bool streams, hipStream_t stream) {
    if (interleaved) return norm ? launch_norm_with<T, D, true, true>(a, streams, stream) : launch_norm_with<T, D, true, false>(a, streams, stream);
    return norm ? launch_norm_with<T, D, false, true>(a, streams, stream) : launch_norm_with<T, D, false, false>(a, streams, stream);
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkNormArgs& a, int dtype, int head_dim, bool interleaved, bool norm, bool streams, hipStream_t stream) {
    if (dtype == 0) return head_dim == 128 ? launch_norm_of<__bf16, 128>(a, interleaved, norm, streams, stream) : launch_norm_of<__bf16, 64>(a, interleaved, norm, streams, stream);
    return head_dim == 128 ? launch_norm_of<_Float16, 128>(a, interleaved, norm, streams, stream) : launch_norm_of<_Float16, 64>(a, interleaved, norm, streams, stream);
}

}  // namespace depsync
