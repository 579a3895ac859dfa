// Attention of drafted tokens over a cache held in 8 bits: the one pass of tree_attn.hpp over a key axis of two stretches,
//   the rows of full blocks: 8-bit numbers k8, v8 (e4m3) with a scale a block each, so s = (scale log2(e) k_scale) q . k8 and o += (p v_scale) v8,
//   then the rows of 16 bits: those of the block that is not full, which all rows see, and the drafted tokens, by the tree,
// cut into parts and joined as there.  8-bit numbers are exact in both 16-bit types, so products go by the matrix cores in those; the K scale goes into
// the factor of the scores, which is one number a tile of 32 keys as blocks are multiples of 32 rows, and the V scale into the weights.
#pragma once
#include <hip/hip_runtime.h>

#include "tree_attn.hpp"

namespace depsync {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

// The two stretches of a sequence: `cached` rows of full blocks; `drafted` rows of 16 bits, of which `held` are cached ones.
__device__ __forceinline__ TreeLengths tree_lengths(const TreeAttn8Args& a, uint32_t b) {
    const uint32_t n = clamp_count(a.cached[b], a.capacity), held = n & ((1u << a.block_log2) - 1u);
    return {n - held, held + (a.drafted ? clamp_count(a.drafted[b], a.tokens) : a.tokens), held};
}

// Two of four 8-bit numbers as numbers of T.
template <typename T> struct Held8;
template <> struct Held8<__bf16> {
    typedef __bf16 T2 __attribute__((ext_vector_type(2)));
    template <bool HIGH> static __device__ __forceinline__ T2 two(uint32_t x) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, HIGH); }
};
template <> struct Held8<_Float16> {
    typedef _Float16 T2 __attribute__((ext_vector_type(2)));
    template <bool HIGH> static __device__ __forceinline__ T2 two(uint32_t x) { return __builtin_bit_cast(T2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, HIGH)); }
};
// Eight of them, in order.
template <typename T> __device__ __forceinline__ typename Mma<T>::V8 eight(uint32_t lo, uint32_t hi) {
    const auto a = Held8<T>::template two<false>(lo), b = Held8<T>::template two<true>(lo), c = Held8<T>::template two<false>(hi), d = Held8<T>::template two<true>(hi);
    return {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 16 x 16 outputs, 32 products each.
__device__ __forceinline__ f32x4 mma16(Mma<__bf16>::V8 a, Mma<__bf16>::V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(Mma<_Float16>::V8 a, Mma<_Float16>::V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Row r of the stretch of 16 bits (null: there is none).
template <typename T>
__device__ __forceinline__ const T* wide_row(const TreeAttn8Args& a, const TreeJob& j, bool values, uint32_t r) {
    if (r >= j.drafted) return nullptr;
    if (r < j.held)
        return (const T*)(values ? a.v_tail : a.k_tail) + (int64_t)j.b * a.tail_s.batch + (int64_t)r * a.tail_s.token + (int64_t)j.h * a.tail_s.head;
    return (const T*)(values ? a.v_new : a.k_new) + (int64_t)j.b * a.new_s.batch + (int64_t)(r - j.held) * a.new_s.token + (int64_t)j.h * a.new_s.head;
}

// The keys of a run of up to 32 in that stretch, from `first` on, that token t sees.
__device__ __forceinline__ uint32_t wide_bits(const TreeAttn8Args& a, const TreeJob& j, uint32_t t, uint32_t first, uint32_t n) {
    if (n == 0) return 0u;
    const uint32_t there = n >= 32 ? ~0u : (1u << n) - 1u;
    const uint32_t held = first < j.held ? min(32u, j.held - first) : 0u;      // of the run's: seen by all
    const uint32_t all = held >= 32 ? ~0u : (1u << held) - 1u;
    if (held >= n) return there;
    const uint32_t d0 = first + held - j.held, left = n - held;               // the run's first drafted token, and how many
    uint32_t bits;
    if (!a.tree) {
        bits = t < d0 ? 0u : t - d0 >= 31 ? ~0u : (2u << (t - d0)) - 1u;
    } else {
        const uint32_t words = (a.tokens + 63) / 64;
        const uint32_t* const w = (const uint32_t*)(a.tree + (int64_t)j.b * a.tree_batch + (int64_t)t * words);
        const uint32_t at = d0 >> 5, by = d0 & 31u;
        const uint32_t lo = w[at], hi = by + left > 32 ? w[at + 1] : 0u;      // (the words end behind the last token)
        bits = (uint32_t)(((uint64_t)hi << 32 | lo) >> by);
    }
    return there & (all | (held < 32 ? bits << held : 0u));
}

// Values of that stretch that are not finite were multiplied as zeros; they are added to the sums of the rows that see them.
template <typename T>
__device__ __forceinline__ f32x4 add_wide_not_finite(const TreeAttn8Args& a, const TreeJob& j, uint32_t block_keys, uint32_t t, uint32_t d, f32x4 o) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (j.end <= j.cache_blocks) return o;
    const uint32_t first = (max(j.begin, j.cache_blocks) - j.cache_blocks) * block_keys, last = min(j.drafted, (j.end - j.cache_blocks) * block_keys);
    for (uint32_t k0 = first; k0 < last; k0 += 32)
        for (uint32_t bits = wide_bits(a, j, t, k0, min(32u, last - k0)); bits; bits &= bits - 1) {
            const T4 x = *(const T4*)(wide_row<T>(a, j, true, k0 + (uint32_t)__builtin_ctz(bits)) + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = (float)x[e];
                if (!(fabsf(v) < INFINITY)) o[e] += v;
            }
        }
    return o;
}

// Rows of a tile's output, rounded and stored or left for the second kernel.  (The stretch of 16 bits counts cached rows that tokens do not.)
template <typename T, int D>
__device__ __forceinline__ void store8_row4(const TreeAttn8Args& a, const TreeJob& j, uint32_t r, uint32_t d, f32x4 o, float m, float l, bool odd, uint32_t block_keys) {
    if (r >= a.rows) return;
    const uint32_t t = r / a.group;
    if (t >= j.drafted - j.held) return;
    if (__builtin_expect(odd, 0)) o = add_wide_not_finite<T>(a, j, block_keys, t, d, o);
    store_row4<T, D>(a, j, r, d, o, m, l, false, block_keys);
}

// ---- few rows ------------------------------------------------------------------------------------------------------------
// 16 NR rows to a workgroup, the keys in blocks of 128 of which each of the four waves walks 32 by itself.  Keys and values go from memory into the registers that the matrix
// cores read, without LDS: which 8 of a row's numbers a lane holds for a product of 32, and which d an output row is, is free as long as both operands
// agree, so that
//   K: a lane holds 16 consecutive bytes of one row, two fragments of the scores' products (queries are read in the same order);
//   V: a lane holds D / 16 consecutive bytes of each of 8 rows, a fragment of as many 16-row blocks of the output (block b's row m is d = D / 16 m + b);
//      pairs of rows are brought together byte by byte, and converted.
// The next two tiles are on their way meanwhile.
template <typename T, int D, int NR>
__global__ __launch_bounds__(256, 2) void tree_attn8_few(const TreeAttn8Args a) {
    using V8 = typename Mma<T>::V8;
    using B8 = Mma<__bf16>::V8;
    constexpr uint32_t ROWS = 16 * NR, PITCH = D + 4;
    constexpr int NJ = D / 64, NB = D / 16, VW = D / 64;               // 16-byte runs of a K row, blocks of 16 d, words of a V row that a lane holds
    __shared__ __align__(16) float join[4][ROWS][PITCH];
    __shared__ float ml[4][ROWS][2];
    __shared__ uint32_t odd;                                           // a value of the stretch of 16 bits is not finite
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uni(tid >> 6), n = lane & 15u, g = lane >> 4;
    const TreeUnit u = tree_unit((a.rows + ROWS - 1) / ROWS);
    if (u.unit >= a.slots * a.kv_heads) return;
    const TreeJob j = tree_job(a, u.unit, TREE_FEW_KEYS);
    const uint32_t r0 = u.row_block * ROWS;
    if (j.n_parts == 0 || j.begin >= j.end || r0 / a.group >= j.drafted - j.held) return;
    if (tid == 0) odd = 0;
    // ---- the rows of full blocks ----
    const uint32_t pitch = uni((uint32_t)a.cache_s.token);             // bytes
    const uint32_t first = uni(j.begin * TREE_FEW_KEYS + wave * 32);
    const uint32_t end8 = min(j.end, j.cache_blocks);
    const uint32_t tiles = uni(first >= j.cached || j.begin >= end8 ? 0u : min(end8 - j.begin, (j.cached - first + TREE_FEW_KEYS - 1) / TREE_FEW_KEYS));
    const int64_t base = (int64_t)j.b * a.cache_s.batch + (int64_t)j.h * a.cache_s.head + (int64_t)first * pitch;
    const char* const kp = uni_ptr((const char*)a.k_cache + base);
    const char* const vp = uni_ptr((const char*)a.v_cache + base);
    const size_t scales = ((size_t)j.b * a.kv_heads + j.h) * a.n_blocks;
    const float* const ksp = (const float*)uni_ptr(a.k_scale + scales);
    const float* const vsp = (const float*)uni_ptr(a.v_scale + scales);
    struct Tile8 { u32x4 k[2][NJ]; uint32_t v[8][VW]; float ks, vs; } buf[2];
    const uint32_t kat = n * pitch + 16 * g, vat = 4 * g * pitch + (D / 16) * n, bytes = uni(31 * pitch + D);
    auto fetch_k = [&](Tile8& x, uint32_t t) __attribute__((always_inline)) {
        const OperandBuf K(kp + (uint64_t)t * TREE_FEW_KEYS * pitch, t < tiles ? bytes : 0u);   // (behind the last: zeros)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int jj = 0; jj < NJ; ++jj) x.k[kt][jj] = K.load16(kat, kt * 16 * pitch + 64 * jj);
        const uint32_t at = min((first + t * TREE_FEW_KEYS) >> a.block_log2, a.n_blocks - 1);
        x.ks = ksp[at];
        x.vs = vsp[at];
    };
    auto fetch_v = [&](Tile8& x, uint32_t t) __attribute__((always_inline)) {
        const OperandBuf V(vp + (uint64_t)t * TREE_FEW_KEYS * pitch, t < tiles ? bytes : 0u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t row = (i < 4 ? i : 12 + i) * pitch;
            if constexpr (VW == 2) {
                const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(V.rsrc, vat, row, 0);
                x.v[i][0] = w[0]; x.v[i][1] = w[1];
            } else {
                x.v[i][0] = __builtin_amdgcn_raw_buffer_load_b32(V.rsrc, vat, row, 0);
            }
        }
    };
    if (tiles) {
        fetch_k(buf[0], 0); fetch_v(buf[0], 0);
        fetch_k(buf[1], 1); fetch_v(buf[1], 1);
    }
    V8 qf[NR][2 * NJ];
    uint32_t token[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const uint32_t at = r0 + 16 * r + n;
        token[r] = min(at, a.rows - 1) / a.group;
        const T* const q = query_row<T>(a, j, at);
#pragma unroll
        for (int f = 0; f < 2 * NJ; ++f) qf[r][f] = q ? *(const V8*)(q + 64 * (f / 2) + 16 * g + 8 * (f % 2)) : V8{};
    }
    f32x4 o[NR][NB];
    float m[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        m[r] = -INFINITY; l[r] = 0.0f;
#pragma unroll
        for (int b = 0; b < NB; ++b) o[r][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const float sc = a.scale;
    // Weights of a tile's scores, times `vs`, as two fragments of products with values of U, which hold twice the bits of one.
    auto weigh = [&]<typename U>(f32x4 (&st)[2], int r, float by, float vs, typename Mma<U>::V8& high, typename Mma<U>::V8& rest) __attribute__((always_inline)) {
        float mx = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])), fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3]))) * by;
        if (__ballot(mx > m[r] + WEIGHT_SLACK)) {                      // (rarely, after the first steps)
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m[r], mx);
            const float alpha = m[r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[r] - m_new);
            m[r] = m_new;
            l[r] *= alpha;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 4; ++v) o[r][b][v] *= alpha;
        }
        const float ref = (m[r] == -INFINITY ? 0.0f : m[r]) - WEIGHT_OFF<T>;   // no key seen yet: keep the exponents finite
#pragma unroll
        for (int v = 0; v < 8; v += 2) {
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[v >> 2][v & 3], by, -ref));
            const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[v >> 2][(v & 3) + 1], by, -ref));
            l[r] += p0 + p1;
            const WeightPair<U> w(p0 * vs, p1 * vs);
            high[v] = w.high[0]; high[v + 1] = w.high[1];
            rest[v] = w.rest[0]; rest[v + 1] = w.rest[1];
        }
    };
    auto step = [&](Tile8& x, uint32_t t) __attribute__((always_inline)) {
        f32x4 st[NR][2] = {};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int f = 0; f < 2 * NJ; ++f) {
                const V8 k = eight<T>(x.k[kt][f / 2][2 * (f % 2)], x.k[kt][f / 2][2 * (f % 2) + 1]);
#pragma unroll
                for (int r = 0; r < NR; ++r) st[r][kt] = mma16(k, qf[r][f], st[r][kt]);
            }
        const float by = sc * x.ks, vs = x.vs;
        fetch_k(x, t + 2);
        B8 high[NR], rest[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) weigh.template operator()<__bf16>(st[r], r, by, vs, high[r], rest[r]);
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            B8 vf[4];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint32_t lo = __builtin_amdgcn_perm(x.v[i + 1][w], x.v[i][w], 0x05010400u), hi = __builtin_amdgcn_perm(x.v[i + 1][w], x.v[i][w], 0x07030602u);
                const auto y0 = Held8<__bf16>::two<false>(lo), y1 = Held8<__bf16>::two<true>(lo), y2 = Held8<__bf16>::two<false>(hi), y3 = Held8<__bf16>::two<true>(hi);
#pragma unroll
                for (int e = 0; e < 2; ++e) { vf[0][i + e] = y0[e]; vf[1][i + e] = y1[e]; vf[2][i + e] = y2[e]; vf[3][i + e] = y3[e]; }
            }
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    o[r][4 * w + b] = mma16(vf[b], high[r], o[r][4 * w + b]);
                    o[r][4 * w + b] = mma16(vf[b], rest[r], o[r][4 * w + b]);
                }
        }
        fetch_v(x, t + 2);
    };
    for (uint32_t t = 0; t < tiles; t += 2) {
        step(buf[0], t);
        if (t + 1 < tiles) step(buf[1], t + 1);
    }
    // ---- the rows of 16 bits ----
    __syncthreads();                                                   // (odd is 0)
    for (uint32_t blk = max(j.begin, j.cache_blocks); blk < j.end; ++blk) {
        const uint32_t at = (blk - j.cache_blocks) * TREE_FEW_KEYS + wave * 32;
        if (at >= j.drafted) break;
        const uint32_t there = min(32u, j.drafted - at);
        f32x4 st[NR][2] = {};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const T* const k = wide_row<T>(a, j, false, at + 16 * kt + n);
#pragma unroll
            for (int f = 0; f < 2 * NJ; ++f) {
                const V8 kf = k ? *(const V8*)(k + 64 * (f / 2) + 16 * g + 8 * (f % 2)) : V8{};
#pragma unroll
                for (int r = 0; r < NR; ++r) st[r][kt] = mma16(kf, qf[r][f], st[r][kt]);
            }
        }
        V8 high[NR], rest[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const uint32_t vis = wide_bits(a, j, token[r], at, there);
#pragma unroll
            for (int v = 0; v < 8; ++v)
                if (!(vis >> (16 * (v >> 2) + 4 * g + (v & 3)) & 1u)) st[r][v >> 2][v & 3] = -INFINITY;
            weigh.template operator()<T>(st[r], r, sc, 1.0f, high[r], rest[r]);
        }
        uint32_t vw[8][NB / 2];                                        // NB numbers of 8 rows each
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const T* const v = wide_row<T>(a, j, true, at + 4 * g + (i < 4 ? i : 12 + i));
            u32x4 x = {0, 0, 0, 0};
            if (v) {
                if constexpr (NB == 8) x = *(const u32x4*)(v + NB * n);
                else { const u32x2 y = *(const u32x2*)(v + NB * n); x[0] = y[0]; x[1] = y[1]; }
            }
            bad |= without_not_finite<T>(x);
#pragma unroll
            for (int w = 0; w < NB / 2; ++w) vw[i][w] = x[w];
        }
        if (bad) odd = 1;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            u32x4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_perm(vw[2 * i + 1][b / 2], vw[2 * i][b / 2], b % 2 ? 0x07060302u : 0x05040100u);
            const V8 vf = __builtin_bit_cast(V8, y);
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                o[r][b] = mma16(vf, high[r], o[r][b]);
                o[r][b] = mma16(vf, rest[r], o[r][b]);
            }
        }
    }
    // ---- the four waves joined ----
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        l[r] += __shfl_xor(l[r], 16);
        l[r] += __shfl_xor(l[r], 32);
        if (g == 0) { ml[wave][16 * r + n][0] = m[r]; ml[wave][16 * r + n][1] = l[r]; }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, ml[w][16 * r + n][0]);
        const float f = m[r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[r] - M);
        const bool none = m[r] == -INFINITY && l[r] == 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int b = 0; b < NB; b += 4) {                          // d = NB (4 g + v) + b
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = none ? 0.0f : o[r][b + e][v] * f;
                *(f32x4*)&join[wave][16 * r + n][NB * (4 * g + v) + b] = x;
            }
    }
    __syncthreads();
    const TreeAttn8Args& late = tree_args<TreeAttn8Args>();
    constexpr uint32_t TPR = 256 / ROWS;                               // threads to a row
    const uint32_t rr = tid / TPR;
    float mm = -INFINITY, L = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, ml[w][rr][0]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float mw = ml[w][rr][0], lw = ml[w][rr][1];
        L += mw == -INFINITY ? lw : lw * __builtin_amdgcn_exp2f(mw - mm);         // (a sum without a maximum is 0, or NaN)
    }
#pragma unroll
    for (uint32_t d = (tid % TPR) * 4; d < D; d += TPR * 4) {
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) x += *(const f32x4*)&join[w][rr][d];
        store8_row4<T, D>(late, j, r0 + rr, d, x, mm, L, odd != 0, TREE_FEW_KEYS);
    }
}

template <typename T, int D>
hipError_t launch_tree_attn8_of(const TreeAttn8Args& a, hipStream_t stream) {
    const uint32_t units = (a.slots * a.kv_heads + 7) / 8 * 8;
    hipError_t e;
    if (a.rows <= 16) e = launch_one(tree_attn8_few<T, D, 1>, units, 256, stream, a);
    else e = launch_one(tree_attn8_few<T, D, 2>, units * ((a.rows + 31) / 32), 256, stream, a);
    if (e != hipSuccess || a.slots == a.batch) return e;
    return launch_one(tree_attn_join<T, D, TreeAttn8Args>, (uint32_t)(((uint64_t)a.batch * a.kv_heads * a.rows + 3) / 4), 256, stream, a);
}

template <typename T>
hipError_t launch_tree_attn8_type(const TreeAttn8Args& a, int head_dim, hipStream_t stream) {
    return head_dim == 128 ? launch_tree_attn8_of<T, 128>(a, stream) : launch_tree_attn8_of<T, 64>(a, stream);
}

}  // namespace depsync
