// Attention of drafted tokens over a cache held in 8 bits: the one pass of tree_attn.hpp over a key axis of two stretches,
//   the rows of full blocks: 8-bit numbers k8, v8 (e4m3) with a scale a block each, so s = (scale log2(e) k_scale) q . k8 and o += (p v_scale) v8,
//   then the rows of 16 bits: those of the block that is not full, which all rows see, and the drafted tokens, by the tree,
// cut into parts and joined as there.  8-bit numbers are exact in both 16-bit types, so products go by the matrix cores in those; the K scale goes into
// the factor of the scores, which is one number a tile of 32 keys as blocks are multiples of 32 rows, and the V scale into the weights.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "tree_attn.hpp"

namespace depsync {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// The two stretches of a sequence: `cached` rows of full blocks; `drafted` rows of 16 bits, of which the first are `held` cached ones and room up to a multiple of
// 32, so that a tile of 32 keys is of one array.
__device__ __forceinline__ uint32_t held_room(uint32_t held) { return (held + 31u) & ~31u; }
__device__ __forceinline__ TreeLengths tree_lengths(const TreeAttn8Args& a, uint32_t b) {
    const uint32_t n = clamp_count(a.cached[b], a.capacity), held = n & ((1u << a.block_log2) - 1u);
    return {n - held, held_room(held) + (a.drafted ? clamp_count(a.drafted[b], a.tokens) : a.tokens), held};
}
__device__ __forceinline__ uint32_t tokens_of(const TreeJob& j) { return j.drafted - held_room(j.held); }

template <typename V> __device__ __forceinline__ void swapped(V& a, V& b) { const V x = a; a = b; b = x; }

// As tree_unit, but 2^together units that follow one another, heads of one sequence, run on one XCD: rows of 64 bytes share cache lines of 128 with their
// neighbours' (4 tokens of 8 heads of 64 over 120001 rows: 47 us, and 36 so; where rows fill their lines it makes no difference to few rows, and 4 x 256 tokens
// took 620 us for 518, the heads of the longest sequence being on fewer XCDs).
__device__ __forceinline__ TreeUnit tree_unit8(uint32_t row_blocks, uint32_t together) {
    const uint32_t slot = blockIdx.x >> 3, n = slot / row_blocks;
    return {(((n >> together) * 8 + (blockIdx.x & 7u)) << together) + (n & ((1u << together) - 1u)), slot % row_blocks};
}

constexpr uint32_t NOWHERE = 1u << 31;   // an offset behind the end of any tile: nothing is read, and zeros come

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

// The scales of a sequence's and head's blocks, as scalar loads take them: by vector loads every wait for one was a wait for all keys on their way.
typedef const __attribute__((address_space(4))) float* Scales;
__device__ __forceinline__ Scales scales_at(const float* p, size_t at) { return (Scales)(uint64_t)uni_ptr(p + at); }

// a / b, of scales.  (The inverse of one beyond 2^126 is no normal number, and would come out as 0.)
__device__ __forceinline__ float quotient(float a, float b) {
    const float k = b > 0x1p64f ? 0x1p-64f : 1.0f;
    return a * k * __builtin_amdgcn_rcpf(b * k);
}

// 16 x 16 outputs, 32 products each.
__device__ __forceinline__ f32x4 mma16(Mma<__bf16>::V8 a, Mma<__bf16>::V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(Mma<_Float16>::V8 a, Mma<_Float16>::V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// The tile of 32 keys at `at` of the stretch of 16 bits: where its rows lie, how far apart, and how many there are.
struct WideRun {
    const char *k, *v;
    uint32_t step;       // bytes
    uint32_t first, n;   // among the rows held or the drafted tokens
    bool held;
};
template <int D>
__device__ __forceinline__ WideRun wide_run(const TreeAttn8Args& a, const TreeJob& j, uint32_t at) {
    WideRun x;
    const uint32_t room = held_room(j.held);
    x.held = at < room;
    x.first = at - (x.held ? 0u : room);
    const uint32_t have = x.held ? j.held : j.drafted - room;
    x.n = x.first < have ? min(32u, have - x.first) : 0u;
    const Strides& s = x.held ? a.tail_s : a.new_s;
    const int64_t off = ((int64_t)j.b * s.batch + (int64_t)x.first * s.token + (int64_t)j.h * s.head) * 2;
    x.k = (const char*)(x.held ? a.k_tail : a.k_new) + off;
    x.v = (const char*)(x.held ? a.v_tail : a.v_new) + off;
    x.step = (uint32_t)s.token * 2u;
    return x;
}
template <int D> __device__ __forceinline__ uint32_t wide_bytes(const WideRun& x) { return x.n ? (x.n - 1) * x.step + D * 2u : 0u; }

// The keys of such a tile that token t sees: rows held are seen by all.
__device__ __forceinline__ uint32_t wide_bits(const TreeAttn8Args& a, const TreeJob& j, const WideRun& x, uint32_t t) {
    if (x.held) return x.n >= 32 ? ~0u : (1u << x.n) - 1u;
    return tree_bits(a, j.b, t, x.first, x.n);
}

// Values of that stretch that are not finite were multiplied as zeros; they are added to the sums of the rows that see them.
template <typename T, int D>
__device__ __forceinline__ f32x4 add_wide_not_finite(const TreeAttn8Args& a, const TreeJob& j, uint32_t block_keys, uint32_t t, uint32_t d, f32x4 o) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (j.end <= j.cache_blocks) return o;
    const uint32_t first = (max(j.begin, j.cache_blocks) - j.cache_blocks) * block_keys, last = min(j.drafted, (j.end - j.cache_blocks) * block_keys);
    for (uint32_t k0 = first; k0 < last; k0 += 32) {
        const WideRun run = wide_run<D>(a, j, k0);
        for (uint32_t bits = wide_bits(a, j, run, t); bits; bits &= bits - 1) {
            const T4 x = *(const T4*)(run.v + (uint64_t)__builtin_ctz(bits) * run.step + d * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = (float)x[e];
                if (!(fabsf(v) < INFINITY)) o[e] += v;
            }
        }
    }
    return o;
}

// Rows of a tile's output, rounded and stored or left for the second kernel.  (The stretch of 16 bits counts cached rows that tokens do not.)
template <typename T, int D>
__device__ __forceinline__ void store8_row4(const TreeAttn8Args& a, const TreeJob& j, uint32_t r, uint32_t d, f32x4 o, float m, float l, bool odd, uint32_t block_keys) {
    if (r >= a.rows) return;
    const uint32_t t = r / a.group;
    if (t >= tokens_of(j)) return;
    if (__builtin_expect(odd, 0)) o = add_wide_not_finite<T, D>(a, j, block_keys, t, d, o);
    store_row4<T, D>(a, j, r, d, o, m, l, false, block_keys);
}

// ---- few rows ------------------------------------------------------------------------------------------------------------
// 16 NR rows to a workgroup, the keys in blocks of 128 of which each of the four waves walks 32 by itself, with the next one or two tiles on their way into registers.  They come in runs
// that fill cache lines (a load of a wave is 1 KB of whole rows): a CU that is nearly alone reads 90 GB/s so, where rows fetched as the matrix cores take them, 64 and 128 bytes
// a row and load, came at 45.  Through LDS of its own a wave then reads them in fragments.  Which 8 of a row's numbers a lane holds for a product of 32,
// and which d an output row is, is free as long as both operands agree, so that
//   K: a lane reads 16 consecutive bytes of one row, two fragments of the scores' products (queries are held in the same order);
//   V: a lane reads D / 16 consecutive bytes of each of 8 rows, a fragment of as many 16-row blocks of the output (block b's row m is d = D / 16 m + b);
//      pairs of rows are brought together byte by byte, and converted.
template <typename T, int D, int NR>
__global__ __launch_bounds__(256, 2) void tree_attn8_few(const TreeAttn8Args a) {
    using V8 = typename Mma<T>::V8;
    using B8 = Mma<__bf16>::V8;
    constexpr uint32_t ROWS = 16 * NR, PITCH = D + 4;
    constexpr int NJ = D / 64, NB = D / 16, VW = D / 64;               // 16-byte runs of a K row, blocks of 16 d, words of a V row that a lane holds
    constexpr uint32_t WAVE = 64 * D > ROWS * PITCH * 4 ? 64 * D : ROWS * PITCH * 4;
    __shared__ __align__(16) char lds[4 * WAVE];                       // a wave's tile, and its results at the end
    __shared__ float ml[4][ROWS][2];
    __shared__ uint32_t odd;                                           // a value of the stretch of 16 bits is not finite
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uni(tid >> 6), n = lane & 15u, g = lane >> 4;
    const TreeUnit u = tree_unit8((a.rows + ROWS - 1) / ROWS, a.together);
    if (u.unit >= a.slots * a.kv_heads) return;
    const TreeJob j = tree_job(a, u.unit, TREE_FEW_KEYS);
    const uint32_t r0 = u.row_block * ROWS;
    if (j.n_parts == 0 || j.begin >= j.end || r0 / a.group >= tokens_of(j)) return;
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
    const Scales ksp = scales_at(a.k_scale, scales), vsp = scales_at(a.v_scale, scales);
    constexpr uint32_t CHUNKS = D / 16, RPI = 64 / CHUNKS, NI = 32 / RPI;   // 16-byte chunks of a row, rows of a load, loads of a tile
    constexpr uint32_t AHEAD = NR == 2 && D == 128 ? 1 : 2;            // tiles on their way (two spill registers there)
    struct Tile8 { u32x4 k[NI], v[NI]; float ks, vs; } buf[AHEAD];
    const uint32_t lrow = lane / CHUNKS, chunk = lane % CHUNKS, bytes = uni(31 * pitch + D);
    auto fetch = [&](Tile8& x, uint32_t t) __attribute__((always_inline)) {
        const uint64_t at = (uint64_t)t * TREE_FEW_KEYS * pitch;
        const OperandBuf K(kp + at, bytes), V(vp + at, bytes);
        const uint32_t off = t < tiles ? lrow * pitch + chunk * 16 : NOWHERE;
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) x.k[i] = K.load16(off, i * RPI * pitch);
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) x.v[i] = V.load16(off, i * RPI * pitch);
        const uint32_t block = uni(min((first + t * TREE_FEW_KEYS) >> a.block_log2, a.n_blocks - 1));
        x.ks = ksp[block];
        x.vs = vsp[block];
    };
    // A row's chunks lie in LDS at exclusive-ors of their number and the row's, by which the lanes that read or write together find different banks.
    auto swz8 = [](uint32_t row) __attribute__((always_inline)) { return D == 128 ? row & 7u : (row >> 1) & 3u; };
    char* const ldsK = lds + wave * WAVE;
    char* const ldsV = ldsK + 32 * D;
    const uint32_t put = lrow * D + ((chunk ^ swz8(lrow)) << 4), kat = n * D + ((g ^ swz8(n)) << 4);
    const uint32_t vat = 4 * g * D + (((n * D / 256) ^ swz8(4 * g)) << 4) + (n * (D / 16) & 15u);
    if (tiles) {
#pragma unroll
        for (uint32_t i = 0; i < AHEAD; ++i) fetch(buf[i], i);
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
    // Weights of a tile's scores, times its V scale, as two fragments of products with values of U, which hold twice the bits of one.  The scale goes into the exponent, and
    // the sum is divided by it again (both off by the same rounding); but a scale so small or large that weights or their sum would fall out of 32 bits is multiplied afterwards.
    auto weigh = [&](f32x4 (&st)[2], int r, float by, float vs, auto held, auto& high, auto& rest) __attribute__((always_inline)) {
        using U = std::conditional_t<std::is_same_v<std::remove_reference_t<decltype(high)>, B8>, __bf16, _Float16>;
        constexpr bool HELD = decltype(held)::value;                   // a tile of 8 bits: with a scale, and without infinities
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
        float ref = (m[r] == -INFINITY ? 0.0f : m[r]) - WEIGHT_OFF<T>;   // no key seen yet: keep the exponents finite
        const bool far = HELD && uni(vs < 0x1p-60f || vs > 0x1p60f ? 1u : 0u);
        float back = 1.0f;
        if (HELD && !far) {
            back = __builtin_amdgcn_rcpf(vs);
            ref += __builtin_amdgcn_logf(back);
        }
        float p[8], sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[v >> 2][v & 3], by, -ref));
            sum[v & 1] += p[v];
        }
        l[r] = __builtin_fmaf(sum[0] + sum[1], back, l[r]);
        if (__builtin_expect(far, 0))
#pragma unroll
            for (int v = 0; v < 8; ++v) p[v] *= vs;
#pragma unroll
        for (int v = 0; v < 8; v += 2) {
            const WeightPair<U> w(p[v], p[v + 1], !HELD);
            high[v] = w.high[0]; high[v + 1] = w.high[1];
            rest[v] = w.rest[0]; rest[v + 1] = w.rest[1];
        }
    };
    auto step = [&](Tile8& x, uint32_t t) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) *(u32x4*)(ldsK + put + i * 1024) = x.k[i];
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) *(u32x4*)(ldsV + put + i * 1024) = x.v[i];
        const float by = sc * x.ks, vs = x.vs;
        fetch(x, t + AHEAD);
        asm volatile("" ::: "memory");                                 // (a wave's LDS accesses keep their order)
        __builtin_amdgcn_wave_barrier();
        u32x4 kr[2][NJ];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int jj = 0; jj < NJ; ++jj) kr[kt][jj] = *(const u32x4*)(ldsK + (kat ^ (64 * jj)) + kt * 16 * D);
        uint32_t vr[8][VW];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t row = i < 4 ? i : 12 + i;                   // behind 4 g, whose low bits it leaves alone
            const char* const p = ldsV + (vat ^ (swz8(row) << 4)) + row * D;
            if constexpr (VW == 2) {
                const u32x2 w = *(const u32x2*)p;
                vr[i][0] = w[0]; vr[i][1] = w[1];
            } else {
                vr[i][0] = *(const uint32_t*)p;
            }
        }
        f32x4 st[NR][2] = {};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int f = 0; f < 2 * NJ; ++f) {
                const V8 k = eight<T>(kr[kt][f / 2][2 * (f % 2)], kr[kt][f / 2][2 * (f % 2) + 1]);
#pragma unroll
                for (int r = 0; r < NR; ++r) st[r][kt] = mma16(k, qf[r][f], st[r][kt]);
            }
        B8 high[NR], rest[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) weigh(st[r], r, by, vs, std::true_type{}, high[r], rest[r]);
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            B8 vf[4];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint32_t lo = __builtin_amdgcn_perm(vr[i + 1][w], vr[i][w], 0x05010400u), hi = __builtin_amdgcn_perm(vr[i + 1][w], vr[i][w], 0x07030602u);
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
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    };
    for (uint32_t t = 0; t < tiles; t += AHEAD) {
        step(buf[0], t);
        if constexpr (AHEAD == 2)
            if (t + 1 < tiles) step(buf[1], t + 1);
    }
    // ---- the rows of 16 bits ----
    __syncthreads();                                                   // (odd is 0)
    for (uint32_t blk = max(j.begin, j.cache_blocks); blk < j.end; ++blk) {
        const uint32_t at = (blk - j.cache_blocks) * TREE_FEW_KEYS + wave * 32;
        if (at >= j.drafted) break;
        const WideRun run = wide_run<D>(a, j, at);
        const OperandBuf K(uni_ptr(run.k), uni(wide_bytes<D>(run))), V(uni_ptr(run.v), uni(wide_bytes<D>(run)));   // rows that are not there: zeros
        u32x4 kf[2][2 * NJ];                                           // everything is asked for before anything is waited for
        uint32_t vw[8][NB / 2];                                        // NB numbers of 8 rows each
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int f = 0; f < 2 * NJ; ++f) kf[kt][f] = K.load16((16 * kt + n) * run.step + 32 * g + 128 * (f / 2) + 16 * (f % 2), 0);   // (rows' ends count offsets of lanes)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t off = (4 * g + (i < 4 ? i : 12 + i)) * run.step + 2 * NB * n;
            if constexpr (NB == 8) {
                const u32x4 x = V.load16(off, 0);
#pragma unroll
                for (int w = 0; w < 4; ++w) vw[i][w] = x[w];
            } else {
                const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(V.rsrc, off, 0, 0);
                vw[i][0] = x[0]; vw[i][1] = x[1];
            }
        }
        f32x4 st[NR][2] = {};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int f = 0; f < 2 * NJ; ++f)
#pragma unroll
                for (int r = 0; r < NR; ++r) st[r][kt] = mma16(__builtin_bit_cast(V8, kf[kt][f]), qf[r][f], st[r][kt]);
        V8 high[NR], rest[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const uint32_t vis = wide_bits(a, j, run, token[r]);
#pragma unroll
            for (int v = 0; v < 8; ++v)
                if (!(vis >> (16 * (v >> 2) + 4 * g + (v & 3)) & 1u)) st[r][v >> 2][v & 3] = -INFINITY;
            weigh(st[r], r, sc, 1.0f, std::false_type{}, high[r], rest[r]);
        }
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u32x4 x = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < NB / 2; ++w) x[w] = vw[i][w];
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
                *(f32x4*)((float*)(lds + wave * WAVE) + (16 * r + n) * PITCH + NB * (4 * g + v) + b) = x;
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
        for (int w = 0; w < 4; ++w) x += *(const f32x4*)((const float*)(lds + w * WAVE) + rr * PITCH + d);
        store8_row4<T, D>(late, j, r0 + rr, d, x, mm, L, odd != 0, TREE_FEW_KEYS);
    }
}

// ---- many rows -----------------------------------------------------------------------------------------------------------
// The form for many rows of tree_attn.hpp: 128 rows to a workgroup, tiles of 32 keys in LDS, where they are numbers of T: 8-bit ones are converted on their way from
// registers into it, once for all four waves (16 conversions and 4 LDS stores a wave and tile, where a wave that converted its fragments would need 64).
//
// Weights of these tiles and their values go into the products as fp16 numbers whatever T is: 8-bit values are exact in it, and its three bits more than bf16 has leave outputs
// as near to 64 bits as with 32-bit weights (4 x 256 tokens in bf16: 1.7e-3 of their norm, the output's own rounding; 2.1e-3 with bf16 weights), in the same
// time.  Tiles of 16 bits keep to T.
//
// A weight carries its block's V scale, relative to one that the part has met (`most`; outputs are in units of it, and are scaled when it changes), so that fp16 weights
// stay in range: the scale goes into the exponent, and the sum is divided by it again.  `most` follows where a block's scale is larger, or less than 2^-8 of it, which random scales
// come to a few times.  (With the largest one kept as the unit, a row that saw blocks of small values alone had weights of few bits: a V scale of 2^-29 of it left 4.)
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void tree_attn8_many(const TreeAttn8Args a) {
    using Tile = KeyTile<T, D>;
    using Mm = Mma<T>;
    using V8 = typename Mm::V8;
    using H = Mma<_Float16>;
    using H8 = H::V8;
    typedef _Float16 T4 __attribute__((ext_vector_type(4)));
    constexpr bool MIXED = !std::is_same_v<T, _Float16>;               // tiles of 16 bits are of another type
    constexpr float OFF = WEIGHT_OFF<_Float16>;
    using Pad = PaddedTile<D>;
    constexpr uint32_t SLOT = Pad::BYTES;                              // a tile of K and one of V
    constexpr int KF = D / 16, NB = D / 32, NV = 2 * NB, AHEAD = 3;    // MFMAs of a tile's scores, of its output (as many), LDS reads ahead of them
    __shared__ __align__(16) char lds[4 * SLOT];
    __shared__ __align__(8) uint32_t tile_scales[4][2];                // of the tile in each slot
    __shared__ uint32_t odd;                                           // a value of the stretch of 16 bits is not finite
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uni(tid >> 6), h2 = lane >> 5;
    const TreeUnit u = tree_unit8((a.rows + TREE_MANY_ROWS - 1) / TREE_MANY_ROWS, a.together);
    if (u.unit >= a.slots * a.kv_heads) return;
    const TreeJob j = tree_job(a, u.unit, TREE_MANY_KEYS);
    const uint32_t r0 = u.row_block * TREE_MANY_ROWS, t_last = (min(r0 + TREE_MANY_ROWS, a.rows) - 1) / a.group;
    if (j.n_parts == 0 || j.begin >= j.end || r0 / a.group >= tokens_of(j)) return;
    // without a tree nothing behind the block's last token is seen
    const uint32_t end = a.tree ? j.end : min(j.end, max(j.begin, j.cache_blocks + (held_room(j.held) + t_last) / TREE_MANY_KEYS + 1));
    constexpr uint32_t NI = Tile::NI / 4;                              // 1 KB copies of a wave: 32 rows of 16 bits over four waves
    const uint32_t lrow = wave * (Tile::RPI * NI) + lane / Tile::CHUNKS, chunk = lane % Tile::CHUNKS;
    const uint32_t row8 = tid >> 3, at8 = (tid & 7u) * (D / 8);        // of a tile of 8 bits: a thread's row, and its D / 8 bytes of it
    const uint32_t pitch = uni((uint32_t)a.cache_s.token);
    const int64_t base = (int64_t)j.b * a.cache_s.batch + (int64_t)j.h * a.cache_s.head;
    const char *const kbase = uni_ptr((const char*)a.k_cache + base), *const vbase = uni_ptr((const char*)a.v_cache + base);
    const size_t scales = ((size_t)j.b * a.kv_heads + j.h) * a.n_blocks;
    const OperandBuf KS(uni_ptr(a.k_scale + scales), a.n_blocks * 4u), VS(uni_ptr(a.v_scale + scales), a.n_blocks * 4u);
    // A tile on its way: of 8 bits the first D / 8 bytes of k[0] and v[0] (D = 64: of h), else all of k and v.
    struct Staged { u32x4 k[NI], v[NI]; u32x2 h[2]; uint32_t ks, vs; } staged[2];
    auto load8 = [&](Staged& f, const OperandBuf& K, const OperandBuf& V, uint32_t off, uint32_t scale) __attribute__((always_inline)) {
        if constexpr (D == 128) {
            f.k[0] = K.load16(off, 0);
            f.v[0] = V.load16(off, 0);
        } else {
            f.h[0] = __builtin_amdgcn_raw_buffer_load_b64(K.rsrc, off, 0, 0);
            f.h[1] = __builtin_amdgcn_raw_buffer_load_b64(V.rsrc, off, 0, 0);
        }
        f.ks = __builtin_amdgcn_raw_buffer_load_b32(KS.rsrc, scale, 0, 0);
        f.vs = __builtin_amdgcn_raw_buffer_load_b32(VS.rsrc, scale, 0, 0);
    };
    auto fetch8 = [&](Staged& f, uint32_t tile) __attribute__((always_inline)) {
        const uint64_t at = (uint64_t)tile * TREE_MANY_KEYS * pitch;
        const uint32_t bytes = tile < end ? 31 * pitch + D : 0u;       // (behind the last: zeros)
        load8(f, OperandBuf(kbase + at, bytes), OperandBuf(vbase + at, bytes), row8 * pitch + at8, (tile * TREE_MANY_KEYS >> a.block_log2) * 4);
    };
    // Of either kind, without a branch around loads: behind one each of the first four tiles was waited for before the next was asked for (3 us).
    auto fetch = [&](const TreeAttn8Args& args, Staged& f, uint32_t tile) __attribute__((always_inline)) {
        const bool wide = tile >= j.cache_blocks;
        const WideRun run = wide_run<D>(args, j, (tile - j.cache_blocks) * TREE_MANY_KEYS);
        const uint64_t at = (uint64_t)tile * TREE_MANY_KEYS * pitch;
        const uint32_t bytes = uni(tile >= end ? 0u : wide ? wide_bytes<D>(run) : 31 * pitch + D);
        const OperandBuf K(uni_ptr(wide ? run.k : kbase + at), bytes), V(uni_ptr(wide ? run.v : vbase + at), bytes);
        const uint32_t off8 = row8 * pitch + at8, off16 = wide ? lrow * run.step + chunk * 16 : NOWHERE;
        load8(f, K, V, D == 128 && wide ? off16 : wide ? NOWHERE : off8, wide ? NOWHERE : (tile * TREE_MANY_KEYS >> a.block_log2) * 4);
#pragma unroll
        for (uint32_t i = D == 128 ? 1 : 0; i < NI; ++i) {
            const uint32_t off = wide ? off16 + i * Tile::RPI * run.step : NOWHERE;   // (rows' ends count offsets of lanes)
            f.k[i] = K.load16(off, 0);
            f.v[i] = V.load16(off, 0);
        }
    };
    auto put8 = [&](const Staged& f, uint32_t slot) __attribute__((always_inline)) {
        char* const to = lds + (slot & 3u) * SLOT + at8 * 2;
#pragma unroll
        for (uint32_t i = 0; i < D / 64; ++i) {
            u32x2 k, v;
            if constexpr (D == 128) { k = u32x2{f.k[0][2 * i], f.k[0][2 * i + 1]}; v = u32x2{f.v[0][2 * i], f.v[0][2 * i + 1]}; }
            else { k = f.h[0]; v = f.h[1]; }
            *(V8*)(to + row8 * Pad::K_PITCH + 16 * i) = eight<T>(k[0], k[1]);
            *(H8*)(to + row8 * Pad::V_PITCH + Pad::K_BYTES + 16 * i) = eight<_Float16>(v[0], v[1]);
        }
        if (tid < 1) *(u32x2*)tile_scales[slot & 3u] = u32x2{f.ks, f.vs};
    };
    auto put = [&](Staged& f, uint32_t tile) __attribute__((always_inline)) {
        const uint32_t slot = tile - j.begin;
        if (tile < j.cache_blocks) {
            put8(f, slot);
        } else {
            bool bad = false;
            char* const to = lds + (slot & 3u) * SLOT + chunk * 16;
#pragma unroll
            for (uint32_t i = 0; i < NI; ++i) {
                u32x4 v = f.v[i];
                bad |= without_not_finite<T>(v);
                *(u32x4*)(to + lrow * Pad::K_PITCH + i * Tile::RPI * Pad::K_PITCH) = f.k[i];
                *(u32x4*)(to + lrow * Pad::V_PITCH + Pad::K_BYTES + i * Tile::RPI * Pad::V_PITCH) = v;
            }
            if (bad) odd = 1;
            const uint32_t one = __builtin_bit_cast(uint32_t, 1.0f);
            if (tid < 1) *(u32x2*)tile_scales[slot & 3u] = u32x2{one, one};
        }
    };
    if (tid == 0) odd = 0;
    // V of the tile before the first, whose weights are zeros: in slot 3
    for (uint32_t i = tid; i < 32 * Pad::V_PITCH / 16; i += 256) *(u32x4*)(lds + 3 * SLOT + Pad::K_BYTES + i * 16) = u32x4{0, 0, 0, 0};
    __syncthreads();
    fetch(a, staged[0], j.begin);
    fetch(a, staged[1], j.begin + 1);
    put(staged[0], j.begin);
    fetch(a, staged[0], j.begin + 2);
    put(staged[1], j.begin + 1);
    fetch(a, staged[1], j.begin + 3);
    RowState<D> row;
    clear_row(row);
    const uint32_t at = r0 + wave * 32 + (lane & 31u), token = min(at, a.rows - 1) / a.group;
    V8 qf[KF];
    {
        const T* const q = query_row<T>(a, j, at);
        const V8 zero = {};
#pragma unroll
        for (int kk = 0; kk < KF; ++kk) qf[kk] = q ? *(const V8*)(q + kk * 16 + h2 * 8) : zero;
    }
    const uint32_t koff = (lane & 31u) * Pad::K_PITCH + h2 * 16;
    const uint32_t voff = Pad::K_BYTES + (4 * h2 + ((lane & 15u) >> 2)) * Pad::V_PITCH + ((lane >> 4) & 1u) * 32 + (lane & 3u) * 8;
    auto read_k = [&](const char* slot, int i) __attribute__((always_inline)) { return *(const u32x4*)(slot + koff + i * 32); };
    auto read_v = [&](const char* slot, int i) __attribute__((always_inline)) {   // slice i / NB of 16 keys, block i % NB of 32 d
        T4 x[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) x[c] = TrRead<_Float16>::read(slot + voff + ((i / NB) * 16 + c * 8) * Pad::V_PITCH + (i % NB) * 64);
        return __builtin_bit_cast(u32x4, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // a product of weights and values, of T where both are of a tile of 16 bits
    auto weighted = [&](auto wide, const u32x4& v, const u32x4& p, const f32x16& o) __attribute__((always_inline)) {
        if constexpr (MIXED && decltype(wide)::value) return Mm::mma(__builtin_bit_cast(V8, v), __builtin_bit_cast(V8, p), o);
        else return H::mma(__builtin_bit_cast(H8, v), __builtin_bit_cast(H8, p), o);
    };
    f32x16 st[2];
    u32x4 pf[2][2] = {};
    const float sc = a.scale;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 16; ++v) st[0][v] = 0.0f;                      // scores of the first tile
#pragma unroll
    for (int i = 0; i < KF; ++i) st[0] = Mm::mma(__builtin_bit_cast(V8, read_k(lds, i)), qf[i], st[0]);
    auto largest = [&](const f32x16& x) __attribute__((always_inline)) {
        float m0 = fmaxf(fmaxf(x[0], x[1]), x[2]), m1 = fmaxf(fmaxf(x[3], x[4]), x[5]);
        m0 = fmaxf(fmaxf(m0, x[6]), x[7]); m1 = fmaxf(fmaxf(m1, x[8]), x[9]);
        m0 = fmaxf(fmaxf(m0, x[10]), x[11]); m1 = fmaxf(fmaxf(m1, x[12]), x[13]);
        return fmaxf(fmaxf(fmaxf(m0, x[14]), x[15]), m1);
    };
    float top = largest(st[0]);                                        // of this lane's scores of the tile to be weighed
    // Scales of the tile to be weighed, read from LDS while the one before is.
    float ks, vs, most = 0.0f, peak = 0.0f;                             // (the unit, and the largest V scale so far)
    auto scales_of = [&](uint32_t slot) __attribute__((always_inline)) {
        const u32x2 x = *(const u32x2*)tile_scales[slot & 3u];
        const uint32_t k = x[0], v = x[1];
        ks = __builtin_bit_cast(float, k);
        vs = __builtin_bit_cast(float, v);
    };
    scales_of(0);
    // Of the V scale `of` (its bits): the logarithm of what it is of `most`, and the inverse.  What is below 2^-60 of the largest counts for nothing, so outputs stay in 32 bits
    // in whatever unit.
    // Rows of 16 bits have no scale that says how large they are, so `most` is 1 for them (2^-60 of the largest if that is more, for the same reason).
    uint32_t of = ~0u, none = 0;
    float off = 0.0f, back = 1.0f;
    // Weights of the tile whose scores are in `sx`, into `px`; scores of the next tile (in slot `next`) into `sy`, and their largest; output of the
    // one before (in slot `before`) with `py`.
    // wide: whether these tiles are of 16 bits.
    auto segment = [&](auto wide, f32x16& sx, u32x4 (&px)[2], f32x16& sy, const u32x4 (&py)[2], const char* next, const char* before, bool masked, uint32_t vis)
                       __attribute__((always_inline)) {
        using W = std::conditional_t<MIXED && decltype(wide)::value, T, _Float16>;
        typedef W W8 __attribute__((ext_vector_type(8)));
        W8 weights[2];
        u32x4 fr[AHEAD + 1];                                              // fragments on their way
        auto rd = [&](int i) __attribute__((always_inline)) { fr[i % (AHEAD + 1)] = i < KF ? read_k(next, i) : read_v(before, i - KF); };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) rd(i);
        if (masked) {
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (!(vis >> (8 * (v / 4) + 4 * h2 + v % 4) & 1u)) sx[v] = -INFINITY;
            top = largest(sx);
        }
        float alpha = 1.0f, unit = 1.0f;
        uint32_t moved = 0;
        if (uni(__builtin_bit_cast(uint32_t, vs)) != of) {             // (once a block)
            of = uni(__builtin_bit_cast(uint32_t, vs));
            if (!wide) peak = fmaxf(peak, vs);
            const float u = wide ? fmaxf(1.0f, peak * 0x1p-60f) : vs;
            none = uni(!wide && (vs < 0x1p-126f || vs < peak * 0x1p-60f) ? 1u : 0u);
            moved = uni((wide ? u != most : !none && (u > most || u < most * 0x1p-8f)) ? 1u : 0u);
            if (moved) { unit = quotient(most, u); most = u; }
            back = none ? 1.0f : quotient(most, vs);                     // (off by the reciprocal's rounding, as off then is)
            off = none ? 0.0f : -__builtin_amdgcn_logf(back);
        }
        const float by = sc * ks, mx = max_halves(top) * by;
        const bool grown = __ballot(mx > row.m + WEIGHT_SLACK) != 0;         // (rarely, after the first steps)
        if (grown) {
            const float m_new = fmaxf(row.m, mx);
            alpha = row.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(row.m - m_new);
            row.m = m_new;
            row.l *= alpha;
        }
        const float ref = (row.m == -INFINITY ? 0.0f : row.m) - OFF - off;   // no key seen yet: keep the exponents finite
        float sum[2] = {0.0f, 0.0f}, x0 = 0.0f, x1 = 0.0f, m0 = -INFINITY, m1 = -INFINITY;
        auto weigh = [&](int v, int half) __attribute__((always_inline)) {       // scores v and v + 1, in two halves
            if (half == 0) {
                x0 = __builtin_fmaf(sx[v], by, -ref);
                x1 = __builtin_fmaf(sx[v + 1], by, -ref);
                x0 = __builtin_amdgcn_exp2f(x0);
            } else {
                x1 = __builtin_amdgcn_exp2f(x1);
                sum[0] += x0; sum[1] += x1;                            // summed in 32 bits, rounded to 16 for the product with V alone
                weights[v >> 3][v & 7] = (W)x0; weights[v >> 3][(v & 7) + 1] = (W)x1;
            }
        };
#pragma unroll
        for (int v = 0; v < 16; ++v) sy[v] = 0.0f;
#pragma unroll
        for (int i = 0; i < KF + NV; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i + AHEAD < KF + NV) rd(i + AHEAD);
            if (i < KF) sy = Mm::mma(__builtin_bit_cast(V8, fr[i % (AHEAD + 1)]), qf[i], sy);
            else row.o[(i - KF) % NB] = weighted(wide, fr[i % (AHEAD + 1)], py[(i - KF) / NB], row.o[(i - KF) % NB]);
            if constexpr (KF == 8) weigh(i & ~1, i & 1);
            else { weigh(2 * i, 0); weigh(2 * i, 1); }
            constexpr int FIRST = KF + NV - 4;                         // the next scores are there by then: four of them to a slot
            if (i >= FIRST) {
                m0 = fmaxf(fmaxf(m0, sy[4 * (i - FIRST)]), sy[4 * (i - FIRST) + 1]);
                m1 = fmaxf(fmaxf(m1, sy[4 * (i - FIRST) + 2]), sy[4 * (i - FIRST) + 3]);
            }
        }
        px[0] = __builtin_bit_cast(u32x4, weights[0]);
        px[1] = __builtin_bit_cast(u32x4, weights[1]);
        asm volatile("" ::"v"(px[0]), "v"(px[1]), "v"(sum[0]), "v"(sum[1]), "v"(m0), "v"(m1));   // (computed here, and not where they are used)
        __builtin_amdgcn_sched_barrier(0);
        row.l = __builtin_fmaf(sum[0] + sum[1], back, row.l);
        top = fmaxf(m0, m1);
        if (__builtin_expect(none, 0)) px[0] = px[1] = u32x4{0, 0, 0, 0};
        if (grown || moved) {                                          // what was added so far went by the reference value and unit before
            alpha *= unit;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) row.o[b][v] *= alpha;
        }
    };
    // One tile: what it copies goes out two tiles before it is put into LDS, and that is a tile before it is read.
    auto step = [&](auto wide, const TreeAttn8Args& args, uint32_t tile, int odd_one) __attribute__((always_inline)) {
        constexpr bool WIDE = decltype(wide)::value;
        uint32_t vis = ~0u;
        if constexpr (WIDE) {
            const WideRun run = wide_run<D>(args, j, (tile - j.cache_blocks) * TREE_MANY_KEYS);
            vis = tile < end ? wide_bits(args, j, run, token) : 0u;
        }
        const uint32_t slot = tile - j.begin;
        // (behind the last tile the scores are of whatever the slot holds, and not used)
        segment(wide, st[odd_one], pf[odd_one], st[odd_one ^ 1], pf[odd_one ^ 1], lds + ((slot + 1) & 3u) * SLOT, lds + ((slot - 1) & 3u) * SLOT, WIDE, vis);
        scales_of(slot + 1);
        put(staged[odd_one], tile + 2);
        fetch(args, staged[odd_one], tile + 4);
        __syncthreads();                                               // the tile put is in its slot, the one read is done with
    };
    // The output of a tile whose weights are in pf[1].
    auto flush = [&](auto wide, uint32_t tile) __attribute__((always_inline)) {
        const char* const slot = lds + ((tile - j.begin) & 3u) * SLOT;
#pragma unroll
        for (int i = 0; i < NV; ++i) row.o[i % NB] = weighted(wide, read_v(slot, i), pf[1][i / NB], row.o[i % NB]);
    };
    uint32_t tile = j.begin;
    // The bulk: tiles of 8 bits up to the last one fetched, without the general step's branches.
    const uint32_t whole = min(end, j.cache_blocks);
    if (tile + 5 < whole) {
        auto quick = [&](int odd_one, uint32_t slot) __attribute__((always_inline)) {
            segment(std::false_type{}, st[odd_one], pf[odd_one], st[odd_one ^ 1], pf[odd_one ^ 1], lds + ((slot + 1) & 3u) * SLOT, lds + ((slot - 1) & 3u) * SLOT, false, ~0u);
            scales_of(slot + 1);
            put8(staged[odd_one], slot + 2);
            fetch8(staged[odd_one], j.begin + slot + 4);
            __syncthreads();
        };
        for (; tile + 5 < whole; tile += 2) {
            quick(0, tile - j.begin);
            quick(1, tile - j.begin + 1);
        }
    }
    const TreeAttn8Args& later = tree_args<TreeAttn8Args>();
    for (; tile + 1 < whole; tile += 2) {
        step(std::false_type{}, later, tile, 0);
        step(std::false_type{}, later, tile + 1, 1);
    }
    if (tile < whole) {                                                // (an odd one: what follows begins with the registers of the first of two)
        step(std::false_type{}, later, tile, 0);
        ++tile;
        st[0] = st[1];
        pf[1][0] = pf[0][0]; pf[1][1] = pf[0][1];
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) { swapped(staged[0].k[i], staged[1].k[i]); swapped(staged[0].v[i], staged[1].v[i]); }
        if constexpr (D == 64) { swapped(staged[0].h[0], staged[1].h[0]); swapped(staged[0].h[1], staged[1].h[1]); }
        swapped(staged[0].ks, staged[1].ks);
        swapped(staged[0].vs, staged[1].vs);
    }
    if (tile > j.begin) flush(std::false_type{}, tile - 1);
    if (tile < end) {
        pf[1][0] = pf[1][1] = u32x4{0, 0, 0, 0};
        of = ~0u;
        for (; tile < end; tile += 2) {                                // (a last one without keys where their number is odd)
            step(std::true_type{}, later, tile, 0);
            step(std::true_type{}, later, tile + 1, 1);
        }
        flush(std::true_type{}, tile - 1);
    }
    const TreeAttn8Args& last_args = tree_args<TreeAttn8Args>();
    static_assert(OFF - (MIXED ? 0.0f : OFF) == (MIXED ? 9.0f : 0.0f), "as LESS has it");
    constexpr float LESS = MIXED ? 0x1p-9f : 1.0f;               // (weights carry 2^OFF, and in T 2^WEIGHT_OFF<T>)
    row.l = (row.l + __shfl_xor(row.l, 32)) * LESS;
    most *= LESS;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = row.o[b][4 * g + e] * most;
            store8_row4<T, D>(last_args, j, at, 32 * b + 8 * g + 4 * h2, o, row.m, row.l, odd != 0, TREE_MANY_KEYS);
        }
}

template <typename T, int D>
hipError_t launch_tree_attn8_of(const TreeAttn8Args& a, hipStream_t stream) {
    const uint32_t at_once = 8u << a.together, units = (a.slots * a.kv_heads + at_once - 1) / at_once * at_once;
    hipError_t e;
    if (!a.few) e = launch_one(tree_attn8_many<T, D>, units * ((a.rows + TREE_MANY_ROWS - 1) / TREE_MANY_ROWS), 256, stream, a);
    else if (a.rows <= 16) e = launch_one(tree_attn8_few<T, D, 1>, units, 256, stream, a);
    else e = launch_one(tree_attn8_few<T, D, 2>, units * ((a.rows + 31) / 32), 256, stream, a);
    if (e != hipSuccess || a.slots == a.batch) return e;
    return launch_one(tree_attn_join<T, D, TreeAttn8Args>, (uint32_t)(((uint64_t)a.batch * a.kv_heads * a.rows + 3) / 4), 256, stream, a);
}

template <typename T>
hipError_t launch_tree_attn8_type(const TreeAttn8Args& a, int head_dim, hipStream_t stream) {
    return head_dim == 128 ? launch_tree_attn8_of<T, 128>(a, stream) : launch_tree_attn8_of<T, 64>(a, stream);
}

}  // namespace depsync
