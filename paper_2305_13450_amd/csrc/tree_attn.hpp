// Attention of drafted tokens over a cache: for every key and value head, rows = tokens x query heads that share it,
//   o_r = sum_k p_rk v_k / sum_k p_rk,   p_rk = exp2(s_rk - m_r),   s_rk = scale log2(e) q_r . k_k
// over the sequence's cached rows and those drafted tokens that the row's tree word names, in one pass over the keys with
// a reference value m (a maximum that may lag), sum and un-normalised output per row.  All scores are computed transposed, as in attn_tile.hpp: a lane
// owns one query row, S^T = K Q^T leaves 16 of 32 keys of it in its registers, and these are the B operand of O^T += V^T P^T as they stand.
//
// The key axis is the cached rows in blocks, then the drafted tokens in blocks; a block never mixes the two.  Where there are few (sequence,
// head) pairs on 256 CUs it is cut into parts of equally many blocks, one workgroup each.  Parts leave their
// maxima, sums and un-normalised outputs in the workspace and a second kernel joins them in order, so results do not depend on timing.
#pragma once
#include <hip/hip_runtime.h>

#include "attn_tile.hpp"
#include "cache_ops.h"
#include "gemm_tile.hpp"

namespace depsync {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// The reference value that weights are relative to follows the running maximum only where that has grown by more than SLACK (base 2): with 32 rows
// to a wave every third step of 500 would rescale the outputs for the sake of some row's new maximum, so hardly one in thirty does.
// Weights are then at most 2^SLACK, at which 16-bit ones are no coarser: their error is relative.  But fp16 has 2^-14 to 2^16 only, and the weights of a
// long cache are mostly far below the largest, so there they carry a factor of 2^OFF, 2^15 at most: below the reference 23 binades keep all bits.
// Sums and outputs carry the factor alike and it cancels.
constexpr float WEIGHT_SLACK = 6.0f;
template <typename T> constexpr float WEIGHT_OFF = 0.0f;
template <> inline constexpr float WEIGHT_OFF<_Float16> = 9.0f;

// Zeros in the place of infinities and NaN; whether there were any.  Two values at a time: what is added carries an exponent of all ones into the sign's
// place, and that bit becomes 16 (comparisons kept 128 scalar registers of conditions).
template <typename T> __device__ __forceinline__ bool without_not_finite(u32x4& v) {
    constexpr uint32_t ONE = __is_same(T, __bf16) ? 0x00800080u : 0x04000400u;   // 1 in the exponents
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t m = ((v[i] & 0x7fff7fffu) + ONE) & 0x80008000u;
        bad |= m;
        v[i] &= ~((m << 1) - (m >> 15));
    }
    return bad != 0;
}

__device__ __forceinline__ uint32_t clamp_count(int32_t v, uint32_t most) { return v < 0 ? 0u : min((uint32_t)v, most); }

// What one 32-key tile of K and of V looks like in LDS, and a lane's offsets into it.
template <typename T, int D> struct KeyTile {
    static constexpr uint32_t PITCH = D * 2, CHUNKS = D / 8, BYTES = 32 * PITCH;
    static constexpr uint32_t RPI = 1024 / PITCH, NI = 32 / RPI;       // rows and number of a wave's 1 KB copies
    // Position of a row's 16-byte chunk: K fragments are a chunk of 32 rows, V fragments (transposing reads) 64 bytes of 4
    // consecutive rows; either way the lanes that read together find different banks.
    static __device__ __forceinline__ uint32_t kswz(uint32_t row) { return D == 128 ? row & 15u : swz(row); }
    static __device__ __forceinline__ uint32_t vswz(uint32_t row) { return D == 128 ? att_vswz(row) : ((row & 2u) << 1) | ((row >> 2) & 3u); }
    static __device__ __forceinline__ uint32_t koff(uint32_t lane) { return (lane & 31u) * PITCH + (((lane >> 5) ^ kswz(lane & 31u)) << 4); }
    static __device__ __forceinline__ uint32_t voff(uint32_t lane) {
        const uint32_t key = 4u * (lane >> 5) + ((lane & 15u) >> 2);
        return key * PITCH + (((((lane >> 4) & 1u) * 2u + ((lane & 3u) >> 1)) ^ vswz(key)) << 4) + (lane & 1u) * 8u;
    }
};

// A lane's query row: running maximum, un-normalised output (O^T: D / 32 blocks of 32 d, 16 of them per lane), and the sum of the
// weights of this lane's keys (its half of every 32; the halves are added at the end).
template <int D> struct RowState {
    f32x16 o[D / 32];
    float m, l;
};

// A value the compiler computes anew from: offsets derived from it are not kept in registers across a loop's steps.
__device__ __forceinline__ uint32_t opaque(uint32_t x) { asm volatile("" : "+v"(x)); return x; }

// The larger of a value and that of the lane 32 further on.  (The results by name: a bit cast of an element where it stands reads the first.)
__device__ __forceinline__ float max_halves(float x) {
    const auto y = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    const uint32_t lower = y[0], upper = y[1];
    return fmaxf(__builtin_bit_cast(float, lower), __builtin_bit_cast(float, upper));
}

// Two weights for products with 16-bit operands, each as a sum of two numbers of T: the weight cut off, and what that took away, rounded.  Together they are
// off by 2 u^2 of the weight, u being T's half step (fp16: and 2^-24, of weights that carry a factor of 2^9), where one rounded number is off by u.
// Neither is negative, and what was taken away counts for at least 2^-16 of the weight (bf16) or the smallest number (fp16): a zero there would make
// NaN of an infinite value that its row does see.
template <typename T> struct WeightPair {
    typedef T T2 __attribute__((ext_vector_type(2)));
    typedef uint16_t Bits __attribute__((ext_vector_type(2)));
    T2 high, rest;
    // infinite: values may be, so `rest` keeps to that least.
    __device__ __forceinline__ WeightPair(float a, float b, bool infinite = true) {
        Bits least;
        if constexpr (__is_same(T, __bf16)) {
            const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
            high = __builtin_bit_cast(T2, __builtin_amdgcn_perm(y, x, 0x07060302u));
            rest[0] = (T)(a - __builtin_bit_cast(float, x & 0xffff0000u));
            rest[1] = (T)(b - __builtin_bit_cast(float, y & 0xffff0000u));
            least = __builtin_elementwise_sub_sat(__builtin_bit_cast(Bits, high), Bits{16 << 7, 16 << 7});
        } else {
            high = __builtin_bit_cast(T2, __builtin_amdgcn_cvt_pkrtz(a, b));
            rest[0] = (T)(a - (float)high[0]);
            rest[1] = (T)(b - (float)high[1]);
            least = __builtin_elementwise_min(__builtin_bit_cast(Bits, high), Bits{1, 1});
        }
        if (infinite) rest = __builtin_bit_cast(T2, __builtin_elementwise_max(__builtin_bit_cast(Bits, rest), least));
    }
};

// One step: KT tiles of 32 keys in LDS against 32 rows.  vis: the tile's keys that a lane's row sees, one bit each.
// Fragments are read two slices ahead of the MFMAs and the order is pinned: left alone the compiler reads them all at once, and spills, or each right
// before the wait for it.  query(kk): the rows' fragment of slice kk.
// Weights go into the product with V as two numbers each: the time here is that of the keys' way, so keeping their bits costs little (one token over 500 rows
// 11.8 -> 12.8 us, 4 x 2048 rows 13.4 -> 14.4, 32 sequences of up to 8192 139 -> 142), and outputs are as near to 64 bits as with 32-bit weights (bf16: 1.62e-3 of
// their norm, 2.07e-3 with rounded weights; nearly all of the former is the output's own rounding).
template <typename T, int D, int KT, int AHEAD, class Q>
__device__ __forceinline__ void tree_step(RowState<D>& row, Q query, const char* ldsK, const char* ldsV, uint32_t lane, float sc,
                                          const uint32_t (&vis)[KT], bool masked) {
    using Tile = KeyTile<T, D>;
    using M = Mma<T>;
    using V8 = typename M::V8;
    constexpr int KF = D / 16;
    const uint32_t h2 = lane >> 5;
    const uint32_t koff = opaque(Tile::koff(lane)), voff = opaque(Tile::voff(lane));
    f32x16 st[KT];
    {
        V8 kf[AHEAD + 1], qf[AHEAD + 1];
        auto rd = [&](int i) __attribute__((always_inline)) {
            kf[i % (AHEAD + 1)] = *(const V8*)(ldsK + (koff ^ ((i % KF) * 32u)) + (i / KF) * Tile::BYTES);
            qf[i % (AHEAD + 1)] = query(i % KF);
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) rd(i);
#pragma unroll
        for (int i = 0; i < KT * KF; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i + AHEAD < KT * KF) rd(i + AHEAD);
            if (i % KF == 0)
#pragma unroll
                for (int v = 0; v < 16; ++v) st[i / KF][v] = 0.0f;
            st[i / KF] = M::mma(kf[i % (AHEAD + 1)], qf[i % (AHEAD + 1)], st[i / KF]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if (masked) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (!(vis[t] >> (8 * (v / 4) + 4 * h2 + v % 4) & 1u)) st[t][v] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int v = 0; v < 16; v += 2) mx = fmaxf(fmaxf(mx, st[t][v]), st[t][v + 1]);
    mx = max_halves(mx) * sc;
    if (__ballot(mx > row.m + WEIGHT_SLACK)) {                       // (rarely, after the first steps)
        const float m_new = fmaxf(row.m, mx);
        const float alpha = row.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(row.m - m_new);
        row.m = m_new;
        row.l *= alpha;
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) row.o[b][v] *= alpha;
    }
    const float ref = (row.m == -INFINITY ? 0.0f : row.m) - WEIGHT_OFF<T>;   // no key seen yet: keep the exponents finite
    V8 pf[2 * KT], rest[2 * KT];
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
            float p[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][v + e], sc, -ref));
                sum[e] += p[e];
            }
            const WeightPair<T> w(p[0], p[1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) { pf[2 * t + (v >> 3)][(v & 7) + e] = w.high[e]; rest[2 * t + (v >> 3)][(v & 7) + e] = w.rest[e]; }
        }
    row.l += sum[0] + sum[1];
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 vf[AHEAD + 1][2];
    constexpr int NB = D / 32, NV = 2 * KT * NB;
    auto rdv = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
            vf[i % (AHEAD + 1)][c] = TrRead<T>::read(ldsV + (voff ^ ((i % NB) * 64u + c * 32u)) + ((i / NB) * 16 + c * 8) * Tile::PITCH);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) rdv(i);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        if (i + AHEAD < NV) rdv(i + AHEAD);
        const V8 x = __builtin_shufflevector(vf[i % (AHEAD + 1)][0], vf[i % (AHEAD + 1)][1], 0, 1, 2, 3, 4, 5, 6, 7);
        row.o[i % NB] = M::mma(x, pf[i / NB], row.o[i % NB]);
        row.o[i % NB] = M::mma(x, rest[i / NB], row.o[i % NB]);
    }
    __builtin_amdgcn_sched_barrier(0);
}

// A wave's prefix by DPP: rows of 16 lanes, then each row's last lane to the next row, and lane 31 to the upper half.  (Six steps through
// ds_bpermute took 0.4 us.)
template <class F>
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x, uint32_t none, F f) {
#define DS_DPP(ctrl, rows) f(x, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, ctrl, rows, 0xf, false))
    x = DS_DPP(0x111, 0xf); x = DS_DPP(0x112, 0xf); x = DS_DPP(0x114, 0xf); x = DS_DPP(0x118, 0xf);   // row_shr 1, 2, 4, 8
    x = DS_DPP(0x142, 0xa); x = DS_DPP(0x143, 0xc);                                                  // row_bcast 15, 31
#undef DS_DPP
    return x;
}
__device__ __forceinline__ uint32_t wave_sums_to(uint32_t x) { return wave_prefix(x, 0u, [](uint32_t p, uint32_t q) { return p + q; }); }
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }

// A sequence's rows of the cache, and what lies behind them: its drafted tokens.  (A cache held in 8 bits has rows of 16 bits too, see tree_attn8.hpp: they
// are `held` of the latter.)
struct TreeLengths { uint32_t cached, drafted, held; };
__device__ __forceinline__ TreeLengths tree_lengths(const TreeAttnArgs& a, uint32_t b) {
    return {a.capacity ? clamp_count(a.cached[b], a.capacity) : 0u, a.drafted ? clamp_count(a.drafted[b], a.tokens) : a.tokens, 0u};
}

// How the key axes of all sequences are cut: the lengths are known here only, so every wave works it out for itself.  Up to 64 sequences, a lane
// each: all parts have as many blocks as lets them fit `slots`, whichever sequence they belong to, and an uneven batch keeps the chip as busy as an even one
// (8 x 63 tokens of 32 heads over 500 to 4096 rows: 39 us, and 47 with each sequence cut as the longest one is).  More sequences leave little to cut: there
// each has as many slots.  All of it stands before the first keys are asked for, so it is kept short (divisions are products: compiled ones, and
// a walk over any number of sequences, made a call of one token 1.1 us longer).
struct TreeCut {
    uint32_t b, cached, drafted, held;   // a sequence and its lengths
    uint32_t first, n, size;             // its first slot, its parts, blocks in each (the last has what is left)
};
template <bool SLOT, class Args>         // of the sequence that slot x belongs to (b = batch: to none), or of sequence x
__device__ __forceinline__ TreeCut tree_cut(const Args& a, uint32_t x, uint32_t keys) {
    TreeCut c;
    const bool wide = a.batch > 64;
    const uint32_t b = !wide ? threadIdx.x & 63u : SLOT ? x / a.part_slots : x;
    const TreeLengths len = b < a.batch ? tree_lengths(a, b) : TreeLengths{0, 0, 0};
    const uint32_t cached = len.cached, drafted = len.drafted;
    const uint32_t blocks = (cached + keys - 1) / keys + (drafted + keys - 1) / keys;
    if (wide) return {b, cached, drafted, len.held, b * a.part_slots, min(a.part_slots, (blocks + a.part_blocks - 1) / a.part_blocks), a.part_blocks};
    const uint32_t all = last_lane(wave_sums_to(blocks));
    // Even sequences fill the slots; of uneven ones the last parts are partly empty, up to nearly one part each, and with so many slots less parts fit in
    // any case (there are at least twice as many as sequences).  q is the quotient or, by rounding, one less, which one block more then makes up for.
    uint32_t n, to;
    for (uint32_t quarter = 0;; ++quarter) {
        const uint32_t by = a.slots - (a.batch * quarter >> 2), more = quarter >> 2;
        const uint32_t q = (uint32_t)((float)all * (__builtin_amdgcn_rcpf((float)by) * (1.0f - 0x1p-20f)));
        c.size = uni(max(a.part_least, q + (q * by < all ? 1u + more : 0u) + (q >> 18)));
        // never more parts than there are blocks for: one too few, which a million blocks can come to, makes the last part longer
        n = (uint32_t)((float)blocks * (__builtin_amdgcn_rcpf((float)c.size) * (1.0f - 0x1p-20f)));
        n += n * c.size < blocks ? 1u : 0u;
        to = wave_sums_to(n);
        if (more || last_lane(to) <= a.slots) break;
    }
    const uint64_t hit = SLOT ? __ballot(to > x) : 1ull << x;
    if (!hit) { c.b = a.batch; return c; }
    c.b = (uint32_t)__builtin_ctzll(hit);
    c.cached = (uint32_t)__builtin_amdgcn_readlane((int)cached, (int)c.b);
    c.drafted = (uint32_t)__builtin_amdgcn_readlane((int)drafted, (int)c.b);
    c.held = (uint32_t)__builtin_amdgcn_readlane((int)len.held, (int)c.b);
    c.n = (uint32_t)__builtin_amdgcn_readlane((int)n, (int)c.b);
    c.first = (uint32_t)__builtin_amdgcn_readlane((int)to, (int)c.b) - c.n;
    return c;
}

// The kernel's arguments, read anew: held from the start on they, and what follows from them, go through more scalar registers than there are (128 of
// them spilled, a third of the few rows' kernel was moves from and to lanes).
template <class Args = TreeAttnArgs>
__device__ __forceinline__ const Args& tree_args() {
    typedef const __attribute__((address_space(4))) Args* Segment;
    Segment p = (Segment)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const Args*)p;
}

// What a workgroup works on, the same in every lane.
struct TreeJob {
    uint32_t b, h;                       // sequence, key and value head
    uint32_t slot, n_parts;              // of all parts, parts of this sequence (0: there is no work)
    uint32_t cached, drafted, held;      // of the sequence
    uint32_t cache_blocks, begin, end;   // blocks of cached rows, this part's blocks
};
template <class Args>
__device__ __forceinline__ TreeJob tree_job(const Args& a, uint32_t unit, uint32_t block_keys) {
    TreeJob j;
    j.h = unit % a.kv_heads;
    j.slot = unit / a.kv_heads;
    uint32_t part = 0, size = ~0u;
    j.n_parts = 1;
    if (a.slots > a.batch) {
        const TreeCut c = tree_cut<true>(a, j.slot, block_keys);
        j.b = uni(c.b);
        j.cached = uni(c.cached);
        j.drafted = uni(c.drafted);
        j.held = uni(c.held);
        j.n_parts = uni(c.n);
        part = uni(j.slot - c.first);
        size = c.size;
        if (j.b >= a.batch || part >= j.n_parts) { j.n_parts = 0; return j; }
    } else {
        j.b = j.slot;
        const TreeLengths len = tree_lengths(a, j.b);
        j.cached = uni(len.cached);
        j.drafted = uni(len.drafted);
        j.held = uni(len.held);
    }
    j.cache_blocks = (j.cached + block_keys - 1) / block_keys;
    const uint32_t blocks = j.cache_blocks + (j.drafted + block_keys - 1) / block_keys;
    j.begin = uni(part * size);
    j.end = part + 1 == j.n_parts ? blocks : j.begin + size;
    return j;
}
// A pair's row blocks run on one XCD (every eighth workgroup does), one after the other, so that its keys come from HBM once.
struct TreeUnit { uint32_t unit, row_block; };
__device__ __forceinline__ TreeUnit tree_unit(uint32_t row_blocks) {
    const uint32_t slot = blockIdx.x >> 3;
    return {(slot / row_blocks) * 8 + (blockIdx.x & 7u), slot % row_blocks};
}
// Workspace: outputs [slot][head][row][D], then maxima and sums [slot][head][row][2].
__device__ __forceinline__ size_t tree_part_row(const TreeAttnArgs& a, uint32_t slot, uint32_t h, uint32_t row) {
    return ((size_t)slot * a.kv_heads + h) * a.rows + row;
}
__device__ __forceinline__ float* tree_sums(const TreeAttnArgs& a, int dim) { return a.parts + (size_t)a.slots * a.kv_heads * a.rows * dim; }

// A run of keys as a workgroup or wave copies it to LDS: where it lies, and how many of its 32 (or 64) rows are there.
struct KeyRun {
    const char *k, *v;
    uint32_t pitch;      // bytes
    uint32_t first, n;   // position among the cached rows or the drafted tokens, rows that are there
    bool drafted;
};
template <int D>
__device__ __forceinline__ KeyRun key_run(const TreeAttnArgs& a, const TreeJob& j, uint32_t block, uint32_t block_keys, uint32_t off, uint32_t keys) {
    KeyRun x;
    x.drafted = block >= j.cache_blocks;
    x.first = (block - (x.drafted ? j.cache_blocks : 0u)) * block_keys + off;
    const uint32_t have = x.drafted ? j.drafted : j.cached;
    x.n = x.first < have ? min(keys, have - x.first) : 0u;
    const Strides& s = x.drafted ? a.new_s : a.cache_s;
    const int64_t at = ((int64_t)j.b * s.batch + (int64_t)x.first * s.token + (int64_t)j.h * s.head) * 2;
    x.k = (const char*)(x.drafted ? a.k_new : a.k_cache) + at;
    x.v = (const char*)(x.drafted ? a.v_new : a.v_cache) + at;
    x.pitch = (uint32_t)s.token * 2u;
    return x;
}
template <int D> __device__ __forceinline__ uint32_t run_bytes(const KeyRun& x) { return x.n ? (x.n - 1) * x.pitch + D * 2u : 0u; }

// The keys of a drafted run of 32 that row `t` sees.
__device__ __forceinline__ uint32_t tree_bits(const TreeAttnArgs& a, uint32_t b, uint32_t t, uint32_t first, uint32_t n) {
    if (n == 0) return 0u;
    const uint32_t there = n >= 32 ? ~0u : (1u << n) - 1u;
    if (!a.tree) return t < first ? 0u : t - first >= 31 ? there : there & ((2u << (t - first)) - 1u);
    const uint32_t words = (a.tokens + 63) / 64;
    const uint32_t* w = (const uint32_t*)(a.tree + (int64_t)b * a.tree_batch + (int64_t)t * words);
    return there & w[first >> 5];
}

// Where row r's query lies; rows that there are not get null.
template <typename T>
__device__ __forceinline__ const T* query_row(const TreeAttnArgs& a, const TreeJob& j, uint32_t r) {
    if (r >= a.rows) return nullptr;
    const uint32_t t = r / a.group, g = r - t * a.group;
    return (const T*)a.q + (int64_t)j.b * a.q_s.batch + (int64_t)t * a.q_s.token + (int64_t)(j.h * a.group + g) * a.q_s.head;
}
template <int D> __device__ __forceinline__ void clear_row(RowState<D>& x) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) x.o[b][v] = 0.0f;
    x.m = -INFINITY;
    x.l = 0.0f;
}

// Values of drafted tokens that are not finite were multiplied as zeros, as 0 x inf would reach rows that do not see their key.  What rows
// that do see it miss is added to their sums at the end (the weight is positive: an infinity stays what it is).
template <typename T>
__device__ __forceinline__ f32x4 add_not_finite(const TreeAttnArgs& a, const TreeJob& j, uint32_t block_keys, uint32_t t, uint32_t d, f32x4 o) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (j.end <= j.cache_blocks) return o;
    const uint32_t first = (max(j.begin, j.cache_blocks) - j.cache_blocks) * block_keys, last = min(j.drafted, (j.end - j.cache_blocks) * block_keys);
    for (uint32_t k0 = first; k0 < last; k0 += 32)
        for (uint32_t bits = tree_bits(a, j.b, t, k0, min(32u, last - k0)); bits; bits &= bits - 1) {
            const uint32_t k = k0 + (uint32_t)__builtin_ctz(bits);
            const T4 x = *(const T4*)((const T*)a.v_new + (int64_t)j.b * a.new_s.batch + (int64_t)k * a.new_s.token + (int64_t)j.h * a.new_s.head + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = (float)x[e];
                if (!(fabsf(v) < INFINITY)) o[e] += v;
            }
        }
    return o;
}

// Four output values of row r, d.. : rounded and stored, or left for the second kernel.
template <typename T, int D>
__device__ __forceinline__ void store_row4(const TreeAttnArgs& a, const TreeJob& j, uint32_t r, uint32_t d, f32x4 o, float m, float l, bool odd, uint32_t block_keys) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (r >= a.rows) return;
    const uint32_t t = r / a.group, g = r - t * a.group;
    if (t >= j.drafted) return;
    const uint32_t hq = j.h * a.group + g;
    if (__builtin_expect(odd, 0)) o = add_not_finite<T>(a, j, block_keys, t, d, o);
    if (j.n_parts > 1) {
        const size_t at = tree_part_row(a, j.slot, j.h, r);
        *(f32x4*)(a.parts + at * D + d) = o;
        if (d == 0) {
            float* const ml = tree_sums(a, D) + at * 2;
            ml[0] = m; ml[1] = l;
        }
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;                    // (no key seen: zeros)
    T4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (T)(o[e] * inv);
    *(T4*)((T*)a.out + (int64_t)j.b * a.out_s.batch + (int64_t)t * a.out_s.token + (int64_t)hq * a.out_s.head + d) = x;
    if (d == 0 && a.lse) a.lse[((size_t)j.b * a.tokens + t) * a.heads + hq] = (m + __builtin_amdgcn_logf(l) - WEIGHT_OFF<T>) * 0.69314718055994531f;
}

// ---- few rows ------------------------------------------------------------------------------------------------------------
// 32 rows to a workgroup.  Where no more share a head's keys, the time is that of reading the keys and values once (32 sequences of 2000 to 8192 rows,
// 8 heads, 668 MB: 142 us, 4.7 TB/s).  Each of the four waves walks 32 of a block's 128 keys by itself, with the next step's 16 KB on its way into registers while it works from its own 16 KB of LDS; no wave
// waits for another until the end, when their results are joined through LDS.
template <typename T, int D> constexpr uint32_t tree_wave_bytes() {
    constexpr uint32_t stage = 2 * KeyTile<T, D>::BYTES, join = 32 * (D + 4) * 4;
    return stage > join ? stage : join;
}
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void tree_attn_few(const TreeAttnArgs a) {
    using Tile = KeyTile<T, D>;
    using V8 = typename Mma<T>::V8;
    constexpr uint32_t WAVE = tree_wave_bytes<T, D>();
    __shared__ __align__(16) char lds[4 * WAVE];
    __shared__ __align__(16) char ldsQ[Tile::BYTES];                  // the queries, laid out like keys
    __shared__ float ml[4][32][2];
    __shared__ uint32_t odd;                                           // a drafted value is not finite
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uni(tid >> 6);
    const TreeUnit u = tree_unit((a.rows + TREE_FEW_ROWS - 1) / TREE_FEW_ROWS);
    if (u.unit >= a.slots * a.kv_heads) return;
    const TreeJob j = tree_job(a, u.unit, TREE_FEW_KEYS);
    const uint32_t r0 = u.row_block * TREE_FEW_ROWS;
    if (j.n_parts == 0 || j.begin >= j.end || r0 / a.group >= j.drafted) return;
    if (tid == 0) odd = 0;
    char* const ldsK = lds + wave * WAVE;
    char* const ldsV = ldsK + Tile::BYTES;
    const uint32_t lrow = lane / Tile::CHUNKS, chunk = lane % Tile::CHUNKS;
    u32x4 kreg[Tile::NI], vreg[Tile::NI];
    auto fetch = [&](const KeyRun& x) __attribute__((always_inline)) {
        const uint32_t bytes = uni(run_bytes<D>(x)), first = lrow * x.pitch + chunk * 16;
        const OperandBuf K(uni_ptr(x.k), bytes), V(uni_ptr(x.v), bytes);   // rows that are not there: zeros
#pragma unroll
        for (uint32_t i = 0; i < Tile::NI; ++i) kreg[i] = K.load16(first + i * Tile::RPI * x.pitch, 0);
#pragma unroll
        for (uint32_t i = 0; i < Tile::NI; ++i) vreg[i] = V.load16(first + i * Tile::RPI * x.pitch, 0);
    };
    KeyRun x = key_run<D>(a, j, j.begin, TREE_FEW_KEYS, wave * 32, 32);
    fetch(x);
    RowState<D> row;
    clear_row(row);
    const uint32_t token = min(r0 + (lane & 31u), a.rows - 1) / a.group;
    const float sc = a.scale;
    for (uint32_t i = tid; i < 32 * Tile::CHUNKS; i += 256) {
        const uint32_t rr = i / Tile::CHUNKS, c = i % Tile::CHUNKS;
        const T* q = query_row<T>(a, j, r0 + rr);
        *(u32x4*)(ldsQ + rr * Tile::PITCH + ((c ^ Tile::kswz(rr)) << 4)) = q ? ((const u32x4*)q)[c] : u32x4{0, 0, 0, 0};
    }
    __syncthreads();
    // a lane's first row of a tile; the swizzles are exclusive-ors that repeat every 16 rows
    const uint32_t kput = lrow * Tile::PITCH + ((chunk ^ Tile::kswz(lrow)) << 4), vput = lrow * Tile::PITCH + ((chunk ^ Tile::vswz(lrow)) << 4);
    for (uint32_t blk = j.begin; blk < j.end; ++blk) {
        if (x.drafted) {
            bool bad = false;
#pragma unroll
            for (uint32_t i = 0; i < Tile::NI; ++i) bad |= without_not_finite<T>(vreg[i]);
            if (bad) odd = 1;
        }
        const uint32_t kp = opaque(kput), vp = opaque(vput);
#pragma unroll
        for (uint32_t i = 0; i < Tile::NI; ++i) *(u32x4*)(ldsK + (kp ^ ((Tile::kswz(i * Tile::RPI)) << 4)) + i * Tile::RPI * Tile::PITCH) = kreg[i];
#pragma unroll
        for (uint32_t i = 0; i < Tile::NI; ++i) *(u32x4*)(ldsV + (vp ^ ((Tile::vswz(i * Tile::RPI)) << 4)) + i * Tile::RPI * Tile::PITCH) = vreg[i];
        const KeyRun now = x;
        if (blk + 1 < j.end) {
            if (blk + 1 == j.cache_blocks) {
                x = key_run<D>(tree_args(), j, blk + 1, TREE_FEW_KEYS, wave * 32, 32);
            } else {
                const uint32_t have = x.drafted ? j.drafted : j.cached;
                x.k += TREE_FEW_KEYS * (uint64_t)x.pitch;
                x.v += TREE_FEW_KEYS * (uint64_t)x.pitch;
                x.first += TREE_FEW_KEYS;
                x.n = x.first < have ? min(32u, have - x.first) : 0u;
            }
            fetch(x);
        }
        asm volatile("" ::: "memory");                                 // (a wave's LDS accesses keep their order)
        __builtin_amdgcn_wave_barrier();
        if (now.n) {
            const uint32_t vis[1] = {now.drafted ? tree_bits(tree_args(), j.b, token, now.first, now.n) : now.n >= 32 ? ~0u : (1u << now.n) - 1u};
            const uint32_t qoff = opaque(Tile::koff(lane));
            tree_step<T, D, 1, 2>(row, [&](int kk) __attribute__((always_inline)) { return *(const V8*)(ldsQ + (qoff ^ (kk * 32u))); },
                               ldsK, ldsV, lane, sc, vis, now.drafted || now.n < 32);
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
    // ---- the four waves joined ----
    row.l += __shfl_xor(row.l, 32);
    if (lane < 32) { ml[wave][lane][0] = row.m; ml[wave][lane][1] = row.l; }
    __syncthreads();
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, ml[w][lane & 31u][0]);
    const float f = row.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(row.m - M);
    float* const mine = (float*)(lds + wave * WAVE);                   // (this wave is done with its keys)
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = row.m == -INFINITY && row.l == 0.0f ? 0.0f : row.o[b][4 * g + e] * f;
            *(f32x4*)(mine + (lane & 31u) * (D + 4) + 32 * b + 8 * g + 4 * (lane >> 5)) = o;
        }
    __syncthreads();
    const TreeAttnArgs& late = tree_args();
    const uint32_t rr = tid >> 3;
    float mm = -INFINITY, L = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, ml[w][rr][0]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float mw = ml[w][rr][0], lw = ml[w][rr][1];
        L += mw == -INFINITY ? lw : lw * __builtin_amdgcn_exp2f(mw - mm);         // (a sum without a maximum is 0, or NaN)
    }
#pragma unroll
    for (uint32_t i = 0; i < D / 32; ++i) {
        const uint32_t d = (tid & 7u) * 4 + 32 * i;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) o += *(const f32x4*)((const float*)(lds + w * WAVE) + rr * (D + 4) + d);
        store_row4<T, D>(late, j, r0 + rr, d, o, mm, L, odd != 0, TREE_FEW_KEYS);
    }
}

// ---- many rows -----------------------------------------------------------------------------------------------------------
// 128 rows to a workgroup of four waves, 32 to a wave, two workgroups to a CU (4 sequences of 256 tokens, 64 heads on 8, over 9000 to 16384 rows: 426 GFLOP
// in 460 to 490 us, 0.9 PFLOP/s).  Here the matrix cores and the exponentials are what bounds, so a wave
// does both at once: beside the weights of tile s of 32 keys (16 scores a lane: about 100 VALU instructions, 600 clocks) run the MFMAs of the
// scores of tile s + 1 and of the output of tile s - 1 (16 of 33 clocks at D = 128), in an order that is pinned.  All waves work on the same
// tiles, which the workgroup copies to four LDS slots: K of s + 1 and V of s - 1 are being read, tile s + 2 goes into the slot that V of s - 2
// has left, and s + 3 and s + 4 are on their way through registers.
//
// Here weights are rounded to 16 bits for the product with V (sums keep 32).  Their errors, half a step each and independent, come to about as much as the
// output's own rounding: 2.21e-3 of the outputs' norm in bf16 and 2.59e-4 in fp16, where 32-bit weights leave 1.66e-3 and 2.05e-4.  The form
// for few rows keeps the rest of each weight; here, where MFMAs and conversions are the time, that took 464 -> 618 us (4 x 256 tokens) and 53 -> 79
// (13 tokens of 32 heads of 64 over 120000 rows), too much for a quarter of an error that is within two roundings of T either way.
//
// Rows lie in LDS at pitches that put what is read together into different banks (16 rows of K 16 bytes each, 4 rows of V 64 bytes each) and leave every
// fragment at a constant distance from a lane's first: with exclusive-ors instead, as above, 24 address instructions a tile went beside the MFMAs.
template <int D> struct PaddedTile {
    static constexpr uint32_t K_PITCH = D * 2 + 16, V_PITCH = D * 2 + 64, K_BYTES = 32 * K_PITCH, BYTES = K_BYTES + 32 * V_PITCH;
};
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void tree_attn_many(const TreeAttnArgs a) {
    using Tile = KeyTile<T, D>;
    using Mm = Mma<T>;
    using V8 = typename Mm::V8;
    typedef T T4 __attribute__((ext_vector_type(4)));
    using Pad = PaddedTile<D>;
    constexpr uint32_t SLOT = Pad::BYTES;                              // a tile of K and one of V
    constexpr int KF = D / 16, NB = D / 32, NV = 2 * NB, AHEAD = 3;    // MFMAs of a tile's scores, of its output (as many), LDS reads ahead of them
    __shared__ __align__(16) char lds[4 * SLOT];
    __shared__ uint32_t odd;                                           // a drafted value is not finite
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uni(tid >> 6), h2 = lane >> 5;
    const TreeUnit u = tree_unit((a.rows + TREE_MANY_ROWS - 1) / TREE_MANY_ROWS);
    if (u.unit >= a.slots * a.kv_heads) return;
    const TreeJob j = tree_job(a, u.unit, TREE_MANY_KEYS);
    const uint32_t r0 = u.row_block * TREE_MANY_ROWS, t_last = (min(r0 + TREE_MANY_ROWS, a.rows) - 1) / a.group;
    if (j.n_parts == 0 || j.begin >= j.end || r0 / a.group >= j.drafted) return;
    // without a tree nothing behind the block's last token is seen
    const uint32_t end = a.tree ? j.end : min(j.end, max(j.begin, j.cache_blocks + t_last / TREE_MANY_KEYS + 1));
    constexpr uint32_t NI = Tile::NI / 4;                              // 1 KB copies of a wave: 32 rows over four waves
    const uint32_t lrow = wave * (Tile::RPI * NI) + lane / Tile::CHUNKS, chunk = lane % Tile::CHUNKS;
    struct Staged { u32x4 k[NI], v[NI]; bool drafted; } staged[2];
    auto fetch = [&](const TreeAttnArgs& args, Staged& f, uint32_t tile) __attribute__((always_inline)) {
        KeyRun x = key_run<D>(args, j, tile, TREE_MANY_KEYS, 0, TREE_MANY_KEYS);
        if (tile >= end) x.n = 0;                                      // (behind the last: zeros)
        const uint32_t bytes = uni(run_bytes<D>(x)), first = lrow * x.pitch + chunk * 16;
        const OperandBuf K(uni_ptr(x.k), bytes), V(uni_ptr(x.v), bytes);
        f.drafted = x.drafted;
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) f.k[i] = K.load16(first + i * Tile::RPI * x.pitch, 0);
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) f.v[i] = V.load16(first + i * Tile::RPI * x.pitch, 0);
    };
    auto finite = [&](Staged& f) __attribute__((always_inline)) {
        bool bad = false;
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) bad |= without_not_finite<T>(f.v[i]);
        if (bad) odd = 1;
    };
    auto put = [&](Staged& f, uint32_t slot) __attribute__((always_inline)) {
        char* const to = lds + (slot & 3u) * SLOT + chunk * 16;
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) {
            *(u32x4*)(to + lrow * Pad::K_PITCH + i * Tile::RPI * Pad::K_PITCH) = f.k[i];
            *(u32x4*)(to + lrow * Pad::V_PITCH + Pad::K_BYTES + i * Tile::RPI * Pad::V_PITCH) = f.v[i];
        }
    };
    if (tid == 0) odd = 0;
    // V of the tile before the first, whose weights are zeros: in slot 3
    for (uint32_t i = tid; i < 32 * Pad::V_PITCH / 16; i += 256) *(u32x4*)(lds + 3 * SLOT + Pad::K_BYTES + i * 16) = u32x4{0, 0, 0, 0};
    __syncthreads();
    fetch(a, staged[0], j.begin);
    fetch(a, staged[1], j.begin + 1);
    if (staged[0].drafted) finite(staged[0]);
    put(staged[0], 0);
    fetch(a, staged[0], j.begin + 2);
    if (staged[1].drafted) finite(staged[1]);
    put(staged[1], 1);
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
    auto read_k = [&](const char* slot, int i) __attribute__((always_inline)) { return *(const V8*)(slot + koff + i * 32); };
    auto read_v = [&](const char* slot, int i) __attribute__((always_inline)) {   // slice i / NB of 16 keys, block i % NB of 32 d
        T4 x[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) x[c] = TrRead<T>::read(slot + voff + ((i / NB) * 16 + c * 8) * Pad::V_PITCH + (i % NB) * 64);
        return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    f32x16 st[2];
    V8 pf[2][2] = {};
    const float sc = a.scale;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 16; ++v) st[0][v] = 0.0f;                      // scores of the first tile
#pragma unroll
    for (int i = 0; i < KF; ++i) st[0] = Mm::mma(read_k(lds, i), qf[i], st[0]);
    auto largest = [&](const f32x16& x) __attribute__((always_inline)) {
        float m0 = fmaxf(fmaxf(x[0], x[1]), x[2]), m1 = fmaxf(fmaxf(x[3], x[4]), x[5]);
        m0 = fmaxf(fmaxf(m0, x[6]), x[7]); m1 = fmaxf(fmaxf(m1, x[8]), x[9]);
        m0 = fmaxf(fmaxf(m0, x[10]), x[11]); m1 = fmaxf(fmaxf(m1, x[12]), x[13]);
        return fmaxf(fmaxf(fmaxf(m0, x[14]), x[15]), m1);
    };
    float top = largest(st[0]);                                        // of this lane's scores of the tile to be weighed
    // Weights of the tile whose scores are in `sx`, into `px`; scores of the next tile (in slot `next`) into `sy`, and their largest; output of the
    // one before (in slot `before`) with `py`.
    auto segment = [&](f32x16& sx, V8 (&px)[2], f32x16& sy, const V8 (&py)[2], const char* next, const char* before, bool masked, uint32_t vis)
                       __attribute__((always_inline)) {
        V8 fr[AHEAD + 1];                                              // fragments on their way
        auto rd = [&](int i) __attribute__((always_inline)) { fr[i % (AHEAD + 1)] = i < KF ? read_k(next, i) : read_v(before, i - KF); };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) rd(i);
        if (masked) {
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (!(vis >> (8 * (v / 4) + 4 * h2 + v % 4) & 1u)) sx[v] = -INFINITY;
            top = largest(sx);
        }
        const float mx = max_halves(top) * sc;
        const bool grown = __ballot(mx > row.m + WEIGHT_SLACK) != 0;   // (rarely, after the first steps)
        float alpha = 1.0f;
        if (grown) {
            const float m_new = fmaxf(row.m, mx);
            alpha = row.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(row.m - m_new);
            row.m = m_new;
            row.l *= alpha;
        }
        const float ref = (row.m == -INFINITY ? 0.0f : row.m) - WEIGHT_OFF<T>;   // no key seen yet: keep the exponents finite
        float sum[2] = {0.0f, 0.0f}, x0 = 0.0f, x1 = 0.0f, m0 = -INFINITY, m1 = -INFINITY;
        auto weigh = [&](int v, int half) __attribute__((always_inline)) {       // scores v and v + 1, in two halves
            if (half == 0) {
                x0 = __builtin_fmaf(sx[v], sc, -ref);
                x1 = __builtin_fmaf(sx[v + 1], sc, -ref);
                x0 = __builtin_amdgcn_exp2f(x0);
            } else {
                x1 = __builtin_amdgcn_exp2f(x1);
                sum[0] += x0; sum[1] += x1;                            // summed in 32 bits, rounded to 16 for the product with V alone (above)
                px[v >> 3][v & 7] = (T)x0; px[v >> 3][(v & 7) + 1] = (T)x1;
            }
        };
#pragma unroll
        for (int v = 0; v < 16; ++v) sy[v] = 0.0f;
#pragma unroll
        for (int i = 0; i < KF + NV; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i + AHEAD < KF + NV) rd(i + AHEAD);
            if (i < KF) sy = Mm::mma(fr[i % (AHEAD + 1)], qf[i], sy);
            else row.o[(i - KF) % NB] = Mm::mma(fr[i % (AHEAD + 1)], py[(i - KF) / NB], row.o[(i - KF) % NB]);
            if constexpr (KF == 8) weigh(i & ~1, i & 1);
            else { weigh(2 * i, 0); weigh(2 * i, 1); }
            constexpr int FIRST = KF + NV - 4;                         // the next scores are there by then: four of them to a slot
            if (i >= FIRST) {
                m0 = fmaxf(fmaxf(m0, sy[4 * (i - FIRST)]), sy[4 * (i - FIRST) + 1]);
                m1 = fmaxf(fmaxf(m1, sy[4 * (i - FIRST) + 2]), sy[4 * (i - FIRST) + 3]);
            }
        }
        asm volatile("" ::"v"(px[0]), "v"(px[1]), "v"(sum[0]), "v"(sum[1]), "v"(m0), "v"(m1));   // (computed here, and not where they are used)
        __builtin_amdgcn_sched_barrier(0);
        row.l += sum[0] + sum[1];
        top = fmaxf(m0, m1);
        if (grown) {                                                   // what was added so far went by the reference value before
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) row.o[b][v] *= alpha;
        }
    };
    // One tile: what it copies goes out two tiles before it is put into LDS, and that is a tile before it is read.
    auto step = [&](const TreeAttnArgs& args, uint32_t tile, int odd_one) __attribute__((always_inline)) {
        KeyRun x = key_run<D>(args, j, tile, TREE_MANY_KEYS, 0, TREE_MANY_KEYS);
        if (tile >= end) x.n = 0;
        const bool masked = x.drafted || x.n < 32;
        uint32_t vis = ~0u;
        if (masked) vis = x.drafted ? tree_bits(args, j.b, token, x.first, x.n) : (1u << x.n) - 1u;
        const uint32_t slot = tile - j.begin;
        // (behind the last tile the scores are of whatever the slot holds, and not used)
        segment(st[odd_one], pf[odd_one], st[odd_one ^ 1], pf[odd_one ^ 1], lds + ((slot + 1) & 3u) * SLOT, lds + ((slot - 1) & 3u) * SLOT, masked, vis);
        if (staged[odd_one].drafted) finite(staged[odd_one]);
        put(staged[odd_one], slot + 2);
        fetch(args, staged[odd_one], tile + 4);
        __syncthreads();                                               // the tile put is in its slot, the one read is done with
    };
    uint32_t tile = j.begin;
    // The bulk: whole tiles of cached rows up to the last one fetched, without the general step's 110 scalar instructions and branches a tile.
    const uint32_t whole = min(end, j.cached / TREE_MANY_KEYS);
    if (tile + 5 < whole) {
        const KeyRun x = key_run<D>(a, j, tile + 4, TREE_MANY_KEYS, 0, TREE_MANY_KEYS);
        const char *kp = uni_ptr(x.k), *vp = uni_ptr(x.v);
        const uint32_t bytes = uni(run_bytes<D>(x)), pitch = uni(x.pitch), first = lrow * pitch + chunk * 16;
        auto quick = [&](int odd_one, uint32_t slot) __attribute__((always_inline)) {
            segment(st[odd_one], pf[odd_one], st[odd_one ^ 1], pf[odd_one ^ 1], lds + ((slot + 1) & 3u) * SLOT, lds + ((slot - 1) & 3u) * SLOT, false, ~0u);
            put(staged[odd_one], slot + 2);
            const OperandBuf K(kp, bytes), V(vp, bytes);
#pragma unroll
            for (uint32_t i = 0; i < NI; ++i) staged[odd_one].k[i] = K.load16(first, i * Tile::RPI * pitch);
#pragma unroll
            for (uint32_t i = 0; i < NI; ++i) staged[odd_one].v[i] = V.load16(first, i * Tile::RPI * pitch);
            kp += TREE_MANY_KEYS * (uint64_t)pitch;
            vp += TREE_MANY_KEYS * (uint64_t)pitch;
            __syncthreads();
        };
        for (; tile + 5 < whole; tile += 2) {
            quick(0, tile - j.begin);
            quick(1, tile - j.begin + 1);
        }
        staged[0].drafted = staged[1].drafted = false;
    }
    const TreeAttnArgs& later = tree_args();
    for (; tile < end; tile += 2) {                                    // (a last one without keys where their number is odd)
        step(later, tile, 0);
        step(later, tile + 1, 1);
    }
    if (j.begin < end) {                                               // the output of the last tile
        const char* const last = lds + ((((end - j.begin) + 1) & ~1u) - 1 & 3u) * SLOT;
#pragma unroll
        for (int i = 0; i < NV; ++i) row.o[i % NB] = Mm::mma(read_v(last, i), pf[1][i / NB], row.o[i % NB]);
    }
    const TreeAttnArgs& last_args = tree_args();
    row.l += __shfl_xor(row.l, 32);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = row.o[b][4 * g + e];
            store_row4<T, D>(last_args, j, at, 32 * b + 8 * g + 4 * h2, o, row.m, row.l, odd != 0, TREE_MANY_KEYS);
        }
}

// ---- parts joined --------------------------------------------------------------------------------------------------------
// One wave per query row: D / 4 lanes hold four output values each, and as many such groups as there are walk the parts.  (8 x 63 tokens of 32 heads in
// 3 parts or so each: 11.5 us for 25 MB; a few rows: 4.7 us, the way through two dependent reads.)
template <typename T, int D, class Args>
__global__ __launch_bounds__(256) void tree_attn_join(const Args a) {
    constexpr uint32_t VEC = D / 4, GROUPS = 64 / VEC;
    typedef T T4 __attribute__((ext_vector_type(4)));
    const uint32_t lane = threadIdx.x & 63u;
    const uint64_t item = (uint64_t)blockIdx.x * 4 + uni(threadIdx.x >> 6);
    const uint32_t pair = (uint32_t)(item / a.rows), r = (uint32_t)(item % a.rows);
    if (pair >= a.batch * a.kv_heads) return;
    const uint32_t b = pair / a.kv_heads, h = pair % a.kv_heads;
    const uint32_t t = r / a.group, hq = h * a.group + r % a.group;
    if (t >= (a.drafted ? clamp_count(a.drafted[b], a.tokens) : a.tokens)) return;
    const TreeCut c = tree_cut<false>(a, b, a.few ? TREE_FEW_KEYS : TREE_MANY_KEYS);
    const uint32_t first = uni(c.first), n = uni(c.n);
    if (n < 2) return;                                                // (the part was the whole, and its row is out)
    const float* const ml = tree_sums(a, D);
    float M = -INFINITY;
    for (uint32_t z = lane; z < n; z += 64) M = fmaxf(M, ml[tree_part_row(a, first + z, h, r) * 2]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) M = fmaxf(M, __shfl_xor(M, d));
    float L = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t grp = lane / VEC, d = (lane % VEC) * 4;
#pragma unroll 4
    for (uint32_t z = grp; z < n; z += GROUPS) {
        const size_t at = tree_part_row(a, first + z, h, r);
        const float mz = ml[at * 2], lz = ml[at * 2 + 1];
        const f32x4 v = *(const f32x4*)(a.parts + at * D + d);
        const float f = mz == -INFINITY ? (lz == 0.0f ? 0.0f : lz) : __builtin_amdgcn_exp2f(mz - M);   // (a sum without a maximum is 0, or NaN)
        L += lz * f;
        // Where the factor is 0 a part is too far below the others to count, but its weights are positive: what is not finite in it stays what it is.
        const bool below = f == 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += (below && fabsf(v[e]) < INFINITY ? 0.0f : v[e]) * (below ? 1.0f : f);
    }
#pragma unroll
    for (uint32_t x = VEC; x < 64; x <<= 1) {
        L += __shfl_xor(L, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], x);
    }
    if (grp) return;
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    T4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (T)(o[e] * inv);
    *(T4*)((T*)a.out + (int64_t)b * a.out_s.batch + (int64_t)t * a.out_s.token + (int64_t)hq * a.out_s.head + d) = x;
    if (d == 0 && a.lse) a.lse[((size_t)b * a.tokens + t) * a.heads + hq] = (M + __builtin_amdgcn_logf(L) - WEIGHT_OFF<T>) * 0.69314718055994531f;
}

template <typename T, int D>
hipError_t launch_tree_attn_of(const TreeAttnArgs& a, hipStream_t stream) {
    const uint32_t units = (a.slots * a.kv_heads + 7) / 8 * 8;
    hipError_t e;
    if (a.few) e = launch_one(tree_attn_few<T, D>, units * ((a.rows + TREE_FEW_ROWS - 1) / TREE_FEW_ROWS), 256, stream, a);
    else e = launch_one(tree_attn_many<T, D>, units * ((a.rows + TREE_MANY_ROWS - 1) / TREE_MANY_ROWS), 256, stream, a);
    if (e != hipSuccess || a.slots == a.batch) return e;
    return launch_one(tree_attn_join<T, D, TreeAttnArgs>, (uint32_t)(((uint64_t)a.batch * a.kv_heads * a.rows + 3) / 4), 256, stream, a);
}

template <typename T>
hipError_t launch_tree_attn_type(const TreeAttnArgs& a, int head_dim, hipStream_t stream) {
    return head_dim == 128 ? launch_tree_attn_of<T, 128>(a, stream) : launch_tree_attn_of<T, 64>(a, stream);
}

}  // namespace depsync
