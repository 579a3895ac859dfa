// Verification of drafted tokens against the target's probabilities.
//
// Whether a token stays is decided in 64 bits: the products are then exact or nearly so, and a sum of 2^17 probabilities is off by 2^-50 or so, where
// one in 32 bits is off by more than a rare token has, and a token next to a border would depend on the order of the sum.
//
// The refusals at a node add up: max(max(p - R0 q, 0) - R1 q, 0) = max(p - (R0 + R1) q, 0), so the weights left after any number of them are known from one
// number C, and R, their sum, is asked for only where another child is looked at: a pass over the row (p and q).  What a sequence reads is a few numbers a
// token, those passes, and the row that the next token is drawn from.
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "tree_attn.hpp"

namespace depsync {

namespace {

// What counts of a probability, and of a random number.
__device__ __forceinline__ double mass(float x) { return x > 0.0f && x < INFINITY ? (double)x : 0.0; }
__device__ __forceinline__ double unit(float u) { return u > 0.0f ? fmin((double)u, 1.0) : 0.0; }

__device__ __forceinline__ double lane_value(double x, uint32_t lane) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)bits, (int)lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(bits >> 32), (int)lane);
    return __builtin_bit_cast(double, lo | hi << 32);
}
__device__ __forceinline__ uint32_t lane_word(uint32_t x, uint32_t lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (int)lane); }
// Sums up to each lane, by DPP: rows of 16 lanes, then each row's last lane to the next row, and lane 31 to the upper half.
__device__ __forceinline__ double sums_to(double x) {
#define DS_DPP(ctrl, rows) { \
        const uint64_t bits = __builtin_bit_cast(uint64_t, x); \
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, ctrl, rows, 0xf, false), \
                       hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), ctrl, rows, 0xf, false); \
        x += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); \
    }
    DS_DPP(0x111, 0xf) DS_DPP(0x112, 0xf) DS_DPP(0x114, 0xf) DS_DPP(0x118, 0xf)   // row_shr 1, 2, 4, 8
    DS_DPP(0x142, 0xa) DS_DPP(0x143, 0xc)                                        // row_bcast 15, 31
#undef DS_DPP
    return x;
}
__device__ __forceinline__ double wave_sum(double x) { return lane_value(sums_to(x), 63); }

// A sequence's arrays.
struct Drafts {
    const float *p, *q;
    const int32_t *ids, *parents;
    uint32_t drafted;
    __device__ __forceinline__ Drafts(const VerifyArgs& a, uint32_t b)
        : p(a.p + (int64_t)b * a.p_batch), q(a.q ? a.q + (int64_t)b * a.q_batch : nullptr), ids(a.ids + (size_t)b * a.tokens),
          parents(a.parents ? a.parents + (int64_t)b * a.parents_batch : nullptr), drafted(uni(a.drafted ? clamp_count(a.drafted[b], a.tokens) : a.tokens)) {}
    __device__ __forceinline__ int32_t parent(uint32_t t) const { return parents ? parents[t] : (int32_t)t - 1; }
};

// A wave's LDS accesses keep their order.
__device__ __forceinline__ void in_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// 64 tokens from t0 on, a lane each.  Their probabilities are gathered from rows far apart once: where launches follow one another the first keeps them.
struct Lot {
    int32_t parent = -1, id = -1;        // -1: none, or not in the vocabulary
    double u = 0.0, px = 0.0, qx = 0.0;
};
__device__ __forceinline__ Lot tokens_of(const VerifyArgs& a, uint32_t b, const Drafts& d, uint32_t t0) {
    const uint32_t t = t0 + (threadIdx.x & 63u);
    Lot x;
    if (t > 0 && t < a.tokens) {
        x.parent = d.parent(t);
        x.id = d.ids[t];
        x.u = unit(a.u[(size_t)b * a.tokens + t]);
    }
    return x;
}
template <bool DRAWN> __device__ __forceinline__ Lot lot_of(const VerifyArgs& a, uint32_t b, const Drafts& d, uint32_t t0, bool kept) {
    const uint32_t t = t0 + (threadIdx.x & 63u);
    Lot x = tokens_of(a, b, d, t0);
    VerifyToken w = {0.0f, 0.0f};
    if (DRAWN && kept && t < a.tokens) w = a.kept[(size_t)b * a.tokens + t];
    if (x.parent >= 0 && (uint32_t)x.parent < t && x.id >= 0 && (uint32_t)x.id < a.vocab) {
        if (!DRAWN || !kept) {
            w.p = d.p[(int64_t)x.parent * a.p_token + x.id];
            if (DRAWN) w.q = d.q[(int64_t)x.parent * a.q_token + x.id];
        }
        x.px = mass(w.p);
        if (DRAWN) x.qx = mass(w.q);
    } else {
        x.id = -1;
    }
    return x;
}

// The children refused at the last token that stays, without q: their probabilities count for nothing.  Their numbers in a table of twice as many places (from a
// number's own on, the first that is free), and a filter of 2^15 bits by which hardly any other token of the vocabulary is looked for in it.  Up to 512 tokens: 8 KB, which cost no
// launch a place on a CU; up to 4096: 36 KB.  (2 stars of 200 refused children over 32000 numbers: 33 us; of 4096: 0.48 ms, nearly all of it the walk from child to child, 0.11 us each.)
constexpr uint32_t FILTER = 1 << 15;
template <uint32_t LISTED> struct Refused {
    static constexpr uint32_t PLACES = 2 * LISTED, FREE = ~0u;
    uint32_t filter[FILTER / 32], table[PLACES];
    static __device__ __forceinline__ uint32_t place(uint32_t id) { return id * 0x9e3779b1u >> (32 - __builtin_ctz(PLACES)); }
    template <uint32_t THREADS> __device__ __forceinline__ void clear(uint32_t thread) {
        for (uint32_t i = thread; i < FILTER / 128; i += THREADS) ((u32x4*)filter)[i] = u32x4{0, 0, 0, 0};
        for (uint32_t i = thread; i < PLACES / 4; i += THREADS) ((u32x4*)table)[i] = u32x4{FREE, FREE, FREE, FREE};
    }
    // (LISTED different ones at most, so a place is free)
    __device__ __forceinline__ void add(uint32_t id) {
        for (uint32_t i = place(id);; i = (i + 1) % PLACES) {
            const uint32_t there = atomicCAS(&table[i], FREE, id);
            if (there == FREE || there == id) break;
        }
        atomicOr(&filter[id % FILTER / 32], 1u << (id % 32));
    }
    __device__ __forceinline__ bool listed(uint32_t id) const {
        for (uint32_t i = place(id);; i = (i + 1) % PLACES) {
            const uint32_t there = table[i];
            if (there == id) return true;
            if (there == FREE) return false;
        }
    }
    __device__ __forceinline__ bool has(uint32_t id) const { return (filter[id % FILTER / 32] >> (id % 32) & 1u) && listed(id); }
};

// From s.at on; every wave that calls this does the same.  The children of the last one that stays are found by a ballot.  first: the lot from 0 on.
// Where R is needed and stale: pass(s) renews it, or returns false, and so does this then.
// Without q one wave of a workgroup calls this, from the first token on, and `refused`, empty before, holds the children of s.last afterwards.
template <bool DRAWN, class Set, class Pass>
__device__ __forceinline__ bool verify_walk(const VerifyArgs& a, uint32_t b, const Drafts& d, const Lot& first, bool kept, VerifyState& s, bool write, Set& refused, Pass pass) {
    const uint32_t lane = threadIdx.x & 63u;
    bool some = false;                                                   // `refused` is not empty: children of earlier lots
    if (write && s.at == 1) a.accepted[(size_t)b * a.tokens] = 0;
    for (uint32_t t0 = s.at & ~63u; t0 < d.drafted; t0 += 64) {
        const uint32_t t = t0 + lane;
        const Lot x0 = t0 ? lot_of<DRAWN>(a, b, d, t0, kept) : first;
        const int32_t parent = t < d.drafted ? x0.parent : -1, id = x0.id;
        const double u = x0.u, px = x0.px, qx = x0.qx;
        uint64_t gone = 0;                                               // refused, of this lot, at this node
        uint64_t open = __ballot(t > s.last && t >= s.at && parent == (int32_t)s.last);
        uint64_t before = 0;                                             // whose token was refused at this node in an earlier lot
        if (!DRAWN && some && open) before = __ballot((open >> lane & 1u) && id >= 0 && refused.listed((uint32_t)id));
        while (open) {
            const uint32_t i = (uint32_t)__builtin_ctzll(open);
            const uint32_t x = lane_word((uint32_t)id, i);
            const double ux = lane_value(u, i);
            double w = lane_value(px, i), test;
            if (DRAWN) {
                if (s.stale) {
                    s.at = t0 + i;
                    if (!pass(s)) return false;
                    s.stale = 0;
                }
                const double qv = lane_value(qx, i);
                w = fmax(w - s.C * qv, 0.0);
                test = ux * qv * s.R;
            } else {
                // a token refused here before has nothing left
                if ((__ballot((uint32_t)id == x) & gone) | (before >> i & 1u)) w = 0.0;
                test = ux * s.R;
            }
            open &= open - 1;
            if ((int32_t)x >= 0 && test < w) {
                s.last = t0 + i;
                if (write) a.accepted[(size_t)b * a.tokens + s.n] = (int32_t)s.last;
                ++s.n;
                s.C = 0.0; s.R = 1.0; s.stale = 0;
                gone = before = 0;
                if (!DRAWN && some) {                                    // (once a lot at most)
                    refused.template clear<64>(lane);
                    in_order();
                    some = false;
                }
                open = __ballot(t > s.last && parent == (int32_t)s.last);
            } else if ((int32_t)x >= 0) {
                gone |= 1ull << i;
                if (DRAWN) { s.C += s.R; s.stale = 1; }
                else s.R = fmax(s.R - w, 0.0);
            }
        }
        if (!DRAWN && gone) {
            if (gone >> lane & 1u) refused.add((uint32_t)id);
            in_order();
            some = true;
        }
    }
    s.at = d.drafted;
    return true;
}

// The weight of a token in a row.
template <bool DRAWN, class Set> struct Weights {
    const float *p, *q;
    double C;
    const Set& refused;
    bool whole;                          // p as it is
    __device__ __forceinline__ Weights(const VerifyArgs& a, const Drafts& drafts, const VerifyState& s, const Set& r)
        : p(drafts.p + (int64_t)s.last * a.p_token), q(DRAWN ? drafts.q + (int64_t)s.last * a.q_token : nullptr), C(s.C), refused(r), whole(false) {}
    __device__ __forceinline__ double of(uint32_t v, float pv, float qv) const {
        const double w = mass(pv);
        if (whole) return w;
        if (DRAWN) return fmax(w - C * mass(qv), 0.0);
        return refused.has(v) ? 0.0 : w;
    }
    // The sum over v, v + step, .. below `end`, eight numbers on their way at a time, also where fewer are left.
    __device__ __forceinline__ double sum(uint32_t v, uint32_t step, uint32_t end) const {
        double x = 0.0;
        for (; v < end; v += 8 * step) {
            float pv[8], qv[8] = {};
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) pv[k] = p[min(v + k * step, end - 1)];
            if (DRAWN)
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) qv[k] = q[min(v + k * step, end - 1)];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
                if (v + k * step < end) x += of(v + k * step, pv[k], qv[k]);
        }
        return x;
    }
};

// (the same in every lane: 12 us longer where the compiler was not told)
__device__ __forceinline__ VerifyState uniform(const VerifyState& x) {
    return {lane_value(x.C, 0), lane_value(x.R, 0), uni(x.last), uni(x.n), uni(x.at), uni(x.stale), uni(x.done)};
}

constexpr uint32_t VERIFY_WAVES = 16;

// The sum of x over a workgroup of `WAVES` waves, the same in every thread; sums[w] stays the sum of wave w until the next call.
template <uint32_t WAVES> __device__ __forceinline__ double everywhere(double x, double* sums) {
    x = wave_sum(x);
    __syncthreads();                                                     // (the sums of the call before are read)
    if ((threadIdx.x & 63u) == 0) sums[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (uint32_t w = 0; w < WAVES; ++w) s += sums[w];
    return s;
}

// The piece whose sum, added to `before` and those in front of it, passes the target: `before` becomes the sum in front of it.  A lane holds each (64 at most, others
// 0).  Where rounding leaves none it is the last that has any weight, and the target infinity.
__device__ __forceinline__ uint32_t find_piece(double mine, double& before, double& target) {
    const double upto = sums_to(mine);
    const uint64_t over = __ballot(before + upto > target && mine > 0.0), some = __ballot(mine > 0.0);
    if (!over) target = INFINITY;
    const uint32_t hit = over ? (uint32_t)__builtin_ctzll(over) : some ? 63u - (uint32_t)__builtin_clzll(some) : 0u;
    if (hit) before += lane_value(upto, hit - 1);
    return hit;
}

// The rest of a sequence in one workgroup: the walk with its passes, and the next token.
// Where the sum passes the target: a run is cut into 16 pieces, a wave sums each, and the piece that the target lies in is the next run, until that is short enough for registers.
// piece_sum: of an earlier launch, of the row's pieces of `size` numbers, one a lane (size 0: there are none).
// tokens: of this wave's lot of the first ones.
template <bool DRAWN, class Set>
__device__ __forceinline__ void verify_rest(const VerifyArgs& a, uint32_t b, const Drafts& d, const Lot& tokens, float u0, VerifyState& s, double piece_sum, uint32_t size, double* sums, VerifyState& come, Set& refused) {
    constexpr uint32_t SHORT = VERIFY_WAVES * 256;
    const uint32_t lane = threadIdx.x & 63u, wave = uni(threadIdx.x >> 6);
    if (!DRAWN) {
        refused.template clear<64 * VERIFY_WAVES>(threadIdx.x);
        __syncthreads();
        if (size) {
            for (uint32_t t0 = wave * 64; t0 < d.drafted; t0 += 64 * VERIFY_WAVES) {
                const Lot x = t0 == wave * 64 ? tokens : tokens_of(a, b, d, t0);
                const uint32_t t = t0 + lane;
                if (t > s.last && t < d.drafted && x.parent == (int32_t)s.last && (uint32_t)x.id < a.vocab) refused.add((uint32_t)x.id);
            }
        } else if (wave == 0) {
            verify_walk<DRAWN>(a, b, d, lot_of<DRAWN>(a, b, d, 0, false), false, s, lane == 0, refused, [](VerifyState&) { return true; });
            if (lane == 0) come = s;
        }
        __syncthreads();
        if (size == 0) s = uniform(come);
    } else if (size == 0) {
        verify_walk<DRAWN>(a, b, d, lot_of<DRAWN>(a, b, d, 0, a.launches > 1), a.launches > 1, s, threadIdx.x == 0, refused, [&](VerifyState& st) __attribute__((always_inline)) {
            const Weights<DRAWN, Set> weight(a, d, st, refused);
            st.R = everywhere<VERIFY_WAVES>(weight.sum(threadIdx.x, 64 * VERIFY_WAVES, a.vocab), sums);
            return true;
        });
    }
    if (threadIdx.x == 0) a.n_accepted[b] = (int32_t)s.n;
    Weights<DRAWN, Set> weight(a, d, s, refused);
    uint32_t begin = 0, end = a.vocab;
    double before = 0.0, target = -1.0;                                  // the sum in front of the run
    const double u = unit(u0);
    int32_t next = -1;
    if (size) {
        const double all = wave_sum(piece_sum);
        if (all > 0.0) {
            target = u * all;
            begin = find_piece(piece_sum, before, target) * size;
            end = min(end, begin + size);
        } else {
            weight.whole = true;
        }
    }
    bool done = false;
    while (end - begin > SHORT || target < 0.0) {
        const uint32_t piece = ((end - begin + VERIFY_WAVES - 1) / VERIFY_WAVES + 63) & ~63u;
        const uint32_t from = begin + wave * piece, to = min(end, from + piece);
        const double all = everywhere<VERIFY_WAVES>(weight.sum(from + lane, 64, to), sums);
        if (target < 0.0) {                                              // the first run is the row
            if (!(all > 0.0)) {
                done = weight.whole;                                     // nothing at all: -1
                if (done) break;
                weight.whole = true;
                continue;
            }
            target = u * all;
        }
        begin += find_piece(lane < VERIFY_WAVES ? sums[lane] : 0.0, before, target) * piece;
        end = min(end, begin + piece);
    }
    if (!done) {
        // 256 numbers to a wave, four to a lane, in order from 64 to 64
        double upto[4], w[4], x = 0.0;
        float pv[4], qv[4] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t v = begin + wave * 256 + k * 64 + lane;
            pv[k] = weight.p[min(v, end - 1)];
            if (DRAWN) qv[k] = weight.q[min(v, end - 1)];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t v = begin + wave * 256 + k * 64 + lane;
            w[k] = v < end ? weight.of(v, pv[k], qv[k]) : 0.0;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            upto[k] = sums_to(w[k]) + x;
            x = lane_value(upto[k], 63);
        }
        __syncthreads();
        if (lane == 0) sums[wave] = x;
        __syncthreads();
        const uint32_t hit = find_piece(lane < VERIFY_WAVES ? sums[lane] : 0.0, before, target);
        if (wave != hit) return;
        uint32_t last_some = 0;
        bool found = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint64_t over = __ballot(before + upto[k] > target && w[k] > 0.0), any = __ballot(w[k] > 0.0);
            if (over && !found) { found = true; next = (int32_t)(begin + hit * 256 + k * 64 + (uint32_t)__builtin_ctzll(over)); }
            if (any) last_some = k * 64 + 63u - (uint32_t)__builtin_clzll(any);
        }
        if (!found) next = (int32_t)(begin + hit * 256 + last_some);
        if (lane == 0) a.next[b] = next;
        return;
    }
    if (threadIdx.x == 0) a.next[b] = next;
}

// One workgroup to a sequence.
template <bool DRAWN, uint32_t LISTED>
__global__ __launch_bounds__(64 * VERIFY_WAVES) void verify_drafts_kernel(const VerifyArgs a) {
    __shared__ double sums[VERIFY_WAVES];
    __shared__ VerifyState come;
    __shared__ __align__(16) Refused<LISTED> refused;
    const uint32_t b = blockIdx.x, lane = threadIdx.x & 63u;
    const Drafts d(a, b);
    VerifyState s = {0.0, 1.0, 0, 1, 1, 0, 0};
    double found[VERIFY_LAUNCHES] = {}, piece_sum = 0.0;
    if (a.launches) {                                                    // what earlier launches found out: all of it is asked for at once
        s = a.states[(size_t)(a.launches - 1) * a.batch + b];
#pragma unroll
        for (uint32_t l = 0; l < VERIFY_LAUNCHES; ++l)
            if (l < a.launches && lane < a.pieces) found[l] = a.sums[((size_t)l * a.batch + b) * a.pieces + lane];
    }
    const Lot tokens = tokens_of(a, b, d, uni(threadIdx.x >> 6) * 64);
    const float u0 = a.u[(size_t)b * a.tokens];
    if (d.drafted == 0) {
        if (threadIdx.x == 0) a.n_accepted[b] = 0;
        return;
    }
#pragma unroll
    for (uint32_t l = 0; l < VERIFY_LAUNCHES; ++l)
        if (l + 1 == (s.done ? s.done : a.launches)) piece_sum = found[l];
    if (a.launches && !s.done) {
        s.R = wave_sum(piece_sum);
        s.stale = 0;
    }
    verify_rest<DRAWN>(a, b, d, tokens, u0, s, piece_sum, s.done ? a.piece : 0u, sums, come, refused);
}

// A row over several workgroups: the first wave of each goes as far as it can without a pass (all of a sequence's do the same), each leaves the sum of its piece of the
// row that it came to, and the next launch goes on from there.
// Latency bounds it, some 5 us a launch: its loads wait for one another (state, tokens, their probabilities, the row), so as many as can go together do, and the gathered ones are kept (32
// trees of 16 over 50000 tokens, on average over their inputs: 41 us before that, and 37).
template <bool DRAWN, uint32_t LISTED>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyArgs a) {
    __shared__ double sums[4];
    __shared__ VerifyState come;
    __shared__ __align__(16) Refused<LISTED> refused;
    const uint32_t b = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, wave = uni(threadIdx.x >> 6);
    VerifyState* const to = a.states + (size_t)a.launch * a.batch + b;
    VerifyState s = {0.0, 1.0, 0, 1, 1, 0, 0};
    if (a.launch) {
        s = a.states[(size_t)(a.launch - 1) * a.batch + b];
        if (s.done) {
            if (piece == 0 && threadIdx.x == 0) *to = s;
            return;
        }
    }
    const Drafts d(a, b);
    if (d.drafted == 0) {
        s.done = 1;
        if (piece == 0 && threadIdx.x == 0) *to = s;
        return;
    }
    Lot first;
    if (wave == 0) first = lot_of<DRAWN>(a, b, d, 0, a.launch > 0);
    if (!DRAWN) {
        refused.template clear<256>(threadIdx.x);
        __syncthreads();
    }
    if (wave == 0) {
        const uint32_t lane = threadIdx.x;
        double piece_sum = 0.0;
        if (a.launch && lane < a.pieces) piece_sum = a.sums[((size_t)(a.launch - 1) * a.batch + b) * a.pieces + lane];
        if (a.launch) {
            s.R = wave_sum(piece_sum);
            s.stale = 0;
        }
        if (verify_walk<DRAWN>(a, b, d, first, a.launch > 0, s, piece == 0 && lane == 0, refused, [](VerifyState&) { return false; })) s.done = a.launch + 1;
        if (lane == 0) come = s;
    }
    if (DRAWN && a.launch == 0 && a.launches > 1)
        for (uint32_t t0 = (piece * 4 + wave) * 64; t0 < a.tokens; t0 += a.pieces * 256) {
            const Lot x = t0 ? lot_of<DRAWN>(a, b, d, t0, false) : first;
            const uint32_t t = t0 + (threadIdx.x & 63u);
            if (t < a.tokens) a.kept[(size_t)b * a.tokens + t] = VerifyToken{(float)x.px, (float)x.qx};
        }
    __syncthreads();
    s = uniform(come);
    const Weights<DRAWN, Refused<LISTED>> weight(a, d, s, refused);
    double x = weight.sum(piece * a.piece + threadIdx.x, 256, min(a.vocab, (piece + 1) * a.piece));
    x = everywhere<4>(x, sums);
    if (threadIdx.x == 0) {
        a.sums[((size_t)a.launch * a.batch + b) * a.pieces + piece] = x;
        if (piece == 0) *to = s;
    }
}

template <bool DRAWN, uint32_t LISTED>
hipError_t launch_verify_with(VerifyArgs a, hipStream_t stream) {
    for (a.launch = 0; a.launch < a.launches; ++a.launch)
        if (hipError_t e = launch_one(verify_sums_kernel<DRAWN, LISTED>, a.batch * a.pieces, 256, stream, a); e != hipSuccess) return e;
    return launch_one(verify_drafts_kernel<DRAWN, LISTED>, a.batch, 64 * VERIFY_WAVES, stream, a);
}

}  // namespace

hipError_t launch_verify_drafts(const VerifyArgs& a, hipStream_t stream) {
    if (a.q) return launch_verify_with<true, VERIFY_FEW>(a, stream);   // (which list nothing)
    return a.tokens <= VERIFY_FEW ? launch_verify_with<false, VERIFY_FEW>(a, stream) : launch_verify_with<false, VERIFY_TOKENS>(a, stream);
}

}  // namespace depsync
