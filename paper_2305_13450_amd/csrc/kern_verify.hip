// Verification of drafted tokens against the target's probabilities.
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

constexpr uint32_t VERIFY_WAVES = 16, FILTER = 1 << 15, LISTED = 256;

// One workgroup to a sequence.
//
// Whether a token stays is decided in 64 bits: the products are then exact or nearly so, and a sum of 2^17 probabilities is off by 2^-50 or so, where
// one in 32 bits is off by more than a rare token has, and a token next to a border would depend on the order of the sum.
//
// The refusals at a node add up: max(max(p - R0 q, 0) - R1 q, 0) = max(p - (R0 + R1) q, 0), so the weights left after any number of them are known from one
// number C, and R, their sum, is asked for only where another child is looked at: a pass over the row (p and q), by the whole workgroup.
// Tokens are taken up in lots of 64, a lane each (in every wave alike): children of the last token that stays are found by a ballot.
template <bool DRAWN>
__global__ __launch_bounds__(64 * VERIFY_WAVES) void verify_drafts_kernel(const VerifyArgs a) {
    __shared__ double sums[VERIFY_WAVES];
    __shared__ uint32_t filter[FILTER / 32], refused_ids[LISTED], n_refused;
    const uint32_t b = blockIdx.x, lane = threadIdx.x & 63u, wave = uni(threadIdx.x >> 6);
    const uint32_t drafted = uni(a.drafted ? clamp_count(a.drafted[b], a.tokens) : a.tokens);
    if (drafted == 0) {
        if (threadIdx.x == 0) a.n_accepted[b] = 0;
        return;
    }
    const float* const P = a.p + (int64_t)b * a.p_batch;
    const float* const Q = DRAWN ? a.q + (int64_t)b * a.q_batch : nullptr;
    const int32_t* const ids = a.ids + (size_t)b * a.tokens;
    const int32_t* const parents = a.parents ? a.parents + (int64_t)b * a.parents_batch : nullptr;
    auto parent_of = [&](uint32_t t) __attribute__((always_inline)) { return parents ? parents[t] : (int32_t)t - 1; };
    // the sum of x over the workgroup, the same in every thread
    auto everywhere = [&](double x) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
        __syncthreads();                                                 // (the sums of the call before are read)
        if (lane == 0) sums[wave] = x;
        __syncthreads();
        double s = 0.0;
#pragma unroll
        for (uint32_t w = 0; w < VERIFY_WAVES; ++w) s += sums[w];
        return s;
    };
    uint32_t last = 0, n = 1;
    double C = 0.0, R = 1.0;
    bool stale = false;                                                  // R is of before the last refusal
    if (threadIdx.x == 0) a.accepted[(size_t)b * a.tokens] = 0;
    for (uint32_t t0 = 0; t0 < drafted; t0 += 64) {
        const uint32_t t = t0 + lane;
        int32_t parent = -1, id = -1;
        double u = 0.0, px = 0.0, qx = 0.0;
        if (t < drafted && t > 0) {
            parent = parent_of(t);
            id = ids[t];
            u = unit(a.u[(size_t)b * a.tokens + t]);
            if (parent >= 0 && (uint32_t)parent < t && id >= 0 && (uint32_t)id < a.vocab) {
                px = mass(P[(int64_t)parent * a.p_token + id]);
                if (DRAWN) qx = mass(Q[(int64_t)parent * a.q_token + id]);
            } else {
                id = -1;
            }
        }
        uint64_t refused = 0;                                            // of this lot, at this node
        uint64_t open = __ballot(t > last && parent == (int32_t)last);
        while (open) {
            const uint32_t i = (uint32_t)__builtin_ctzll(open);
            open &= open - 1;
            const uint32_t x = lane_word((uint32_t)id, i);
            const double ux = lane_value(u, i);
            double w = lane_value(px, i), test;
            if (DRAWN) {
                if (stale) {
                    const float *p = P + (int64_t)last * a.p_token, *q = Q + (int64_t)last * a.q_token;
                    double s = 0.0;
                    for (uint32_t v = threadIdx.x; v < a.vocab; v += 64 * VERIFY_WAVES) s += fmax(mass(p[v]) - C * mass(q[v]), 0.0);
                    R = everywhere(s);
                    stale = false;
                }
                const double qv = lane_value(qx, i);
                w = fmax(w - C * qv, 0.0);
                test = ux * qv * R;
            } else {
                // a token refused here before has nothing left
                bool again = (__ballot((uint32_t)id == x) & refused) != 0;
                for (uint32_t e0 = 0; e0 < t0 && !again; e0 += 64) {
                    const uint32_t e = e0 + lane;
                    again = __ballot(e > last && parent_of(e) == (int32_t)last && (uint32_t)ids[e] == x) != 0;
                }
                if (again) w = 0.0;
                test = ux * R;
            }
            if ((int32_t)x >= 0 && test < w) {
                last = t0 + i;
                if (threadIdx.x == 0) a.accepted[(size_t)b * a.tokens + n] = (int32_t)last;
                ++n;
                C = 0.0; R = 1.0; stale = false;
                refused = 0;
                open = __ballot(t > last && parent == (int32_t)last);
            } else if ((int32_t)x >= 0) {
                refused |= 1ull << i;
                if (DRAWN) { C += R; stale = true; }
                else R = fmax(R - w, 0.0);
            }
        }
    }
    // ---- the next token ----
    if (threadIdx.x == 0) a.n_accepted[b] = (int32_t)n;
    const float *p = P + (int64_t)last * a.p_token, *q = DRAWN ? Q + (int64_t)last * a.q_token : nullptr;
    if (!DRAWN) {
        // The children refused, whose probabilities count for nothing: their numbers, and a filter of 2^15 bits by which hardly any other token is compared with them.
        for (uint32_t w = threadIdx.x; w < FILTER / 32; w += 64 * VERIFY_WAVES) filter[w] = 0;
        __syncthreads();
        if (wave == 0) {
            uint32_t count = 0;
            for (uint32_t t0 = last & ~63u; t0 < drafted; t0 += 64) {
                const uint32_t t = t0 + lane;
                const bool child = t > last && t < drafted && parent_of(t) == (int32_t)last;
                const uint32_t id = child ? (uint32_t)ids[t] : 0u;
                const uint64_t children = __ballot(child);
                const uint32_t at = count + (uint32_t)__builtin_popcountll(children & ((1ull << lane) - 1));
                if (child) atomicOr(&filter[id % FILTER / 32], 1u << (id % 32));
                if (child && at < LISTED) refused_ids[at] = id;
                count += (uint32_t)__builtin_popcountll(children);
            }
            if (lane == 0) n_refused = count;
        }
        __syncthreads();
    }
    bool whole = false;                                                  // p as it is
    auto refused_here = [&](uint32_t v) __attribute__((always_inline)) {
        if (n_refused <= LISTED) {
            for (uint32_t e = 0; e < n_refused; ++e)
                if (refused_ids[e] == v) return true;
        } else {
            for (uint32_t t = last + 1; t < drafted; ++t)
                if (parent_of(t) == (int32_t)last && (uint32_t)ids[t] == v) return true;
        }
        return false;
    };
    auto weight = [&](uint32_t v) __attribute__((always_inline)) {
        const double w = mass(p[v]);
        if (whole) return w;
        if (DRAWN) return fmax(w - C * mass(q[v]), 0.0);
        if ((filter[v % FILTER / 32] >> (v % 32) & 1u) && refused_here(v)) return 0.0;
        return w;
    };
    // Where the sum passes the target: a run is cut into 16 pieces, a wave sums each, and the piece that the target lies in is the next run.  Where rounding
    // leaves none, it is the last one that has any weight.
    uint32_t begin = 0, end = a.vocab;
    double before = 0.0, target = -1.0;                                  // the sum in front of the run
    int32_t next = -1;
    for (;;) {
        const uint32_t piece = ((end - begin + VERIFY_WAVES - 1) / VERIFY_WAVES + 63) & ~63u;
        const uint32_t from = begin + wave * piece, to = min(end, from + piece);
        double s = 0.0;
#pragma unroll 4
        for (uint32_t v = from + lane; v < to; v += 64) s += weight(v);
        const double all = everywhere(s);
        if (target < 0.0) {                                              // the first run is the row
            if (!(all > 0.0)) {
                if (whole) break;
                whole = true;
                continue;
            }
            target = unit(a.u[(size_t)b * a.tokens]) * all;
        }
        uint32_t hit = VERIFY_WAVES, some = 0;
        double sum = before, in_front = before, in_front_of_some = before;
        for (uint32_t w = 0; w < VERIFY_WAVES; ++w) {
            if (sums[w] > 0.0) { some = w; in_front_of_some = sum; }
            if (hit == VERIFY_WAVES && sum + sums[w] > target) { hit = w; in_front = sum; }
            sum += sums[w];
        }
        if (hit == VERIFY_WAVES) { hit = some; in_front = in_front_of_some; target = INFINITY; }
        before = in_front;
        begin += hit * piece;
        end = min(end, begin + piece);
        if (piece == 64) {
            const double w = begin + lane < end ? weight(begin + lane) : 0.0;
            double upto = w;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const double y = __shfl_up(upto, d);
                if (lane >= (uint32_t)d) upto += y;
            }
            const uint64_t over = __ballot(before + upto > target && w > 0.0), any = __ballot(w > 0.0);
            next = (int32_t)(begin + (over ? (uint32_t)__builtin_ctzll(over) : 63u - (uint32_t)__builtin_clzll(any | 1u)));
            break;
        }
    }
    if (threadIdx.x == 0) a.next[b] = next;
}

}  // namespace

hipError_t launch_verify_drafts(const VerifyArgs& a, hipStream_t stream) {
    return a.q ? launch_one(verify_drafts_kernel<true>, a.batch, 64 * VERIFY_WAVES, stream, a) : launch_one(verify_drafts_kernel<false>, a.batch, 64 * VERIFY_WAVES, stream, a);
}

}  // namespace depsync
