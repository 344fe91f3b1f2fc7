// kb_attn_tile.hpp -- attention, forward: the softmax of a wave's 32 query rows
// over one tile of keys in LDS, with its two matrix products.
#pragma once

#include "kb_attn.hpp"

namespace kb {

// The softmax state of a lane's query over the tiles so far: terms are exp(scale
// (s - m)).  In 32 bits m is the maximum.  In 16 bits it is a reference, held as
// scale m / ln 2 (one instruction makes a term's exponent), that follows the
// maximum only when a term would pass 2^kSlack of the one that set it (scaling the
// sums takes as long as a quarter of a tile's products), and next to l, the sum of
// the terms, there is the sum of the rounded terms, those whose product with v is
// divided by it: where one term outweighs the others, o is its v to the last bit.
// (Terms in two parts, as the attention over pages has them for few rows, would take
// half as many products again: 6 packed prompts of up to 4095 tokens, bf16, 402 us
// instead of 311, whose error against 64 bits is 2.0e-3; the rounding of o alone makes
// 1.6e-3.)
// F16 holds small terms badly (subnormal from 2^-14, nothing under 2^-25), so there
// the reference is set 2^kBelow under the maximum: terms of up to 2^15, and what the
// format takes from one is at most 2^-34 of the largest.
template <int DT>
constexpr float kSlack = DT == DT_F16 ? 6.f : 8.f;
template <int DT>
constexpr float kBelow = DT == DT_F16 ? 9.f : 0.f;

// Sums of terms times values: terms of up to 2^kSlack, or many of 1, pass binary32's
// range with values whose mean does not.  Sums past kLarge are computed once more, with
// the n keys' terms, relative to their maximum, times 2^-large_shift(n): they come to
// 1/2 together.  (Of other sums 2^16 can be joined.  F16: 2^30 terms of 2^15 and values
// of 2^16 stay far inside; there only an infinity or a NaN is past kLarge.)
constexpr float kLarge = 0x1p110f;
template <int DT>
constexpr bool kScaled = DT != DT_F16;
template <int DT>
__device__ __forceinline__ int large_shift(int n) {
    return !kScaled<DT> || n < 2 ? 0 : 33 - __builtin_clz((uint32_t)(n - 1));
}

template <int N>
__device__ __forceinline__ bool too_large(const f32x16 (&acc)[N]) {
    float largest = 0.f;  // (or NaN)
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) largest = __builtin_elementwise_maximum(largest, fabsf(acc[k][r]));
    return !(largest <= kLarge);
}

struct Softmax {
    float m = -INFINITY, l = 0.f, rounded = 0.f;
    bool low = false;
};

// Binary32 holds a reference of 2^22 or more too coarsely for terms relative to
// it: by the rounding of scale m / ln 2 alone they would be 0 or infinite.  So a
// reference is not set by scores below -2^22 (the lowest numbers of bf16 in a row of
// k, as a mask; they are noted in `low`), and a work-group with a row that ends up
// with such scores alone, or with a larger reference, computes its sums once more
// (CAREFUL), m being a score as in 32 bits.
constexpr float kCoarse = 4194304.f;
__device__ __forceinline__ bool too_coarse(const Softmax& sm) {
    return sm.m == -INFINITY ? sm.low : fabsf(sm.m) >= kCoarse;
}

// What m is held in: log2 units of m, and natural ones.  (Scale over what the
// scores are multiplied by: the rounding of that factor leaves lse again.)
template <int DT>
__device__ __forceinline__ float unit_log2(float scale) {
    return DT == DT_F32 ? scale * kLog2e : 1.f;
}
template <int DT>
__device__ __forceinline__ float unit_natural(float scale) {
    return DT == DT_F32 ? scale : scale / (scale * kLog2e);
}

template <int DT>
__device__ __forceinline__ float add_terms(frag_t<DT> f, float l) {
    typedef storage_t<DT> two __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const two x = {f[e], f[e + 1]}, one = {(storage_t<DT>)1.f, (storage_t<DT>)1.f};
        if constexpr (DT == DT_F16) l = __builtin_amdgcn_fdot2(x, one, l, false);
        if constexpr (DT == DT_BF16) l = __builtin_amdgcn_fdot2_f32_bf16(x, one, l, false);
    }
    return l;
}

// The keys of one tile for 32 query rows of a wave.  PART: some (row, key)
// pairs are not seen; the lane's row sees the tile's keys below hi, and with GAPS
// only those whose bit is set in `present` (the values of the others are zeros).
// CAREFUL: m is the largest score, as in 32 bits, terms go into the product (and
// their rounded sum) times 2^-shift, and mma_seen for rows that are not seen.
template <int DT, int DP, bool PART, bool CAREFUL, bool GAPS = false>
__device__ __forceinline__ void tile_forward(f32x16 (&acc)[DP / 32], Softmax& sm, const frag_t<DT> (&qf)[DP / 16],
                                             const storage_t<DT>* kt, const storage_t<DT>* vt, const Reader<DT, DP>& rd,
                                             float to_log2, int hi, uint64_t present = ~(uint64_t)0, int shift = 0) {
    constexpr bool SCORE = DT == DT_F32 || CAREFUL;  // m is a score
    const int g = rd.lane >> 5;
    float &m = sm.m, &l = sm.l;
    f32x16 s[2] = {};
#pragma unroll
    for (int c = 0; c < DP / 16; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t) s[t] = mma(rd.row_frag(kt, 32 * t, c), qf[c], s[t]);
    constexpr bool AHEAD = !SCORE;
    constexpr int P = DP / 16;  // products with v for 32 keys
    constexpr int F = 4;        // their values are read that many products ahead
    frag_t<DT> a[F];
    const auto values = [&](int n) { return rd.col_frag(vt, n / P * 32 + n % P / (DP / 32) * 16, n % (DP / 32)); };
    if (AHEAD) {
#pragma unroll
        for (int n = 0; n < F; ++n) a[n] = values(n);
    }
    if (DT != DT_F32) {
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int k = 0; k < DP / 8 - 4; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    }
    if (PART) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (32 * t + 8 * (r >> 2) + 4 * g + (r & 3) >= hi ||
                    (GAPS && !((present >> (4 * g)) >> (32 * t + 8 * (r >> 2) + (r & 3)) & 1)))
                    s[t][r] = -INFINITY;
    }
    // a NaN among the scores makes top NaN, and the row's results are NaN whatever m is
    float top = __builtin_elementwise_maximum(s[0][0], s[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r)
        top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(s[0][r], s[1][r]), top);
    const auto follow = [&](float now, float alpha) {
        m = now;
        l *= alpha;
        sm.rounded *= alpha;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
    };
    if constexpr (SCORE) {
        const float now = fmaxf(m, __builtin_elementwise_maximum(top, other_half(top)));
        follow(now, now == m ? 1.f : __builtin_amdgcn_exp2f((m - now) * to_log2));
    } else {
        // either half of the row says alone whether the reference has to follow
        const bool none = m == -INFINITY;
        const auto passes = [&](float x) {
            return none ? x > -INFINITY : fmaf(x, to_log2, -m) > kSlack<DT> + kBelow<DT>;
        };
        if (__any(passes(top))) {
            top = __builtin_elementwise_maximum(top, other_half(top));
            float now = passes(top) ? fmaf(top, to_log2, -kBelow<DT>) : m;
            if (now < -kCoarse) {
                sm.low |= now > -INFINITY;
                now = -INFINITY;  // (m is that, or passes() is false)
            }
            follow(now, now == m ? 1.f : __builtin_amdgcn_exp2f(m - now));
        }
    }
    const float ref = m == -INFINITY ? 0.f : m;  // nothing seen yet: every term is 0
    const auto term = [&](float x) {
        return __builtin_amdgcn_exp2f(SCORE ? fmaf(x - ref, to_log2, kBelow<DT>) : fmaf(x, to_log2, -ref));
    };
    if constexpr (AHEAD) {
        // The second 32 keys' terms are made between the first 32's products.
#pragma unroll
        for (int r = 0; r < 16; ++r) l += s[0][r] = term(s[0][r]);
        frag_t<DT> b[2] = {narrow<DT>(s[0], 0), narrow<DT>(s[0], 1)};
        sm.rounded = add_terms<DT>(b[1], add_terms<DT>(b[0], sm.rounded));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < 2 * P; ++n) {
            if (n == P) {
                b[0] = narrow<DT>(s[1], 0);
                b[1] = narrow<DT>(s[1], 1);
            }
            acc[n % (DP / 32)] = mma(a[n % F], b[n % P / (DP / 32)], acc[n % (DP / 32)]);
            if (n + F < 2 * P) a[n % F] = values(n + F);
            if (n < P) {
#pragma unroll
                for (int r = n * 16 / P; r < (n + 1) * 16 / P; ++r) s[1][r] = term(s[1][r]);
#pragma unroll
                for (int r = (n - 1) * 16 / P; n > 0 && r < n * 16 / P; ++r) l += s[1][r];
            } else if (n == P) {
#pragma unroll
                for (int r = (P - 1) * 16 / P; r < 16; ++r) l += s[1][r];
                sm.rounded = add_terms<DT>(b[1], add_terms<DT>(b[0], sm.rounded));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                l += s[t][r] = term(s[t][r]);
                if (CAREFUL && kScaled<DT>) s[t][r] = ldexpf(s[t][r], -shift);
            }
            const frag_t<DT> b[2] = {narrow<DT>(s[t], 0), narrow<DT>(s[t], 1)};
            if (DT != DT_F32) sm.rounded = add_terms<DT>(b[1], add_terms<DT>(b[0], sm.rounded));
            mma_rows<DT, DP, PART && CAREFUL>(acc, vt, rd, 32 * t, b, 0, hi);
        }
    }
}

}  // namespace kb
