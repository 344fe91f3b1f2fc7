// kb_paged.hpp -- device helpers of the paged cache: which sequence a token
// belongs to, and where its keys lie.
#pragma once

#include "kb_ops.hpp"

namespace kb {

// n / p.page for 0 <= n < 2^31.
__device__ __forceinline__ int page_of(const PagedParams& p, int n) {
    return (int)(__umulhi((uint32_t)(n + p.page_add), p.page_mul) >> p.page_shift);
}

// Elements from page 0's first row to that of place `at` in a page.
__device__ __forceinline__ int64_t row_offset(const HeadView& c, int page, int at) {
    const uint64_t of_page = (uint64_t)(uint32_t)page * (uint32_t)c.sb + ((uint64_t)((uint32_t)page * (uint32_t)((uint64_t)c.sb >> 32)) << 32);
    return (int64_t)(of_page + (uint64_t)(uint32_t)at * (uint32_t)c.sl + ((uint64_t)((uint32_t)at * (uint32_t)((uint64_t)c.sl >> 32)) << 32));
}

// Keys of sequence b, its new tokens' included.
__device__ __forceinline__ int paged_len(const PagedParams& p, int b) {
    return min(max(p.lens[b], 0), p.width * p.page);
}

// The tokens [first, first + n) of sequence b.
struct Tokens {
    int first, n;
};
__device__ __forceinline__ Tokens tokens_of(const PagedParams& p, int b) {
    if (p.starts == nullptr) return {b, 1};
    const int first = min(max(p.starts[b], 0), p.tokens), end = min(max(p.starts[b + 1], 0), p.tokens);
    return {first, max(0, end - first)};
}

// Its tokens and its keys.
struct Sequence {
    int first, n, len;
};
__device__ __forceinline__ Sequence sequence_of(const PagedParams& p, int b) {
    const Tokens t = tokens_of(p, b);
    return {t.first, t.n, paged_len(p, b)};
}

// Number of the first block of `ROWS` query rows of sequence b (paged_blocks).
template <int ROWS>
__device__ __forceinline__ int64_t block_before(const PagedParams& p, int b) {
    return (int64_t)(p.starts ? min(max(p.starts[b], 0), p.tokens) : b) * p.group / ROWS + b;
}

// How many of `n` ascending values f(0 .. n - 1) are at most x: 64 are looked at
// at once, one a lane.
template <typename F>
__device__ __forceinline__ int count_up_to(int n, int64_t x, int lane, const F& f) {
    int from = 0;
    for (int left = n; left > 0;) {  // (left shrinks: step < left, or it is the last round)
        const int step = (left + 63) / 64, at = (lane + 1) * step - 1;
        const bool below = at < left && f(from + at) <= x;
        const int whole = __popcll(__ballot(below));
        from += whole * step;
        left = min(step - 1, left - whole * step);
    }
    return from;
}

}  // namespace kb
