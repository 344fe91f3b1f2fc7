// kb_attn_fwd.hip -- softmax attention, forward: for query i over the keys j
// that it sees, s_j = scale q_i . k_j, lse = log S(exp s_j),
// o = S(exp(s_j - lse) v_j).
//
// One pass over the keys with the running maximum m and sum l of the softmax:
// a tile's terms are exp(s_j - m) for the new maximum, and what was summed
// before is scaled by exp(m_old - m).  A work-group takes 128 query rows, 32 a
// wave; the query heads that share a key head are rows of the same work-group
// (row = query * group + head), so that a tile of keys serves all of them.
//
// Measured on an MI355X: 4 x 32 heads x 2047, dim 128, f16, causal: 183 us, 0.75
// PFLOP/s, where a large library product of 16-bit matrices reaches 1.2 (both are
// held back by power: on zeros 146 us, and 1.8 PFLOP/s).  Matrix instructions are
// under way 43% of the time, vector ones and LDS reads (at 128 bytes a clock) each
// for about as long: what is lost is the softmax that no product runs beside.  512
// queries on 16,384 keys: 147 us, 0.92 PFLOP/s.  Single tokens
// (16 ragged sequences of up to 8191 keys, 32 heads on 8): 91 us, 4.4 TB/s, where a
// large copy moves 4.8.
#include <cfloat>
#include <type_traits>

#include "kb_attn.hpp"

namespace kb {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = kAttnRows;
constexpr int kKeys = kAttnKeys;

// The softmax state of a lane's query over the tiles so far: terms are exp(scale
// (s - m)).  In 32 bits m is the maximum.  In 16 bits it is a reference, held as
// scale m / ln 2 (one instruction makes a term's exponent), that follows the
// maximum only when a term would pass 2^kSlack of the one that set it (scaling the
// sums takes as long as a quarter of a tile's products), and next to l, the sum of
// the terms, there is the sum of the rounded terms, those whose product with v is
// divided by it: where one term outweighs the others, o is its v to the last bit.
// F16 holds small terms badly (subnormal from 2^-14, nothing under 2^-25), so there
// the reference is set 2^kBelow under the maximum: terms of up to 2^15, and what the
// format takes from one is at most 2^-34 of the largest.
template <int DT>
constexpr float kSlack = DT == DT_F16 ? 6.f : 8.f;
template <int DT>
constexpr float kBelow = DT == DT_F16 ? 9.f : 0.f;
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
// pairs are not seen; the lane's row sees the tile's keys below hi.  CAREFUL: m is
// the largest score, as in 32 bits, and mma_seen for rows that are not seen.
template <int DT, int DP, bool PART, bool CAREFUL>
__device__ __forceinline__ void tile_forward(f32x16 (&acc)[DP / 32], Softmax& sm, const frag_t<DT> (&qf)[DP / 16],
                                             const storage_t<DT>* kt, const storage_t<DT>* vt, const Reader<DT, DP>& rd,
                                             float to_log2, int hi) {
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
                if (32 * t + 8 * (r >> 2) + 4 * g + (r & 3) >= hi) s[t][r] = -INFINITY;
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
            for (int r = 0; r < 16; ++r) l += s[t][r] = term(s[t][r]);
            const frag_t<DT> b[2] = {narrow<DT>(s[t], 0), narrow<DT>(s[t], 1)};
            if (DT != DT_F32) sm.rounded = add_terms<DT>(b[1], add_terms<DT>(b[0], sm.rounded));
            mma_rows<DT, DP, PART && CAREFUL>(acc, vt, rd, 32 * t, b, 0, hi);
        }
    }
}

template <int DT, int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, DT == DT_F32 ? 1 : 2) attn_forward_kernel(AttnParams p) {
    using T = storage_t<DT>;
    using L = Tile<DT, DP>;
    using F = Filler<DT, DP, kKeys, kThreads>;
    __shared__ __align__(16) T kt[2][L::size(kKeys)];
    __shared__ __align__(16) T vt[2][L::size(kKeys)];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5;
    const int part = (int)blockIdx.y;
    const int n_blocks = pair_blocks(p);
    const HeadBlock at = head_block(blockIdx.x, p.kv_heads, p.batch * p.kv_heads, n_blocks);
    const uint32_t first = (uint32_t)(n_blocks - 1 - at.block) * kRows;  // causal: the longest first
    const int qlen = seq_len(p.q_lens, at.b, p.len_q), klen = seq_len(p.k_lens, at.b, p.len_k);

    const uint32_t row = first + wave * 32 + (lane & 31);
    const int i = (int)(row / p.group), hq = at.h * p.group + (int)(row % p.group);
    const bool exists = i < p.len_q, live = i < qlen;
    const int wave_first = __builtin_amdgcn_readfirstlane((int)((first + wave * 32) / p.group));
    const int wave_last = __builtin_amdgcn_readfirstlane((int)((first + wave * 32 + 31) / p.group));
    const int block_last = (int)((first + kRows - 1) / p.group);
    const bool any = (int)(first / p.group) < qlen;
    const int lim = key_limit(min(i, qlen - 1), qlen, klen, p.causal);
    const int wave_any = wave_first < qlen ? key_limit(min(wave_last, qlen - 1), qlen, klen, p.causal) : 0;
    const int block_all = any ? key_limit(min((int)(first / p.group), qlen - 1), qlen, klen, p.causal) : 0;
    // the part's tiles of those that the work-group's rows see
    const int all = any ? key_limit(min(block_last, qlen - 1), qlen, klen, p.causal) : 0;
    const int tiles = (all + kKeys - 1) / kKeys;
    const int start = (int)((int64_t)tiles * part / p.parts) * kKeys;
    const int end = min(all, (int)((int64_t)tiles * (part + 1) / p.parts) * kKeys);

    const T* q = (const T*)p.q.p + at.b * p.q.sb + hq * p.q.sh + i * p.q.sl;
    const T* k = (const T*)p.k.p + at.b * p.k.sb + at.h * p.k.sh;
    const T* v = (const T*)p.v.p + at.b * p.v.sb + at.h * p.v.sh;
    frag_t<DT> qf[DP / 16];
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) qf[c] = load_frag<DT, WHOLE>(q, c, g, p.dim, live);
    const Reader<DT, DP> rd(lane);
    const F fk(p.k.sl, p.dim), fv(p.v.sl, p.dim);
    const auto fill = [&](int j0, int buf) {
        if (WHOLE) {
            fk.fill(kt[buf], k, p.k.sl, j0, klen, p.dim);
            fv.fill(vt[buf], v, p.v.sl, j0, klen, p.dim);
        } else {
            stage<DT, DP, kKeys, kThreads>(kt[buf], k, p.k.sl, j0, klen, p.dim);
            stage<DT, DP, kKeys, kThreads>(vt[buf], v, p.v.sl, j0, klen, p.dim);
        }
    };

    const float to_log2 = p.scale * kLog2e;
    f32x16 acc[DP / 32];
    Softmax sm;
    const auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) acc[db] = f32x16{};
        sm = Softmax{};
        if (start < end) fill(start, 0);
        int j0 = start, buf = 0;
        const auto next = [&] {
            tile_wait();
            __syncthreads();  // the tile is there, and the other one is read
            if (j0 + kKeys < end) fill(j0 + kKeys, buf ^ 1);
        };
        // first the tiles that every row of the work-group sees whole
        for (; j0 + kKeys <= min(block_all, end); j0 += kKeys, buf ^= 1) {
            next();
            if (wave_any > 0)
                tile_forward<DT, DP, false, CAREFUL && DT != DT_F32>(acc, sm, qf, kt[buf], vt[buf], rd, to_log2, 0);
        }
        for (; j0 < end; j0 += kKeys, buf ^= 1) {
            next();
            if (j0 < wave_any) tile_forward<DT, DP, true, CAREFUL>(acc, sm, qf, kt[buf], vt[buf], rd, to_log2, lim - j0);
        }
    };
    pass(std::false_type{});
    if constexpr (DT == DT_F32) {
        if (p.causal && __syncthreads_or(non_finite(acc))) pass(std::true_type{});
    } else if (__syncthreads_or((p.causal && non_finite(acc)) || too_coarse(sm))) {
        pass(std::true_type{});
        if (sm.m > -INFINITY) sm.m = __builtin_amdgcn_fmed3f(fmaf(sm.m, to_log2, -kBelow<DT>), -FLT_MAX, FLT_MAX);
    }
    if (!exists) return;
    const float l = sm.l + other_half(sm.l), rounded = sm.rounded + other_half(sm.rounded);
    if (p.parts > 1) {
        const int64_t dim = part_dim(p);
        float* to = p.ws + ((((int64_t)at.b * p.kv_heads + at.h) * p.len_q * p.group + row) * p.parts + part) * (dim + 4);
        if (g == 0) *(f32x4*)(to + dim) = f32x4{live ? sm.m : -INFINITY, live ? l : 0.f, live ? rounded : 0.f, 0.f};
        store_part<DP>(to, acc, p.dim, g);
        return;
    }
    const bool some = live && l != 0.f;  // NaN too: it goes on to o
    store_column<DT, DP>((T*)p.o.p + at.b * p.o.sb + hq * p.o.sh + i * p.o.sl, acc, 1.f / (DT == DT_F32 ? l : rounded), some, p.dim, g);
    if (g == 0)
        p.lse[((int64_t)at.b * p.heads + hq) * p.len_q + i] =
            some ? fmaf(sm.m, unit_natural<DT>(p.scale), kLn2 * __builtin_amdgcn_logf(l)) : -INFINITY;
}

// The parts of a row joined: each part's sums are relative to its own m.  A
// thread has four elements of a row.
template <int DT>
__global__ void __launch_bounds__(kThreads) attn_join_kernel(AttnParams p) {
    using T = storage_t<DT>;
    const int quads = (p.dim + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t row = id / quads;  // [batch][key head][query][head of the group]
    const int d = (int)(id % quads) * 4;
    if (row >= (int64_t)p.batch * p.heads * p.len_q) return;
    const int64_t stride = part_dim(p) + 4;
    const float* in = p.ws + row * p.parts * stride;
    float m = -INFINITY;
    for (int s = 0; s < p.parts; ++s) m = fmaxf(m, in[s * stride + stride - 4]);
    const float shift = m == -INFINITY ? 0.f : m;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f, rounded = 0.f;
    for (int s = 0; s < p.parts; ++s) {
        const f32x4 stat = *(const f32x4*)(in + s * stride + stride - 4), x = *(const f32x4*)(in + s * stride + d);
        const float w = __builtin_amdgcn_exp2f((stat[0] - shift) * unit_log2<DT>(p.scale));
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(w, x[e], acc[e]);
        l = fmaf(w, stat[1], l);
        rounded = fmaf(w, stat[2], rounded);
    }
    const int64_t per_head = (int64_t)p.len_q * p.group;
    const int pair = (int)(row / per_head), in_head = (int)(row % per_head);
    const int b = pair / p.kv_heads, hq = pair % p.kv_heads * p.group + in_head % p.group, i = in_head / p.group;
    const bool some = l != 0.f;
    const float f = some ? 1.f / (DT == DT_F32 ? l : rounded) : 0.f;
    store_quad<DT>((T*)p.o.p + b * p.o.sb + hq * p.o.sh + i * p.o.sl, d, p.dim, some ? acc[0] * f : 0.f,
                   some ? acc[1] * f : 0.f, some ? acc[2] * f : 0.f, some ? acc[3] * f : 0.f);
    if (d == 0)
        p.lse[((int64_t)b * p.heads + hq) * p.len_q + i] = some ? fmaf(m, unit_natural<DT>(p.scale), kLn2 * __builtin_amdgcn_logf(l)) : -INFINITY;
}

template <int DT, int DP>
hipError_t forward(const AttnParams& p, hipStream_t stream) {
    const int64_t blocks = ((int64_t)p.len_q * p.group + kRows - 1) / kRows * p.batch * p.kv_heads;
    const dim3 grid((unsigned)blocks, (unsigned)p.parts);
    if (p.whole)
        attn_forward_kernel<DT, DP, true><<<grid, kThreads, 0, stream>>>(p);
    else
        attn_forward_kernel<DT, DP, false><<<grid, kThreads, 0, stream>>>(p);
    if (p.parts > 1) {
        const int64_t quads = (int64_t)p.batch * p.heads * p.len_q * ((p.dim + 3) / 4);
        attn_join_kernel<DT><<<dim3((unsigned)((quads + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(p);
    }
    return hipGetLastError();
}

template <int DT>
hipError_t forward(const AttnParams& p, hipStream_t stream) {
    if (p.dim <= 64) return forward<DT, 64>(p, stream);
    if (p.dim <= 96) return forward<DT, 96>(p, stream);
    return forward<DT, 128>(p, stream);
}

}  // namespace

hipError_t launch_attn_forward(int dtype, const AttnParams& p, hipStream_t stream) {
    if (dtype == DT_F32) return forward<DT_F32>(p, stream);
    if (dtype == DT_F16) return forward<DT_F16>(p, stream);
    return forward<DT_BF16>(p, stream);
}

}  // namespace kb
