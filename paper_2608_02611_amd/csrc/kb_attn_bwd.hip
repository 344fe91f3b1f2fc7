// kb_attn_bwd.hip -- softmax attention, backward.  With p_ij = exp(s_ij - lse_i),
// D_i = dout_i . o_i and t_ij = p_ij (dout_i . v_j - D_i):
//   dq_i = scale S_j t_ij k_j,  dk_j = scale S_i t_ij q_i,  dv_j = S_i p_ij dout_i.
//
// The probabilities are computed again, once where the keys stay and the
// queries pass (dk, dv: 4 products) and once where the queries stay and the
// keys pass (dq: 3 products).  The 2 products more than the 5 that are needed
// buy sums in registers: no atomics, no partial gradients in memory, the same
// bits on every call.
//
// F16 holds p and t of a long row badly (its least normal number is 6e-5), so
// they are scaled by powers of two before they are rounded: p, at most 1, by
// 2^10; t, at most 2 |dout| |v|, so that this bound comes to at most 2^15.
//
// Measured on an MI355X: 4 x 32 heads x 2047, dim 128, f16, causal: 590 us, of
// which, in the fastest passes of a trace, dk and dv take 336 and dq 241: 0.58
// PFLOP/s of the 5 products, 0.82 of the 7 that are done, where a large library
// product reaches 1.2.  Of its time the kernel for dk and dv has matrix instructions
// under way for 43% and LDS reads (at 128 bytes a clock) for 66% (each product of
// 32 x 32 reads one or two operands there; twice as many keys a wave would halve
// that, at 512 registers a lane).
#include <type_traits>

#include "kb_attn.hpp"

namespace kb {
namespace {

constexpr int kThreads = 256;
constexpr float kProbLog2 = 10.f;

// F16, before all else: the largest finite squared norm of each block of
// kNormBlock rows of v, 16 lanes a row.
template <int DT>
__global__ void __launch_bounds__(kThreads) attn_v_norms_kernel(AttnParams p, BackwardLayout l) {
    using T = storage_t<DT>;
    constexpr int N = Vec16<T>::N;
    __shared__ float largest[kThreads / 16];
    const int blocks = (p.len_k + kNormBlock - 1) / kNormBlock, id = (int)blockIdx.x;
    const int block = id % blocks, h = id / blocks % p.kv_heads, b = id / blocks / p.kv_heads;
    const int n = seq_len(p.k_lens, b, p.len_k), sub = threadIdx.x & 15;
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < kNormBlock / 16; ++k) {
        const int j = block * kNormBlock + k * 16 + (threadIdx.x >> 4);
        const T* x = (const T*)p.v.p + b * p.v.sb + h * p.v.sh + j * p.v.sl;
        float sq = 0.f;
        if (j < n && sub * N < p.dim) {
            const auto u = load_vec(x, sub * N, p.dim);
#pragma unroll
            for (int e = 0; e < N; ++e) sq = fmaf((float)u[e], (float)u[e], sq);
        }
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) sq += __shfl_xor(sq, s);
        if (sq < INFINITY) top = fmaxf(top, sq);
    }
    if (sub == 0) largest[threadIdx.x >> 4] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kThreads / 16; ++k) top = fmaxf(top, largest[k]);
        p.ws[l.v_norms + id] = top;
    }
}

// e with |x| < 2^e from the largest x^2 (0 for x = 0).
__device__ __forceinline__ int bound_exponent(float sq) {
    if (!(sq > 0.f)) return 0;
    const int ex = (int)(__float_as_uint(sq) >> 23) - 127;  // sq < 2^(ex + 1)
    return ((ex + 1) >> 1) + ((ex + 1) & 1);
}

// The largest of n values that are not negative, in every thread of a
// work-group; shared: a float for each wave.
__device__ __forceinline__ float block_max(const float* x, int64_t n, float* shared) {
    float top = 0.f;
    for (int64_t k = threadIdx.x; k < n; k += kThreads) top = fmaxf(top, x[k]);
    top = __uint_as_float(wave_max_u32(__float_as_uint(top)));
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(shared[0], shared[1]), fmaxf(shared[2], shared[3]));
    __syncthreads();
    return top;
}

// F16: 2^(14 - e), |t| < 2^(1 + e), from the squared norms of the rows of dout and
// v that enter.  (The exponent stays within binary32: the norm of an F16 row of
// 128 is under 2^20 and, if not 0, at least 2^-24.)
__device__ __forceinline__ float score_scale(float dout_sq, float v_sq) {
    return __uint_as_float((uint32_t)(127 + 14 - bound_exponent(dout_sq) - bound_exponent(v_sq)) << 23);
}

// dk and dv of 128 keys, 32 a wave.  The keys stay (key rows in registers, value
// rows in LDS, which leaves registers for two waves a SIMD) while the query
// rows of every head of the group pass in tiles of 32.
constexpr int kKeyRows = kAttnKeyRows;
constexpr int kQueries = kAttnQueries;

// Order of N products, each with READS of its own: those of AHEAD products are
// under way before the first product.
template <int N, int AHEAD, int READS = 1>
__device__ __forceinline__ void reads_ahead() {
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * READS, 0);
#pragma unroll
    for (int k = 0; k < N - AHEAD; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

// The exponent of a probability, in base 2, from a score s and the row's lse as
// row_lse gives it.  In 32 bits the difference comes first and is rounded once, so
// that its error does not grow with |lse| (scores near 5000: p to 7e-7 of itself,
// 1.5e-4 with lse / ln 2 rounded beforehand; 2 x 12 heads, 513 x 257: 98 us, 96 with
// that).  In 16 bits one instruction makes it, whose error, 2^-23 of |lse|, stays
// under f16's rounding up to an lse of 2^12.
template <int DT>
__device__ __forceinline__ float row_lse(float lse) {
    return DT == DT_F32 ? lse : lse * kLog2e;
}
template <int DT>
__device__ __forceinline__ float score_factor(float scale) {
    return DT == DT_F32 ? scale : scale * kLog2e;
}
template <int DT>
__device__ __forceinline__ float exponent(float s, float factor, float lse) {
    const float x = fmaf(s, factor, -lse);
    return DT == DT_F32 ? x * kLog2e : x;
}

// One tile of queries for a wave's 32 keys: s and t with a key a column.  PART:
// the lane's key is seen by the tile's queries from lo on.
template <int DT, int DP, bool PART, bool CAREFUL>
__device__ __forceinline__ void tile_keys(f32x16 (&dk)[DP / 32], f32x16 (&dv)[DP / 32], const frag_t<DT> (&kf)[DP / 16],
                                          const storage_t<DT>* vt, const storage_t<DT>* qt, const storage_t<DT>* dt,
                                          const float* rows, const Reader<DT, DP>& rd, float factor, float t_over_p,
                                          int lo) {
    const int g = rd.lane >> 5;
    f32x16 s = {}, t;
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {  // t starts from -D
        const f32x4 dot = *(const f32x4*)(rows + 8 * r4 + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) t[4 * r4 + e] = -dot[e];
    }
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        s = mma(rd.row_frag(qt, 0, c), kf[c], s);
        t = mma(rd.row_frag(dt, 0, c), rd.row_frag(vt, 0, c), t);
    }
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 lse = *(const f32x4*)(rows + kQueries + 8 * r4 + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 4 * r4 + e;
            // F16: the power of two of p goes into its exponent
            float x = exponent<DT>(s[r], factor, DT == DT_F16 ? lse[e] - kProbLog2 : lse[e]);
            if (PART) x = 8 * r4 + 4 * g + e >= lo ? x : -INFINITY;
            s[r] = __builtin_amdgcn_exp2f(x);
            t[r] = s[r] * t[r];
            if (DT == DT_F16) t[r] *= t_over_p;
            if (PART) t[r] = 8 * r4 + 4 * g + e >= lo ? t[r] : 0.f;
        }
    }
    const frag_t<DT> pf[2] = {narrow<DT>(s, 0), narrow<DT>(s, 1)}, tf[2] = {narrow<DT>(t, 0), narrow<DT>(t, 1)};
    mma_rows<DT, DP, PART && CAREFUL>(dv, dt, rd, 0, pf, lo, kQueries);
    mma_rows<DT, DP, PART && CAREFUL>(dk, qt, rd, 0, tf, lo, kQueries);
}

// CAREFUL: a launch of its own, for the work-groups that the first one marked (in
// the same kernel it would cost the first pass the registers that it needs).
template <int DT, int DP, bool WHOLE, bool CAREFUL>
__global__ void __launch_bounds__(kThreads, DT == DT_F32 || CAREFUL ? 1 : 2) attn_backward_keys_kernel(AttnParams p, BackwardLayout l) {
    const int part = (int)blockIdx.y;
    uint32_t* mark = (uint32_t*)(p.ws + l.marks) + (int64_t)part * gridDim.x + blockIdx.x;
    if (CAREFUL && *mark == 0) return;
    using T = storage_t<DT>;
    using L = Tile<DT, DP>;
    using F = Filler<DT, DP, kQueries, kThreads>;
    __shared__ __align__(16) T vt[L::size(kKeyRows)];
    __shared__ __align__(16) T qt[2][L::size(kQueries)];
    __shared__ __align__(16) T dt[2][L::size(kQueries)];
    __shared__ __align__(16) float rows[2][2 * kQueries];  // D, lse
    __shared__ float scratch[8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 5;
    const HeadBlock at = head_block(blockIdx.x, p.kv_heads, p.batch * p.kv_heads, (p.len_k + kKeyRows - 1) / kKeyRows);
    const int qlen = seq_len(p.q_lens, at.b, p.len_q), klen = seq_len(p.k_lens, at.b, p.len_k);
    const int first = at.block * kKeyRows, j = first + wave * 32 + (lane & 31);
    const bool live = j < klen;
    // F16: p is held 2^10 p
    const float p_scale = DT == DT_F16 ? __uint_as_float((127u + (uint32_t)kProbLog2) << 23) : 1.f;
    float t_scale = 1.f;
    if (DT == DT_F16) {
        const int64_t pair = (int64_t)at.b * p.kv_heads + at.h;
        const int64_t rows_of = ((int64_t)p.len_q * p.group + kAttnRows - 1) / kAttnRows;
        const int64_t keys_of = (p.len_k + kNormBlock - 1) / kNormBlock;
        const float dout_sq = block_max(p.ws + l.dout_norms + pair * rows_of, rows_of, scratch);
        t_scale = score_scale(dout_sq, block_max(p.ws + l.v_norms + pair * keys_of, keys_of, scratch));
    }
    const float t_over_p = t_scale / p_scale;

    const T* k = (const T*)p.k.p + at.b * p.k.sb + at.h * p.k.sh + (int64_t)j * p.k.sl;
    const T* v = (const T*)p.v.p + at.b * p.v.sb + at.h * p.v.sh;
    frag_t<DT> kf[DP / 16];
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) kf[c] = load_frag<DT, WHOLE>(k, c, g, p.dim, live);
    if (WHOLE) {
        const Filler<DT, DP, kAttnReach, kThreads> fv(p.v.sl, p.dim);
#pragma unroll
        for (int r = 0; r < kKeyRows; r += kAttnReach) fv.fill(vt + L::size(r), v, p.v.sl, first + r, klen, p.dim);
    } else {
        stage<DT, DP, kKeyRows, kThreads>(vt, v, p.v.sl, first, klen, p.dim);
    }

    // the queries that see a key: [sees(j), qlen)
    const auto sees = [&](int key) { return p.causal ? min(qlen, max(0, key - (klen - qlen))) : 0; };
    const int lo = sees(j);
    const int start = first < klen ? sees(first) / kQueries * kQueries : qlen;
    const bool wave_live = first + wave * 32 < klen;
    const int wave_lo = sees(first + wave * 32);
    const int block_hi = sees(first + kKeyRows - 1);  // from here on every key is seen
    const int steps = (qlen - start + kQueries - 1) / kQueries;  // tiles of one head

    const F fq(p.q.sl, p.dim), fd(p.dout.sl, p.dim);
    const T* q = (const T*)p.q.p + at.b * p.q.sb + at.h * p.group * p.q.sh;
    const T* dout = (const T*)p.dout.p + at.b * p.dout.sb + at.h * p.group * p.dout.sh;
    const float* row_values = p.ws + ((int64_t)at.b * p.heads + at.h * p.group) * p.len_q;
    const auto fill = [&](int h, int i0, int buf) {
        if (WHOLE) {
            fq.fill(qt[buf], q + h * p.q.sh, p.q.sl, i0, qlen, p.dim);
            fd.fill(dt[buf], dout + h * p.dout.sh, p.dout.sl, i0, qlen, p.dim);
        } else {
            stage<DT, DP, kQueries, kThreads>(qt[buf], q + h * p.q.sh, p.q.sl, i0, qlen, p.dim);
            stage<DT, DP, kQueries, kThreads>(dt[buf], dout + h * p.dout.sh, p.dout.sl, i0, qlen, p.dim);
        }
        if (wave == 0) {
            const float* from = row_values + (int64_t)h * p.len_q + i0;
            if (i0 + (lane & 31) >= qlen) rows[buf][lane] = lane < 32 ? 0.f : INFINITY;
            else if (lane < 32) send<4>(background(from), lane * 4, 0, rows[buf]);
            else send<4>(background(from + l.lse), (lane & 31) * 4, 0, rows[buf]);
        }
    };

    const Reader<DT, DP> rd(lane);
    const float factor = score_factor<DT>(p.scale);
    const T* v_rows = vt + wave * L::size(32);
    // the part's tiles of those of all heads, in their order
    const int64_t tiles = (int64_t)steps * p.group;
    const int64_t end = tiles * (part + 1) / p.key_parts;
    int64_t tile = tiles * part / p.key_parts;
    int h = steps ? (int)(tile / steps) : 0, i0 = steps ? start + (int)(tile % steps) * kQueries : 0, buf = 0;
    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    if (tile < end) fill(h, i0, 0);
    const auto next = [&] {
        tile_wait();
        __syncthreads();  // the tile is there, and the other one is read
        const bool last = i0 + kQueries >= qlen;
        if (tile + 1 < end) fill(last ? h + 1 : h, last ? start : i0 + kQueries, buf ^ 1);
    };
    for (; tile < end; ++h, i0 = start) {
        for (; tile < end && i0 < min(block_hi, qlen); i0 += kQueries, buf ^= 1, ++tile) {
            next();
            if (wave_live && i0 + kQueries > wave_lo)
                tile_keys<DT, DP, true, CAREFUL>(dk, dv, kf, v_rows, qt[buf], dt[buf], rows[buf], rd, factor, t_over_p,
                                                 lo - i0);
        }
        for (; tile < end && i0 < qlen; i0 += kQueries, buf ^= 1, ++tile) {
            next();
            if (wave_live) tile_keys<DT, DP, false, false>(dk, dv, kf, v_rows, qt[buf], dt[buf], rows[buf], rd, factor, t_over_p, 0);
        }
    }
    if (!CAREFUL && p.causal) {
        const int bad = __syncthreads_or(non_finite(dk) || non_finite(dv));
        if (threadIdx.x == 0) *mark = bad;
    }
    if (j >= p.len_k) return;
    const float k_scale = p.scale / t_scale, v_scale = 1.f / p_scale;
    if (p.key_parts > 1) {
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                dk[db][r] = live ? dk[db][r] * k_scale : 0.f;
                dv[db][r] = live ? dv[db][r] * v_scale : 0.f;
            }
        const int64_t keys = (int64_t)p.batch * p.kv_heads * p.len_k, dim = part_dim(p);
        const int64_t key = ((int64_t)at.b * p.kv_heads + at.h) * p.len_k + j;
        float* to = p.ws + l.dkv + (key * p.key_parts + part) * dim;
        store_part<DP>(to, dk, p.dim, g);
        store_part<DP>(to + keys * p.key_parts * dim, dv, p.dim, g);
        return;
    }
    store_column<DT, DP>((T*)p.dk.p + at.b * p.dk.sb + at.h * p.dk.sh + j * p.dk.sl, dk, k_scale, live, p.dim, g);
    store_column<DT, DP>((T*)p.dv.p + at.b * p.dv.sb + at.h * p.dv.sh + j * p.dv.sl, dv, v_scale, live, p.dim, g);
}

// dq of 128 query rows (row = query * group + head, as in the forward pass),
// 32 a wave, while the keys pass in tiles of 64.
constexpr int kRows = kAttnRows;
constexpr int kKeys = kAttnKeys;

// One tile of keys for a wave's 32 query rows; PART: the lane's row sees the
// tile's keys below hi, one of its rows those below seen.
template <int DT, int DP, bool PART, bool CAREFUL>
__device__ __forceinline__ void tile_queries(f32x16 (&dq)[DP / 32], const frag_t<DT> (&qf)[DP / 16],
                                             const frag_t<DT> (&df)[DP / 16], const storage_t<DT>* kt,
                                             const storage_t<DT>* vt, const Reader<DT, DP>& rd, float factor,
                                             float lse, float dot, int hi, int seen) {
    const int g = rd.lane >> 5;
#pragma unroll
    for (int u = 0; u < kKeys / 32; ++u) {
        if (PART && 32 * u >= seen) break;
        f32x16 s = {}, t = {};
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            s = mma(rd.row_frag(kt, 32 * u, c), qf[c], s);
            t = mma(rd.row_frag(vt, 32 * u, c), df[c], t);
        }
        if (DT != DT_F32 && !(PART && CAREFUL)) reads_ahead<DP / 8, 4>();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            t[r] = __builtin_amdgcn_exp2f(exponent<DT>(s[r], factor, lse)) * (t[r] - dot);
            if (PART) t[r] = 32 * u + 8 * (r >> 2) + 4 * g + (r & 3) < hi ? t[r] : 0.f;
        }
        const frag_t<DT> tf[2] = {narrow<DT>(t, 0), narrow<DT>(t, 1)};
        mma_rows<DT, DP, PART && CAREFUL>(dq, kt, rd, 32 * u, tf, 0, hi);
        if (DT != DT_F32 && !(PART && CAREFUL)) {
            reads_ahead<DP / 16, 3, 2>();
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

template <int DT, int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, DT == DT_F32 ? 1 : 2) attn_backward_queries_kernel(AttnParams p, BackwardLayout l) {
    using T = storage_t<DT>;
    using L = Tile<DT, DP>;
    using F = Filler<DT, DP, kKeys, kThreads>;
    __shared__ __align__(16) T kt[2][L::size(kKeys)];
    __shared__ __align__(16) T vt[2][L::size(kKeys)];
    __shared__ float scratch[8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5;
    const int n_blocks = pair_blocks(p);
    const HeadBlock at = head_block(blockIdx.x, p.kv_heads, p.batch * p.kv_heads, n_blocks);
    const uint32_t first = (uint32_t)(n_blocks - 1 - at.block) * kRows;
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
    const int part = (int)blockIdx.y;
    const int all = any ? key_limit(min(block_last, qlen - 1), qlen, klen, p.causal) : 0;
    const int tiles = (all + kKeys - 1) / kKeys;
    const int start = (int)((int64_t)tiles * part / p.parts) * kKeys;
    const int end = min(all, (int)((int64_t)tiles * (part + 1) / p.parts) * kKeys);

    const T* q = (const T*)p.q.p + at.b * p.q.sb + hq * p.q.sh + i * p.q.sl;
    const T* dout = (const T*)p.dout.p + at.b * p.dout.sb + hq * p.dout.sh + i * p.dout.sl;
    const T* k = (const T*)p.k.p + at.b * p.k.sb + at.h * p.k.sh;
    const T* v = (const T*)p.v.p + at.b * p.v.sb + at.h * p.v.sh;
    frag_t<DT> qf[DP / 16], df[DP / 16];
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        qf[c] = load_frag<DT, WHOLE>(q, c, g, p.dim, live);
        df[c] = load_frag<DT, WHOLE>(dout, c, g, p.dim, live);
    }
    // D_i and lse_i (row_lse), for here and for the keys' kernel.  A row with no
    // seen score has lse = -infinity, and its terms exp(-infinity - lse) are to be
    // 0: it gets 0.  A row of the padding gets +infinity, which makes its terms 0, and
    // so does one whose lse is held too coarsely for a term to be known even to a
    // factor of 2 (they would be 0 or infinite, and end up in the keys' gradients).
    const int64_t at_row = ((int64_t)at.b * p.heads + hq) * p.len_q + i;
    const T* o = (const T*)p.o.p + at.b * p.o.sb + hq * p.o.sh + i * p.o.sl;
    float dot = 0.f, sq = 0.f;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        const frag_t<DT> of = load_frag<DT, WHOLE>(o, c, g, p.dim, live);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dot = fmaf((float)df[c][e], (float)of[e], dot);
            if (DT == DT_F16) sq = fmaf((float)df[c][e], (float)df[c][e], sq);
        }
    }
    dot += other_half(dot);
    float lse = live ? p.lse[at_row] : INFINITY;
    lse = lse == -INFINITY ? 0.f : row_lse<DT>(lse);
    if (fabsf(lse) >= row_lse<DT>(kLn2 * 16777216.f)) lse = INFINITY;
    if (part == 0 && exists && g == 0) {
        p.ws[at_row] = dot;
        p.ws[l.lse + at_row] = lse;
    }
    float t_scale = 1.f;
    if (DT == DT_F16) {
        const int64_t pair = (int64_t)at.b * p.kv_heads + at.h, keys_of = (p.len_k + kNormBlock - 1) / kNormBlock;
        sq += other_half(sq);
        sq = sq < INFINITY ? sq : 0.f;
        t_scale = score_scale(sq, block_max(p.ws + l.v_norms + pair * keys_of, keys_of, scratch));
        lse -= __builtin_amdgcn_logf(t_scale);  // a power of two: it goes into the exponent
        if (part == 0) {
            const float top = __uint_as_float(wave_max_u32(__float_as_uint(sq)));
            if (lane == 0) scratch[wave] = top;
            __syncthreads();
            if (threadIdx.x == 0)
                p.ws[l.dout_norms + pair * n_blocks + n_blocks - 1 - at.block] =
                    fmaxf(fmaxf(scratch[0], scratch[1]), fmaxf(scratch[2], scratch[3]));
        }
    }

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
    const Reader<DT, DP> rd(lane);
    const float factor = score_factor<DT>(p.scale);
    f32x16 dq[DP / 32];
    const auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) dq[db] = f32x16{};
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
            if (wave_any > 0) tile_queries<DT, DP, false, false>(dq, qf, df, kt[buf], vt[buf], rd, factor, lse, dot, 0, 0);
        }
        for (; j0 < end; j0 += kKeys, buf ^= 1) {
            next();
            if (j0 < wave_any)
                tile_queries<DT, DP, true, CAREFUL>(dq, qf, df, kt[buf], vt[buf], rd, factor, lse, dot, lim - j0, wave_any - j0);
        }
    };
    pass(std::false_type{});
    if (p.causal && __syncthreads_or(non_finite(dq))) pass(std::true_type{});
    if (!exists) return;
    if (p.parts > 1) {
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) dq[db][r] = live ? dq[db][r] * (p.scale / t_scale) : 0.f;
        store_part<DP>(p.ws + l.dq + (at_row * p.parts + part) * part_dim(p), dq, p.dim, g);
        return;
    }
    store_column<DT, DP>((T*)p.dq.p + at.b * p.dq.sb + hq * p.dq.sh + i * p.dq.sl, dq, p.scale / t_scale, live, p.dim, g);
}

// Sums over the parts, in their order.  A thread has four elements of a row; the
// rows of dq come first, then those of dk, then of dv.
template <int DT>
__global__ void __launch_bounds__(kThreads) attn_backward_join_kernel(AttnParams p, BackwardLayout l) {
    using T = storage_t<DT>;
    const int quads = (p.dim + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    int64_t row = id / quads;
    const int d = (int)(id % quads) * 4;
    const int64_t q_rows = p.parts > 1 ? (int64_t)p.batch * p.heads * p.len_q : 0;
    const int64_t k_rows = p.key_parts > 1 ? (int64_t)p.batch * p.kv_heads * p.len_k : 0;
    if (row >= q_rows + 2 * k_rows) return;
    const bool is_q = row < q_rows;
    if (!is_q) row -= q_rows;
    const bool is_v = !is_q && row >= k_rows;
    const int parts = is_q ? p.parts : p.key_parts;
    const float* in = p.ws + (is_q ? l.dq : l.dkv) + row * parts * part_dim(p) + d;
    f32x4 sum = *(const f32x4*)in;
    for (int k = 1; k < parts; ++k) {
        const f32x4 x = *(const f32x4*)(in + k * part_dim(p));
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += x[e];
    }
    if (is_v) row -= k_rows;
    const int len = is_q ? p.len_q : p.len_k, heads = is_q ? p.heads : p.kv_heads;
    const int i = (int)(row % len), h = (int)(row / len % heads), b = (int)(row / len / heads);
    const HeadView& to = is_q ? p.dq : is_v ? p.dv : p.dk;
    store_quad<DT>((T*)to.p + b * to.sb + h * to.sh + i * to.sl, d, p.dim, sum[0], sum[1], sum[2], sum[3]);
}

template <int DT, int DP, bool WHOLE>
hipError_t backward(const AttnParams& p, hipStream_t stream) {
    const BackwardLayout l = backward_layout(p);
    const int64_t pairs = (int64_t)p.batch * p.kv_heads;
    const int64_t v_blocks = pairs * ((p.len_k + (int64_t)kNormBlock - 1) / kNormBlock);
    if (DT == DT_F16 && v_blocks > 0) attn_v_norms_kernel<DT><<<dim3((unsigned)v_blocks), kThreads, 0, stream>>>(p, l);
    if (row_blocks(p) > 0)
        attn_backward_queries_kernel<DT, DP, WHOLE>
            <<<dim3((unsigned)row_blocks(p), (unsigned)p.parts), kThreads, 0, stream>>>(p, l);
    if (key_blocks(p) > 0) {
        const dim3 grid((unsigned)key_blocks(p), (unsigned)p.key_parts);
        attn_backward_keys_kernel<DT, DP, WHOLE, false><<<grid, kThreads, 0, stream>>>(p, l);
        if (p.causal) attn_backward_keys_kernel<DT, DP, WHOLE, true><<<grid, kThreads, 0, stream>>>(p, l);
    }
    const int64_t join_rows = (p.parts > 1 ? (int64_t)p.batch * p.heads * p.len_q : 0) +
                              (p.key_parts > 1 ? 2 * pairs * p.len_k : 0);
    if (join_rows > 0) {
        const int64_t quads = join_rows * ((p.dim + 3) / 4);
        attn_backward_join_kernel<DT><<<dim3((unsigned)((quads + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(p, l);
    }
    return hipGetLastError();
}

template <int DT, int DP>
hipError_t backward(const AttnParams& p, hipStream_t stream) {
    return p.whole ? backward<DT, DP, true>(p, stream) : backward<DT, DP, false>(p, stream);
}

template <int DT>
hipError_t backward(const AttnParams& p, hipStream_t stream) {
    if (p.dim <= 64) return backward<DT, 64>(p, stream);
    if (p.dim <= 96) return backward<DT, 96>(p, stream);
    return backward<DT, 128>(p, stream);
}

}  // namespace

hipError_t launch_attn_backward(int dtype, const AttnParams& p, hipStream_t stream) {
    if (dtype == DT_F32) return backward<DT_F32>(p, stream);
    if (dtype == DT_F16) return backward<DT_F16>(p, stream);
    return backward<DT_BF16>(p, stream);
}

}  // namespace kb
