// kb_attn_paged.hip -- softmax attention of new tokens over a paged cache: query
// i of a sequence's Q new tokens, with K keys in the cache, sees (causal) keys
// j <= i + K - Q; s_j = scale q_i . k_j, lse = log S(exp s_j),
// o = S(exp(s_j - lse) v_j).
//
// Few rows a sequence (rows: queries x heads of the group; single tokens): bound by
// the bytes of the keys and values, each read once.  All tiles of 64 keys of all
// (sequence, key head, block of rows) pairs are numbered one behind the other, and
// each work-group takes the same number of them, whatever the sequences' lengths
// are; the pairs that this cuts are joined by a second kernel.  Many rows: bound by
// the matrix products; work-groups of 128 rows over tiles in LDS, as in the
// attention over dense keys.
//
// Measured on an MI355X, where a large copy moves 4.8 TB/s and a large library
// product of bf16 matrices reaches 1.15 to 1.23 PFLOP/s (32 heads on 8, dim 128): one
// token each of 64 sequences of up to 8191 keys, pages of 16, bf16: 143 us, 5.1 TB/s;
// one of 131,071 keys, f16: 100 us, 5.4 TB/s; five each of 32 sequences of up to 4000
// keys: 52 us, 3.5 TB/s, of which the second kernel has 6 and the beginnings of short
// pairs most of what is lost; 6 packed prompts of up to 4095 tokens: 282 to 315 us, 0.76
// to 0.85 PFLOP/s, by the clock that the card holds (7% to 13% more than dense keys:
// products under way 42% of the time, as there, and 100 more instructions for a tile's
// addresses).  8 heads' 200 keys of 64 elements, f32: 9.3 us, four steps behind each
// other on each wave.
#include <cfloat>
#include <type_traits>

#include "kb_attn_tile.hpp"
#include "kb_paged.hpp"

namespace kb {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kKeys = kPagedTile;
static_assert(kKeys == 16 * kWaves, "a wave has 16 keys of a tile");

// What a key's row is at: its page, or -1, and its place there.
struct Place {
    int page, at;
};
__device__ __forceinline__ Place place_of(const PagedParams& p, const int32_t* table, int key, int end) {
    Place w{-1, 0};
    if (key < end) {
        const int n = page_of(p, key);
        w.page = table[n];
        w.at = key - n * p.page;
    }
    return w;
}
__device__ __forceinline__ bool in_cache(const PagedParams& p, int page) { return (uint32_t)page < (uint32_t)p.pages; }

// ---------------------------------------------------------------- few rows --
//
// A wave has 16 keys of a tile and all 16 NB rows.  Scores are 16 x 16 products
// K Q^T: lane l (c = l % 16, g = l / 16) gives key c's elements and has the scores
// of row c with keys 4g .. 4g+3.  Those are, without moving, the right operand of
// 16 x 16 products V^T P over 16 keys, whose left operand is of keys 4g .. 4g+3 at
// element c: a lane reads VB elements of these four keys' rows and pairs them up in
// registers; product e takes element VB c + e, so that a lane's results are 4 VB
// elements of row c in a row.  Nothing passes through LDS, and no wave waits for
// another, until a pair's sums are joined.  Pages of other sizes than multiples of 16
// look every row up by itself (pages of 8: single tokens of up to 8191 keys the same 143
// us, the five drafted tokens 58 for 52).

template <int DT>
__device__ __forceinline__ f32x4 mma16(frag_t<DT> a, frag_t<DT> b, f32x4 c) {
    if constexpr (DT == DT_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
template <int DT>
struct Four {
    typedef storage_t<DT> type __attribute__((ext_vector_type(4)));
};
template <int DT>
using four_t = typename Four<DT>::type;
__device__ __forceinline__ f32x4 mma4(four_t<DT_F16> a, four_t<DT_F16> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma4(four_t<DT_BF16> a, four_t<DT_BF16> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma4(four_t<DT_F32> a, four_t<DT_F32> b, f32x4 c) {
#pragma unroll
    for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], b[k], c, 0, 0, 0);
    return c;
}

// N words of a row from element d on, zeros past dim or if !in.  WHOLE: rows are
// aligned and these elements lie within dim or past it.
template <int DT, int N, bool WHOLE>
__device__ __forceinline__ void load_words(const storage_t<DT>* row, int d, int dim, bool in, uint32_t (&out)[N]) {
    using T = storage_t<DT>;
    constexpr int W = 4 / (int)sizeof(T), M = N < 4 ? N : 4;  // elements of a word, words of a load
    typedef uint32_t words __attribute__((ext_vector_type(M), aligned(WHOLE ? 4 * M : sizeof(T))));
    typedef T elements __attribute__((ext_vector_type(M * W)));
#pragma unroll
    for (int k = 0; k < N; k += M) {
        const int at = d + k * W;
        words v = {};
        if (in && at + M * W <= dim) {
            v = *(const words*)(row + at);
        } else if (!WHOLE && in && at < dim) {
            elements x = {};
#pragma unroll
            for (int e = 0; e < M * W; ++e)
                if (at + e < dim) x[e] = row[at + e];
            v = __builtin_bit_cast(words, x);
        }
#pragma unroll
        for (int e = 0; e < M; ++e) out[k + e] = v[e];
    }
}

// What is the same in all lanes, so that the compiler sees it.
__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)((uint64_t)v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// The 16 keys of a wave's step, in registers.
template <int DT, int DP>
struct Step {
    using T = storage_t<DT>;
    static constexpr int KB = 16 / (int)sizeof(T);  // elements of a key that a lane has in a row, 4 KB apart
    static constexpr int KC = DP / (4 * KB);
    static constexpr int VB = DP / 16;
    static constexpr int VW = VB * (int)sizeof(T) / 4;
    uint32_t k[KC][4], v[4][VW];
    uint32_t seen;  // bit c: key c is there

    // The keys of 16 places, lane c knowing key c's.  (WHOLE: load_words.)
    template <bool WHOLE>
    __device__ __forceinline__ void load(const PagedParams& p, const T* kc, const T* vc, Place w, int lane) {
        const int c = lane & 15, g = lane >> 4;
        const bool have = in_cache(p, w.page);
        seen = (uint32_t)__ballot(have) & 0xFFFFu;
        const T* kr = kc + (have ? row_offset(p.cache[0], w.page, w.at) : 0);
#pragma unroll
        for (int n = 0; n < KC; ++n) load_words<DT, 4, WHOLE>(kr, (4 * n + g) * KB, p.dim, have, k[n]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int page = __shfl(w.page, 4 * g + j), at = __shfl(w.at, 4 * g + j);
            const bool in = in_cache(p, page);
            const T* vr = vc + (in ? row_offset(p.cache[1], page, at) : 0);
            load_words<DT, VW, WHOLE>(vr, VB * c, p.dim, in, v[j]);
        }
    }
    // The same where the 16 keys lie in one page: kr, vr: row 0 of them, of which
    // `rows` are there; at: where the lane reads (StepPlaces).  The bounds of a buffer
    // descriptor make zeros of the other rows.
    __device__ __forceinline__ void load_page(const T* kr, const T* vr, int rows, uint32_t k_row, uint32_t v_row,
                                              const uint32_t (&k_at)[KC], const uint32_t (&v_at)[4][(VW + 3) / 4]) {
        rows = __builtin_amdgcn_readfirstlane(rows);
        seen = (1u << rows) - 1u;
        const auto kd = __builtin_amdgcn_make_buffer_rsrc((void*)uniform((int64_t)kr), 0, rows * k_row, 0x00020000);
        const auto vd = __builtin_amdgcn_make_buffer_rsrc((void*)uniform((int64_t)vr), 0, rows * v_row, 0x00020000);
#pragma unroll
        for (int n = 0; n < KC; ++n) {
            const u32v4 x = __builtin_bit_cast(u32v4, __builtin_amdgcn_raw_buffer_load_b128(kd, (int)k_at[n], 0, 0));
#pragma unroll
            for (int e = 0; e < 4; ++e) k[n][e] = x[e];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < (VW + 3) / 4; ++n) {
                if constexpr (VW >= 4) {
                    const u32v4 x = __builtin_bit_cast(u32v4, __builtin_amdgcn_raw_buffer_load_b128(vd, (int)v_at[j][n], 0, 0));
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[j][4 * n + e] = x[e];
                } else {
                    typedef uint32_t two __attribute__((ext_vector_type(2)));
                    const two x = __builtin_bit_cast(two, __builtin_amdgcn_raw_buffer_load_b64(vd, (int)v_at[j][n], 0, 0));
#pragma unroll
                    for (int e = 0; e < 2; ++e) v[j][e] = x[e];
                }
            }
    }
    // Element e of the four keys' pieces.
    __device__ __forceinline__ four_t<DT> values(int e) const {
        if constexpr (DT == DT_F32) {
            return four_t<DT>{__uint_as_float(v[0][e]), __uint_as_float(v[1][e]), __uint_as_float(v[2][e]),
                              __uint_as_float(v[3][e])};
        } else {
            const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;  // the high halves of two words, or the low ones
            typedef uint32_t two __attribute__((ext_vector_type(2)));
            return __builtin_bit_cast(four_t<DT>, two{__builtin_amdgcn_perm(v[1][e / 2], v[0][e / 2], pick),
                                                      __builtin_amdgcn_perm(v[3][e / 2], v[2][e / 2], pick)});
        }
    }
};

// 16 bits: infinities and NaN as 0.
template <int DT>
__device__ __forceinline__ four_t<DT> finite_ones(four_t<DT> v) {
    typedef uint16_t bits __attribute__((ext_vector_type(4)));
    constexpr uint16_t kExponent = DT == DT_F16 ? 0x7C00 : 0x7F80;
    bits u = __builtin_bit_cast(bits, v);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if ((u[k] & kExponent) == kExponent) u[k] = 0;
    return __builtin_bit_cast(four_t<DT>, u);
}

// Elements of a row of K or Q as an operand of their product.
template <int DT>
__device__ __forceinline__ f32x4 mma_scores(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 c) {
    const u32v4 x = {a[0], a[1], a[2], a[3]}, y = {b[0], b[1], b[2], b[3]};
    if constexpr (DT == DT_F32) return mma4(__builtin_bit_cast(four_t<DT>, x), __builtin_bit_cast(four_t<DT>, y), c);
    else return mma16<DT>(__builtin_bit_cast(frag_t<DT>, x), __builtin_bit_cast(frag_t<DT>, y), c);
}

// The softmax state of a lane's row, for each of the NB blocks of 16: terms are
// exp(scale (s - m)), F16's 2^kBelow of that so that small ones keep their bits, m a
// score that follows the maximum when a term would pass 2^kSlack; l: their sum over
// the lane's keys.
// Where the sums of term times value end up large (kLarge), the pair is computed once
// more, CAREFUL: m is the maximum, and terms go into these sums times 2^-shift.  In 16
// bits an infinite value then counts in the product with a term's first part alone: its
// second part is 0, or negative where the first one was rounded up, which would make a
// NaN of the infinity.
template <int NB>
struct Rows {
    float m[NB], l[NB];
};

template <int DT, int DP, int NB, bool CAREFUL>
__device__ __forceinline__ void step_forward(f32x4 (&acc)[NB][DP / 16], Rows<NB>& st,
                                             const uint32_t (&q)[NB][Step<DT, DP>::KC][4],
                                             const Step<DT, DP>& in, float to_log2, const int (&lim)[NB], int key0,
                                             int every, int lane, int shift = 0) {
    using T = storage_t<DT>;
    using S = Step<DT, DP>;
    const int g = lane >> 4;
    f32x4 s[NB] = {};
#pragma unroll
    for (int n = 0; n < S::KC; ++n)
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = mma_scores<DT>(in.k[n], q[b][n], s[b]);
    const bool full = in.seen == 0xFFFFu && key0 + 16 <= every;  // every row sees every key
    if (!full) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!(in.seen >> (4 * g + r) & 1) || key0 + 4 * g + r >= lim[b]) s[b][r] = -INFINITY;
    }
    four_t<DT> hi[NB], lo[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        float top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(s[b][0], s[b][1]),
                                                  __builtin_elementwise_maximum(s[b][2], s[b][3]));
        constexpr float kMost = CAREFUL ? 0.f : kSlack<DT>;
        const auto passes = [&] { return st.m[b] == -INFINITY ? top > -INFINITY : (top - st.m[b]) * to_log2 > kMost; };
        if (__any(passes())) {
            // a NaN makes the row's results NaN whatever m is
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (passes()) {
                const float alpha = st.m[b] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((st.m[b] - top) * to_log2);
                st.m[b] = top;
                st.l[b] *= alpha;
#pragma unroll
                for (int e = 0; e < S::VB; ++e) acc[b][e] *= alpha;
            }
        }
        const float ref = st.m[b] == -INFINITY ? 0.f : st.m[b];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float t = __builtin_amdgcn_exp2f(fmaf(s[b][r] - ref, to_log2, kBelow<DT>));
            st.l[b] += t;
            if (CAREFUL && kScaled<DT>) t = ldexpf(t, -shift);
            // 16 bits: the term in two parts, so that what it is rounded by is not lost
            hi[b][r] = (T)t;
            if constexpr (DT != DT_F32) lo[b][r] = (T)(t - (float)hi[b][r]);
        }
    }
#pragma unroll
    for (int e = 0; e < S::VB; ++e) {
        const four_t<DT> a = in.values(e);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            acc[b][e] = mma4(a, hi[b], acc[b][e]);
            if constexpr (DT != DT_F32) acc[b][e] = mma4(CAREFUL ? finite_ones<DT>(a) : a, lo[b], acc[b][e]);
        }
    }
}

// Tiles of sequence b, for one key head and block of rows, and its units: beginning
// a pair takes as long as kBegin tiles, so that a work-group with many short ones has
// no more to do than others.  (Or one for all of it.)  Five drafted tokens of 32
// sequences: 90 us for tiles alone, 56.7, 54.5, 52.8 with 2, 3, 5 for a beginning; single
// tokens of 64 sequences 150.7, 152.5, 154.
template <int ROWS>
constexpr int kBegin = ROWS == 16 ? 2 : 5;
__device__ __forceinline__ int tiles_of(int len) { return max(1, (len + kKeys - 1) / kKeys); }
template <int ROWS>
__device__ __forceinline__ int units_of(const PagedParams& p, int len) {
    return p.pairs ? 1 : tiles_of(len) + kBegin<ROWS>;
}
template <int ROWS>
__device__ __forceinline__ int blocks_of(const PagedParams& p, int n) {
    return (int)(((uint32_t)n * (uint32_t)p.group + ROWS - 1) / ROWS);
}

// ONE_PAGE: rows are read in aligned 16-byte chunks, and a wave's 16 keys lie in one
// page (its size is a multiple of 16).
template <int DT, int DP, int NB, bool ONE_PAGE>
__global__ void __launch_bounds__(kThreads, DP == 64 && NB == 1 && DT != DT_F32 ? 4 : 2) paged_few_kernel(PagedParams p) {
    using T = storage_t<DT>;
    using S = Step<DT, DP>;
    constexpr int ROWS = 16 * NB, PITCH = DP + 4;
    __shared__ __align__(16) float sums[kWaves][ROWS][PITCH];
    __shared__ float stat_m[kWaves][ROWS], stat_l[kWaves][ROWS];
    __shared__ int wave_large[kWaves];
    __shared__ int64_t wave_units[kWaves];
    __shared__ int64_t start_units;
    __shared__ int start_seq;
    __shared__ Sequence sequences[64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int me = (int)blockIdx.x;

    // Where this work-group's units begin: in_seq units into sequence seq.
    PagedHeader* headers = (PagedHeader*)p.ws;
    if (!p.pairs && !p.by_pair && threadIdx.x == 0) headers[me].valid = 0;
    int64_t all, workers, first, end, in_seq;
    int seq;
    if (p.small) {
        // Each wave for itself, a sequence a lane, in 32 bits.  The quotients are exact: of
        // products under 2^41, held in binary64, they are no nearer to the next integer
        // than 1 / workers.
        int units = 0;
        if (lane < p.batch) {
            const Sequence s = sequence_of(p, lane);
            units = blocks_of<ROWS>(p, s.n) * p.kv_heads * units_of<ROWS>(p, s.len);
            sequences[lane] = s;  // (every wave writes the same, and reads what it has written)
        }
        int upto = units;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int before = __shfl_up(upto, m);
            if (lane >= m) upto += before;
        }
        const int sum = __builtin_amdgcn_readlane(upto, 63);
        all = sum;
        workers = min(p.workers, sum);
        if (me >= workers) return;
        const auto share = [&](int n) { return (int)((double)sum * (double)n / (double)(int)workers); };
        first = share(me);
        end = share(me + 1);
        seq = __popcll(__ballot(upto <= (int)first));
        in_seq = (int)first - __builtin_amdgcn_readlane(upto - units, seq);
    } else {
        // The units before each thread's sequences.
        const auto units_at = [&](int b) {
            const Sequence s = sequence_of(p, b);
            return (int64_t)blocks_of<ROWS>(p, s.n) * p.kv_heads * units_of<ROWS>(p, s.len);
        };
        const int each = (p.batch + kThreads - 1) / kThreads, mine = (int)threadIdx.x * each;
        int64_t units = 0;
        for (int b = mine; b < min(mine + each, p.batch); ++b) units += units_at(b);
        int64_t upto = units;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int64_t before = __shfl_up(upto, m);
            if (lane >= m) upto += before;
        }
        if (lane == 63) wave_units[wave] = upto;
        __syncthreads();
        int64_t before = upto - units;
        all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += wave_units[w];
            all += wave_units[w];
        }
        workers = min((int64_t)p.workers, all);
        if (me >= workers) return;
        first = all * me / workers;
        end = all * (me + 1) / workers;
        if (before <= first && first < before + units) {
            int b = mine;
            int64_t at = before;
            for (; b < p.batch - 1; ++b) {
                const int64_t n = units_at(b);
                if (first < at + n) break;
                at += n;
            }
            start_seq = b;
            start_units = first - at;
        }
        __syncthreads();
        seq = start_seq;
        in_seq = start_units;
    }
    seq = __builtin_amdgcn_readfirstlane(seq);
    all = uniform(all);
    workers = uniform(workers);
    first = uniform(first);
    end = uniform(end);
    in_seq = uniform(in_seq);

    const float to_log2 = p.scale * kLog2e;
    // Where a lane reads in 16 rows of one page, in bytes; past dim: nowhere.
    constexpr uint32_t kNowhere = 0x7FFFFFF0u;
    constexpr int PIECE = S::VW >= 4 ? S::KB : S::VB;  // elements of a load of V
    const uint32_t k_row = (uint32_t)p.cache[0].sl * (uint32_t)sizeof(T), v_row = (uint32_t)p.cache[1].sl * (uint32_t)sizeof(T);
    uint32_t k_at[S::KC], v_at[4][(S::VW + 3) / 4];
#pragma unroll
    for (int n = 0; n < S::KC; ++n) {
        const int d = (4 * n + g) * S::KB;
        k_at[n] = d < p.dim ? c * k_row + d * (int)sizeof(T) : kNowhere;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < (S::VW + 3) / 4; ++n) {
            const int d = S::VB * c + n * PIECE;
            v_at[j][n] = d < p.dim ? (4 * g + j) * v_row + d * (int)sizeof(T) : kNowhere;
        }
    const auto slot = [&](int worker, int n) {
        return p.ws + (int64_t)p.headers * (sizeof(PagedHeader) / sizeof(float)) +
               ((int64_t)worker * 2 + n) * ROWS * PITCH;
    };
    for (int64_t unit = first; unit < end && seq < p.batch;) {
        Sequence tok = p.small ? sequences[seq] : sequence_of(p, seq);
        tok = Sequence{__builtin_amdgcn_readfirstlane(tok.first), __builtin_amdgcn_readfirstlane(tok.n),
                       __builtin_amdgcn_readfirstlane(tok.len)};
        const int klen = tok.len, n_tiles = tiles_of(klen), n_units = units_of<ROWS>(p, klen);
        const int n_blocks = blocks_of<ROWS>(p, tok.n);
        if (n_blocks == 0) {  // (a sequence without new tokens has no unit)
            ++seq;
            in_seq = 0;
            continue;
        }
        const int pair = __builtin_amdgcn_readfirstlane(p.small ? (int)((uint32_t)in_seq / (uint32_t)n_units)
                                                                : (int)(in_seq / n_units));
        const int in_pair = (int)(in_seq - (int64_t)pair * n_units);
        const int take = (int)min((int64_t)(n_units - in_pair), end - unit);
        const int tile = __builtin_amdgcn_readfirstlane(p.pairs ? 0 : max(0, in_pair - kBegin<ROWS>));
        const int tile_end = __builtin_amdgcn_readfirstlane(p.pairs ? n_tiles : max(0, in_pair + take - kBegin<ROWS>));
        const auto advance = [&] {
            unit += take;
            in_seq += take;
            if (in_seq == (int64_t)n_blocks * p.kv_heads * n_units) {
                ++seq;
                in_seq = 0;
            }
        };
        if (tile == tile_end) {  // no more than a pair's beginning
            advance();
            continue;
        }
        const int block = __builtin_amdgcn_readfirstlane(pair / p.kv_heads), h = pair - block * p.kv_heads;

        // the rows, and the keys that they see
        int lim[NB];
        uint32_t q[NB][S::KC][4];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint32_t row = (uint32_t)block * ROWS + b * 16 + c;
            const int i = (int)(row / (uint32_t)p.group), hq = h * p.group + (int)(row - (uint32_t)i * p.group);
            const bool live = i < tok.n;
            lim[b] = live ? key_limit(i, tok.n, klen, p.causal) : 0;
            const T* at = (const T*)p.q.p + (int64_t)(tok.first + (live ? i : 0)) * p.q.st + (live ? hq : 0) * p.q.sh;
#pragma unroll
            for (int n = 0; n < S::KC; ++n) load_words<DT, 4, ONE_PAGE>(at, (4 * n + g) * S::KB, p.dim, live, q[b][n]);
        }
        const int row_first = (int)((uint32_t)block * ROWS / (uint32_t)p.group);
        const int row_last = min(tok.n - 1, (int)(((uint32_t)block * ROWS + ROWS - 1) / (uint32_t)p.group));
        const int every = key_limit(row_first, tok.n, klen, p.causal);  // what the first row sees, all others see
        const int any = key_limit(row_last, tok.n, klen, p.causal);
        const int take_end = min(any, tile_end * kKeys);
        const int rows = (int)min((int64_t)ROWS, (int64_t)tok.n * p.group - (int64_t)block * ROWS);

        // A product takes every key to every row, with 0 where a row does not see it,
        // and 0 times NaN is NaN.  So where the sums are computed once more, rows of
        // several queries are so query by query, each with its own keys alone (only >= 0).
        const bool by_query = p.causal && row_first < row_last;
        bool careful = false;
        int only = -1;
        for (;;) {
            const int key_end = __builtin_amdgcn_readfirstlane(
                only < 0 ? take_end : min(take_end, key_limit(only, tok.n, klen, p.causal)));

            f32x4 acc[NB][S::VB];
            Rows<NB> st;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                st.m[b] = -INFINITY;
                st.l[b] = 0.f;
#pragma unroll
                for (int e = 0; e < S::VB; ++e) acc[b][e] = f32x4{};
            }
            const int32_t* table = p.table + (int64_t)__builtin_amdgcn_readfirstlane(seq) * p.table_stride;
            const T* kc = (const T*)p.cache[0].p + h * p.cache[0].sh;
            const T* vc = (const T*)p.cache[1].p + h * p.cache[1].sh;
            const int key0 = tile * kKeys + 16 * wave;
            const int shift = careful ? large_shift<DT>(klen) : 0;
            // one step is computed while the next one's keys are on their way
            Step<DT, DP> a, b;
            if (careful) {
#pragma unroll 1
                for (int key = key0; key < key_end; key += kKeys) {
                    a.template load<ONE_PAGE>(p, kc, vc, place_of(p, table, key + c, key_end), lane);
                    step_forward<DT, DP, NB, true>(acc, st, q, a, to_log2, lim, key, every, lane, shift);
                }
            } else if constexpr (ONE_PAGE) {
                // the pages of 64 steps, one a lane
                int pages = 0;
                const auto load = [&](Step<DT, DP>& to, int n) {
                    const int key = key0 + n * kKeys;
                    if (n % 64 == 0) {
                        const int of_lane = key + lane * kKeys;
                        pages = of_lane < key_end ? table[page_of(p, of_lane)] : -1;
                    }
                    const int page = __builtin_amdgcn_readlane(pages, n % 64);
                    const int at = key - page_of(p, key) * p.page;
                    const int rows = in_cache(p, page) ? min(max(key_end - key, 0), 16) : 0;
                    const int some = rows ? page : 0;
                    to.load_page(kc + row_offset(p.cache[0], some, at), vc + row_offset(p.cache[1], some, at), rows, k_row, v_row,
                                 k_at, v_at);
                };
                load(a, 0);
#pragma unroll 1
                for (int n = 0, key = key0; key < key_end; n += 2, key += 2 * kKeys) {  // (a step without a key adds nothing)
                    load(b, n + 1);
                    step_forward<DT, DP, NB, false>(acc, st, q, a, to_log2, lim, key, every, lane);
                    load(a, n + 2);
                    step_forward<DT, DP, NB, false>(acc, st, q, b, to_log2, lim, key + kKeys, every, lane);
                }
            } else {
                // and the places of the one after that
                Place w = place_of(p, table, key0 + c, key_end);
                Place next = place_of(p, table, key0 + kKeys + c, key_end);
                a.template load<false>(p, kc, vc, w, lane);
#pragma unroll 1
                for (int key = key0; key < key_end; key += 2 * kKeys) {
                    w = next;
                    next = place_of(p, table, key + 2 * kKeys + c, key_end);
                    b.template load<false>(p, kc, vc, w, lane);
                    step_forward<DT, DP, NB, false>(acc, st, q, a, to_log2, lim, key, every, lane);
                    w = next;
                    next = place_of(p, table, key + 3 * kKeys + c, key_end);
                    a.template load<false>(p, kc, vc, w, lane);
                    step_forward<DT, DP, NB, false>(acc, st, q, b, to_log2, lim, key + kKeys, every, lane);
                }
            }

            // the waves' sums, joined through LDS
            float largest = 0.f;  // (or NaN)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
#pragma unroll
                for (int e = 0; e < S::VB; ++e)
#pragma unroll
                    for (int r = 0; r < 4; ++r) largest = __builtin_elementwise_maximum(largest, fabsf(acc[b][e][r]));
                st.l[b] += __shfl_xor(st.l[b], 16);
                st.l[b] += __shfl_xor(st.l[b], 32);
                if (g == 0) {
                    stat_m[wave][b * 16 + c] = st.m[b];
                    stat_l[wave][b * 16 + c] = st.l[b];
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < S::VB; e += 4)
                        *(f32x4*)&sums[wave][b * 16 + c][S::VB * (4 * g + r) + e] =
                            f32x4{acc[b][e][r], acc[b][e + 1][r], acc[b][e + 2][r], acc[b][e + 3][r]};
            }
            const bool sums_are_large = __any(!(largest <= kLarge));
            if (lane == 0) wave_large[wave] = sums_are_large;
            __syncthreads();
            if (!careful && (wave_large[0] | wave_large[1] | wave_large[2] | wave_large[3])) {
                careful = true;
                only = by_query ? row_first : -1;
                __syncthreads();  // every wave has read that
                continue;
            }
            const bool begun = tile == 0, ended = tile_end == n_tiles;
            float* part = begun && ended ? nullptr : slot(me, begun ? 1 : 0);
            for (int n = threadIdx.x; n < rows * (DP / 4); n += kThreads) {
                const int r = n / (DP / 4), d = n % (DP / 4) * 4;
                const uint32_t row = (uint32_t)block * ROWS + r;
                const int i = (int)(row / (uint32_t)p.group), hq = h * p.group + (int)(row - (uint32_t)i * p.group);
                if (only >= 0 && i != only) continue;
                float m = stat_m[0][r];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) m = fmaxf(m, stat_m[w][r]);
                const float ref = m == -INFINITY ? 0.f : m;
                f32x4 o = {};
                float l = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float f = __builtin_amdgcn_exp2f((stat_m[w][r] - ref) * to_log2);
                    const f32x4 x = *(const f32x4*)&sums[w][r][d];
                    l = fmaf(f, stat_l[w][r], l);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = fmaf(f, x[e], o[e]);
                }
                if (part != nullptr) {
                    *(f32x4*)(part + r * PITCH + d) = o;
                    if (d == 0) *(f32x4*)(part + r * PITCH + DP) = f32x4{m, l, __int_as_float(shift), 0.f};
                    continue;
                }
                const int64_t t = tok.first + i;
                const bool some = l != 0.f;
                const float f = kScaled<DT> ? ldexpf(1.f / l, shift) : 1.f / l;
                store_quad<DT>((T*)p.o.p + t * p.o.st + hq * p.o.sh, d, p.dim, some ? o[0] * f : 0.f, some ? o[1] * f : 0.f,
                               some ? o[2] * f : 0.f, some ? o[3] * f : 0.f);
                if (d == 0 && p.lse != nullptr)
                    p.lse[t * p.heads + hq] =
                        some ? fmaf(m, p.scale, kLn2 * (__builtin_amdgcn_logf(l) - kBelow<DT>)) : -INFINITY;
            }
            if (threadIdx.x == 0 && !p.pairs && begun && (p.by_pair || !ended)) {
                // the worker that has the pair's last tile
                const int64_t last = unit + (n_units - in_pair) - 1;
                headers[p.by_pair ? (block_before<ROWS>(p, seq) + block) * p.kv_heads + h : me] = PagedHeader{
                    seq, block, h, me,
                    p.small ? (int)((double)((last + 1) * workers - 1) / (double)all) : (int)(((last + 1) * workers - 1) / all),
                    !ended, rows, 0};
            }
            __syncthreads();  // the sums are read
            if (only < 0 || ++only > row_last) break;
        }
        advance();
    }
}

// A pair that work-groups share, joined.  WAVES waves have a row, each every
// WAVES-th part of it, DP / 64 elements a lane; up to AHEAD of a wave's parts are on
// their way together.
constexpr int kJoinThreads = 512;
template <int DT, int DP, int NB, int WAVES>
__global__ void __launch_bounds__(kJoinThreads) paged_few_join_kernel(PagedParams p) {
    using T = storage_t<DT>;
    constexpr int ROWS = 16 * NB, PITCH = DP + 4, E = DP / 64, AHEAD = 8, EACH = kJoinThreads / 64 / WAVES;
    __shared__ float sums[WAVES][DP];
    __shared__ f32x4 stats[WAVES];  // m, l, shift
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) % WAVES;
    const int r = (int)blockIdx.y * EACH + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) / WAVES;
    if (p.by_pair) {
        // A pair's number may be no pair's, and then has no header.  (Nor has it one where the
        // starts do not ascend and count_up_to gives a sequence that begins later: unsigned.)
        const int64_t block = blockIdx.x / (uint32_t)p.kv_heads;
        const auto first_block = [&](int b) { return block_before<ROWS>(p, b); };
        const int seq = count_up_to(p.batch, block, lane, first_block) - 1;
        if (seq < 0 || (uint64_t)((block - first_block(seq)) * ROWS) >= (uint64_t)tokens_of(p, seq).n * p.group) return;
    }
    const PagedHeader h = ((const PagedHeader*)p.ws)[blockIdx.x];
    if (!h.valid || r >= h.rows) return;
    const int me = h.first;
    const float to_log2 = p.scale * kLog2e;
    const float* base = p.ws + (int64_t)p.headers * (sizeof(PagedHeader) / sizeof(float)) + r * PITCH;
    const int parts = h.last - me + 1;
    const auto part = [&](int k) { return base + ((int64_t)(me + k) * 2 + (k == 0)) * ROWS * PITCH; };
    // o is held times 2^-shift, the largest of the parts' shifts (0, but for large sums)
    float m = -INFINITY, l = 0.f, o[E];
    int shift = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int k0 = wave; k0 < parts; k0 += WAVES * AHEAD) {
        float x[AHEAD][E], xm[AHEAD], xl[AHEAD];
        int xs[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            const int k = k0 + n * WAVES;
            xm[n] = -INFINITY;
            xs[n] = 0;
            if (k < parts) {
                const float* at = part(k);
                const f32x4 stat = *(const f32x4*)(at + DP);
                xm[n] = stat[0];
                xl[n] = stat[1];
                if (kScaled<DT>) xs[n] = __float_as_int(stat[2]);
#pragma unroll
                for (int e = 0; e < E; ++e) x[n][e] = at[lane * E + e];
            }
        }
        float now = m;
        int most = shift;
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            now = fmaxf(now, xm[n]);
            most = max(most, xs[n]);
        }
        const float ref = now == -INFINITY ? 0.f : now;
        float f = __builtin_amdgcn_exp2f((m - ref) * to_log2);
        l *= f;
        if (kScaled<DT>) f = ldexpf(f, shift - most);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= f;
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            if (k0 + n * WAVES >= parts) continue;
            f = __builtin_amdgcn_exp2f((xm[n] - ref) * to_log2);
            l = fmaf(f, xl[n], l);
            if (kScaled<DT>) f = ldexpf(f, xs[n] - most);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(f, x[n][e], o[e]);
        }
        m = now;
        shift = most;
    }
    const uint32_t row = (uint32_t)h.block * ROWS + r;
    const int i = (int)(row / (uint32_t)p.group), hq = h.head * p.group + (int)(row - (uint32_t)i * p.group);
    const Tokens tok = tokens_of(p, h.seq);
    if (i >= tok.n) return;  // (starts that do not ascend: pairs may share a number, and a header has some of each)
    const int64_t t = tok.first + i;
    const auto write = [&](int d, float x) {
        const bool some = l != 0.f;
        if (kScaled<DT>) x = ldexpf(x / l, shift);
        else x /= l;
        if (d < p.dim) ((T*)p.o.p)[t * p.o.st + hq * p.o.sh + d] = (T)(some ? x : 0.f);
        if (d == 0 && p.lse != nullptr)
            p.lse[t * p.heads + hq] = some ? fmaf(m, p.scale, kLn2 * (__builtin_amdgcn_logf(l) - kBelow<DT>)) : -INFINITY;
    };
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) write(lane * E + e, o[e]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) sums[wave][lane * E + e] = o[e];
        if (lane == 0) stats[wave] = f32x4{m, l, __int_as_float(shift), 0.f};
        __syncthreads();
        const int d = threadIdx.x;
        if (d >= p.dim) return;
        f32x4 stat[WAVES];
        m = -INFINITY;
        shift = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            stat[w] = stats[w];
            m = fmaxf(m, stat[w][0]);
            shift = max(shift, __float_as_int(stat[w][2]));
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float x = 0.f;
        l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f((stat[w][0] - ref) * to_log2);
            l = fmaf(f, stat[w][1], l);
            x = fmaf(kScaled<DT> ? ldexpf(f, __float_as_int(stat[w][2]) - shift) : f, sums[w][d], x);
        }
        write(d, x);
    }
}

template <int DT, int DP, int NB>
hipError_t few(const PagedParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)p.workers);
    // (rows of a page that lie apart: the bounds of a descriptor tell them from each other)
    const bool apart = p.cache[0].sl >= p.dim && p.cache[1].sl >= p.dim;
    if (p.whole && apart && p.page % 16 == 0) paged_few_kernel<DT, DP, NB, true><<<grid, kThreads, 0, stream>>>(p);
    else paged_few_kernel<DT, DP, NB, false><<<grid, kThreads, 0, stream>>>(p);
    if (!p.pairs) {
        const int64_t most = (p.starts != nullptr ? (int64_t)p.tokens : 1) * p.group;
        const int rows = (int)(most < 16 * NB ? most : 16 * NB);
        // Eight waves a row where a pair is likely to have more parts than a wave reads at
        // once (one sequence of 8000 keys: 16.7 us, 28.6 with one wave; five drafted tokens of
        // 32 sequences: 52 us with one, 70 with eight).
        if (p.by_pair && p.workers > 8 * p.headers)
            paged_few_join_kernel<DT, DP, NB, 8>
                <<<dim3((unsigned)p.headers, (unsigned)rows), kJoinThreads, 0, stream>>>(p);
        else
            paged_few_join_kernel<DT, DP, NB, 1>
                <<<dim3((unsigned)p.headers, (unsigned)((rows + 7) / 8)), kJoinThreads, 0, stream>>>(p);
    }
    return hipGetLastError();
}

// --------------------------------------------------------------- many rows --

constexpr int kRows = kAttnRows;

// Where a tile's rows are, lane n of every wave knowing row n's page and its place
// there, and which of them are there.
struct TilePages {
    int page, in_page;
    uint64_t present;
};
// The table by buffer loads, for the reason that tiles are filled by them.  Past its
// end they give 0; no key is there, and none is taken from that page.
__device__ __forceinline__ int page_in_table(const PagedParams& p, __amdgpu_buffer_rsrc_t table, int key) {
    return (int)__builtin_amdgcn_raw_buffer_load_b32(table, page_of(p, key) * 4, 0, 0);
}

// Rows of a tile from their pages, in the background as Filler does it: one
// descriptor for the rows that a wave fills at once, which are in one page.
template <int DT, int DP>
struct PagedFiller {
    using T = storage_t<DT>;
    using F = Filler<DT, DP, kKeys, kThreads>;
    using L = Tile<DT, DP>;
    static constexpr int SLOTS = F::SLOTS, STEP = F::STEP, STEPS = F::STEPS;
    uint32_t offset;
    bool in;

    __device__ __forceinline__ PagedFiller(int64_t stride, int dim) {
        const int d = ((int)threadIdx.x % SLOTS ^ L::turn((int)threadIdx.x / SLOTS)) * L::VEC;
        in = d < dim;
        offset = ((uint32_t)(((int)threadIdx.x & 63) / SLOTS) * (uint32_t)stride + (uint32_t)d) * (uint32_t)sizeof(T);
    }
    // base: the head's element 0 of page 0; lane n knows row n's address.
    __device__ __forceinline__ void fill(T* tile, const T* base, const PagedParams& p, const HeadView& c,
                                         const TilePages& at) const {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        T* to = tile + wave * L::KB;
        const uint64_t address = (uint64_t)(base + row_offset(c, at.page, at.in_page));
        // (the lanes are asked while all of them are there: the one that knows a row may
        // have no chunk of its own to send for)
        if (at.present == ~(uint64_t)0 && p.page % kKeys == 0) {  // all of the tile in one page
            const auto from = background((const void*)readlane_u64(address, 0));
            const int row = (int)c.sl * (int)sizeof(T);  // (kKeys of them are within 2^31 bytes)
            if (!in) return;  // (zeros from the beginning)
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
                send<16>(from, offset, (k * STEP + wave * L::KB_ROWS) * row, to + k * (STEP / L::KB_ROWS * L::KB));
        } else if (at.present == ~(uint64_t)0) {
            uint64_t from[STEPS];
#pragma unroll
            for (int k = 0; k < STEPS; ++k) from[k] = readlane_u64(address, k * STEP + wave * L::KB_ROWS);
            if (!in) return;
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
                send<16>(background((const void*)from[k]), offset, 0, to + k * (STEP / L::KB_ROWS * L::KB));
        } else {
#pragma unroll 1
            for (int k = 0; k < STEPS; ++k) {
                const int row = k * STEP + wave * L::KB_ROWS;  // the wave's first; if it is not there, none is
                const uint64_t from = readlane_u64(address, row);
                if (in && (at.present >> (row + lane / SLOTS) & 1)) {
                    send<16>(background((const void*)from), offset, 0, to);
                } else {
                    const u32v4 zero = {0, 0, 0, 0};
                    *(u32v4*)(to + lane * L::VEC) = zero;
                }
                to += STEP / L::KB_ROWS * L::KB;
            }
        }
    }
};

// The same through registers: any page size, any alignment.
template <int DT, int DP>
__device__ __forceinline__ void paged_stage(storage_t<DT>* tile, const storage_t<DT>* base, const PagedParams& p,
                                            const HeadView& c, const TilePages& at) {
    using L = Tile<DT, DP>;
    static_assert(kKeys * L::CHUNKS % kThreads == 0, "every thread has the same number of chunks");
#pragma unroll
    for (int k = 0; k < kKeys * L::CHUNKS / kThreads; ++k) {
        const int idx = k * kThreads + (int)threadIdx.x, row = idx / L::CHUNKS, d = idx % L::CHUNKS * L::VEC;
        const int page = __shfl(at.page, row), in_page = __shfl(at.in_page, row);
        u32v4 v = {0, 0, 0, 0};
        if (at.present >> row & 1) v = load_chunk(base + row_offset(c, page, in_page), d, p.dim);
        *(u32v4*)(tile + L::at(row, d)) = v;
    }
}

template <int DT, int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, DT == DT_F32 ? 1 : 2) paged_many_kernel(PagedParams p) {
    using T = storage_t<DT>;
    using L = Tile<DT, DP>;
    __shared__ __align__(16) T kt[2][L::size(kKeys)];
    __shared__ __align__(16) T vt[2][L::size(kKeys)];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5;
    const int part = (int)blockIdx.y;
    // the block's sequence: the last one whose first block is no later
    const int h = (int)(blockIdx.x % (uint32_t)p.kv_heads);
    const int64_t block = paged_blocks(p, kRows) - 1 - blockIdx.x / (uint32_t)p.kv_heads;
    int seq, klen;
    Tokens tok;
    int64_t block0;
    if (p.batch <= 64) {  // a sequence a lane: all that is asked of them on its way at once
        Sequence mine{0, 0, 0};
        if (lane < p.batch) mine = sequence_of(p, lane);
        const int of_lane = (int)((uint32_t)mine.first * (uint32_t)p.group / kRows) + lane;  // block_before
        seq = __popcll(__ballot(lane < p.batch && of_lane <= block)) - 1;
        if (seq < 0) return;
        tok = {__builtin_amdgcn_readlane(mine.first, seq), __builtin_amdgcn_readlane(mine.n, seq)};
        klen = __builtin_amdgcn_readlane(mine.len, seq);
        block0 = __builtin_amdgcn_readlane(of_lane, seq);
    } else {
        const auto first_block = [&](int b) { return block_before<kRows>(p, b); };
        seq = __builtin_amdgcn_readfirstlane(count_up_to(p.batch, block, lane, first_block)) - 1;
        if (seq < 0) return;
        tok = tokens_of(p, seq);
        klen = paged_len(p, seq);
        block0 = first_block(seq);
    }
    if (block < block0 || (block - block0) * kRows >= (int64_t)tok.n * p.group) return;  // between two sequences
    const uint32_t first = (uint32_t)(block - block0) * kRows;

    const uint32_t row = first + wave * 32 + (lane & 31);
    const int i = (int)(row / (uint32_t)p.group), hq = h * p.group + (int)(row % (uint32_t)p.group);
    const bool live = i < tok.n;
    const int wave_first = __builtin_amdgcn_readfirstlane((int)((first + wave * 32) / (uint32_t)p.group));
    const int wave_last = __builtin_amdgcn_readfirstlane((int)((first + wave * 32 + 31) / (uint32_t)p.group));
    const int block_last = (int)((first + kRows - 1) / (uint32_t)p.group);
    const int lim = key_limit(min(i, tok.n - 1), tok.n, klen, p.causal);
    const int wave_any = wave_first < tok.n ? key_limit(min(wave_last, tok.n - 1), tok.n, klen, p.causal) : 0;
    const int block_all = key_limit((int)(first / (uint32_t)p.group), tok.n, klen, p.causal);
    const int all = key_limit(min(block_last, tok.n - 1), tok.n, klen, p.causal);
    const int tiles = (all + kKeys - 1) / kKeys;
    const int start = (int)((int64_t)tiles * part / p.parts) * kKeys;
    const int end = min(all, (int)((int64_t)tiles * (part + 1) / p.parts) * kKeys);

    const T* q = (const T*)p.q.p + (int64_t)(tok.first + (live ? i : 0)) * p.q.st + hq * p.q.sh;
    const T* k = (const T*)p.cache[0].p + h * p.cache[0].sh;
    const T* v = (const T*)p.cache[1].p + h * p.cache[1].sh;
    frag_t<DT> qf[DP / 16];
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) qf[c] = load_frag<DT, WHOLE>(q, c, g, p.dim, live);
    const Reader<DT, DP> rd(lane);
    const PagedFiller<DT, DP> fk(p.cache[0].sl, p.dim), fv(p.cache[1].sl, p.dim);
    if (WHOLE && p.dim != L::PITCH) {  // what no tile's rows fill
        for (int n = threadIdx.x * L::VEC; n < 2 * L::size(kKeys); n += kThreads * L::VEC) {
            const u32v4 zero = {0, 0, 0, 0};
            *(u32v4*)(&kt[0][0] + n) = zero;
            *(u32v4*)(&vt[0][0] + n) = zero;
        }
        __syncthreads();
    }
    const auto rows_of = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t*>(p.table + (int64_t)seq * p.table_stride), 0,
                                                           (uint32_t)p.width * 4u, 0x00020000);
    const auto look = [&](int j0) { return page_in_table(p, rows_of, j0 + lane); };
    // Fills the tile from key j0 on; which of its rows are there.
    const auto fill = [&](int j0, int page, int buf) {
        const int key = j0 + lane;
        const TilePages at{page, key - page_of(p, key) * p.page, __ballot(in_cache(p, page) && key < end)};
        if (WHOLE) {
            fk.fill(kt[buf], k, p, p.cache[0], at);
            fv.fill(vt[buf], v, p, p.cache[1], at);
        } else {
            paged_stage<DT, DP>(kt[buf], k, p, p.cache[0], at);
            paged_stage<DT, DP>(vt[buf], v, p, p.cache[1], at);
        }
        return at.present;
    };

    const float to_log2 = p.scale * kLog2e;
    f32x16 acc[DP / 32];
    Softmax sm;
    int shift = 0;
    const auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) acc[db] = f32x16{};
        sm = Softmax{};
        // a tile is used, the next one is filled, the pages of the one after that are looked up
        uint64_t now = 0, ahead = 0;
        int page = look(start);
        if (start < end) ahead = fill(start, page, 0);
        page = look(start + kKeys);
        int j0 = start, buf = 0;
        const auto next = [&] {
            tile_wait();
            __syncthreads();  // the tile is there, and the other one is read
            now = ahead;
            if (j0 + kKeys < end) {
                ahead = fill(j0 + kKeys, page, buf ^ 1);
                page = look(j0 + 2 * kKeys);
            }
        };
        // first the tiles that every row of the work-group sees whole, up to a key without a page
        bool ready = false;
        for (; j0 + kKeys <= min(block_all, end); j0 += kKeys, buf ^= 1) {
            next();
            ready = now != ~(uint64_t)0;
            if (ready) break;
            if (wave_any > 0)
                tile_forward<DT, DP, false, CAREFUL>(acc, sm, qf, kt[buf], vt[buf], rd, to_log2, 0, ~(uint64_t)0, shift);
        }
        for (; j0 < end; j0 += kKeys, buf ^= 1) {
            if (!ready) next();
            ready = false;
            if (j0 < wave_any)
                tile_forward<DT, DP, true, CAREFUL, true>(acc, sm, qf, kt[buf], vt[buf], rd, to_log2, lim - j0, now, shift);
        }
    };
    pass(std::false_type{});
    if (__syncthreads_or(too_large(acc) || (DT != DT_F32 && too_coarse(sm)))) {
        shift = large_shift<DT>(all);
        pass(std::true_type{});
        if (DT != DT_F32 && sm.m > -INFINITY) sm.m = __builtin_amdgcn_fmed3f(fmaf(sm.m, to_log2, -kBelow<DT>), -FLT_MAX, FLT_MAX);
    }
    if (!live) return;
    const float l = sm.l + other_half(sm.l), rounded = sm.rounded + other_half(sm.rounded);
    const int64_t t = tok.first + i;
    if (p.parts > 1) {
        const int64_t dim = (p.dim + 3) / 4 * 4;
        float* to = p.ws + ((t * p.heads + hq) * p.parts + part) * (dim + 4);
        if (g == 0) *(f32x4*)(to + dim) = f32x4{sm.m, l, rounded, (float)shift};
        store_part<DP>(to, acc, p.dim, g);
        return;
    }
    const bool some = l != 0.f;  // NaN too: it goes on to o
    const float f = DT == DT_F32 ? ldexpf(1.f / l, shift) : 1.f / rounded;
    store_column<DT, DP>((T*)p.o.p + t * p.o.st + hq * p.o.sh, acc, f, some, p.dim, g);
    if (g == 0 && p.lse != nullptr)
        p.lse[t * p.heads + hq] = some ? fmaf(sm.m, unit_natural<DT>(p.scale), kLn2 * __builtin_amdgcn_logf(l)) : -INFINITY;
}

// The parts of a row joined, four elements a thread.
template <int DT>
__global__ void __launch_bounds__(kThreads) paged_many_join_kernel(PagedParams p) {
    using T = storage_t<DT>;
    const int quads = (p.dim + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t row = id / quads;  // [token][head]
    const int d = (int)(id % quads) * 4;
    if (row >= (int64_t)p.tokens * p.heads) return;
    const int64_t t = row / p.heads;
    const int hq = (int)(row - t * p.heads);
    if (p.starts != nullptr && (t < p.starts[0] || t >= p.starts[p.batch])) return;  // no sequence's
    const int64_t dim = (p.dim + 3) / 4 * 4, stride = dim + 4;
    const float* in = p.ws + row * p.parts * stride;
    float m = -INFINITY, most = 0.f;  // (most: the largest of the parts' shifts)
    for (int s = 0; s < p.parts; ++s) {
        m = fmaxf(m, in[s * stride + dim]);
        if (kScaled<DT>) most = fmaxf(most, in[s * stride + dim + 3]);
    }
    const float ref = m == -INFINITY ? 0.f : m;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f, rounded = 0.f;
    for (int s = 0; s < p.parts; ++s) {
        const f32x4 stat = *(const f32x4*)(in + s * stride + dim), x = *(const f32x4*)(in + s * stride + d);
        const float w = __builtin_amdgcn_exp2f((stat[0] - ref) * unit_log2<DT>(p.scale));
        const float scaled = kScaled<DT> ? ldexpf(w, (int)(stat[3] - most)) : w;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(scaled, x[e], acc[e]);
        l = fmaf(w, stat[1], l);
        rounded = fmaf(scaled, stat[2], rounded);
    }
    const bool some = l != 0.f;
    const float f = !some ? 0.f : DT == DT_F32 ? ldexpf(1.f / l, (int)most) : 1.f / rounded;
    store_quad<DT>((T*)p.o.p + t * p.o.st + hq * p.o.sh, d, p.dim, some ? acc[0] * f : 0.f, some ? acc[1] * f : 0.f,
                   some ? acc[2] * f : 0.f, some ? acc[3] * f : 0.f);
    if (d == 0 && p.lse != nullptr)
        p.lse[row] = some ? fmaf(m, unit_natural<DT>(p.scale), kLn2 * __builtin_amdgcn_logf(l)) : -INFINITY;
}

template <int DT, int DP>
hipError_t many(const PagedParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)(paged_blocks(p, kRows) * p.kv_heads), (unsigned)p.parts);
    // rows that a wave fills at once lie in one page
    if (p.whole && p.page % Tile<DT, DP>::KB_ROWS == 0) paged_many_kernel<DT, DP, true><<<grid, kThreads, 0, stream>>>(p);
    else paged_many_kernel<DT, DP, false><<<grid, kThreads, 0, stream>>>(p);
    if (p.parts > 1) {
        const int64_t quads = (int64_t)p.tokens * p.heads * ((p.dim + 3) / 4);
        paged_many_join_kernel<DT><<<dim3((unsigned)((quads + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(p);
    }
    return hipGetLastError();
}

template <int DT>
hipError_t paged(const PagedParams& p, hipStream_t stream) {
    if (few_rows(p)) {
        if (p.dim <= 64) return few_block(p) == 16 ? few<DT, 64, 1>(p, stream) : few<DT, 64, 2>(p, stream);
        if constexpr (DT != DT_F32) {
            if (few_block(p) == 32) return few<DT, 128, 2>(p, stream);
        }
        return few<DT, 128, 1>(p, stream);
    }
    if (p.dim <= 64) return many<DT, 64>(p, stream);
    if (p.dim <= 96) return many<DT, 96>(p, stream);
    return many<DT, 128>(p, stream);
}

}  // namespace

hipError_t launch_attn_paged(int dtype, const PagedParams& p, hipStream_t stream) {
    if (dtype == DT_F32) return paged<DT_F32>(p, stream);
    if (dtype == DT_F16) return paged<DT_F16>(p, stream);
    return paged<DT_BF16>(p, stream);
}

}  // namespace kb
