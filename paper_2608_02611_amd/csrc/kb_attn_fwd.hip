// kb_attn_fwd.hip -- softmax attention, forward: for query i over the keys j
// that it sees, s_j = scale q_i . k_j, lse = log S(exp s_j),
// o = S(exp(s_j - lse) v_j).
//
// One pass over the keys with the running maximum m and sum l of the softmax:
// a tile's terms are exp(s_j - m) for the new maximum, and what was summed
// before is scaled by exp(m_old - m).  A work-group takes 128 query rows, 32 a
// wave; the query heads that share a key head are rows of the same work-group
// (row = query * group + head), so that a tile of keys serves all of them.
#include "kb_attn.hpp"

namespace kb {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 128;  // query rows of a work-group
constexpr int kKeys = 64;   // keys of a tile

template <int DT, int DP>
__global__ void __launch_bounds__(kThreads) attn_forward_kernel(AttnParams p) {
    using T = storage_t<DT>;
    using L = Tile<DT, DP>;
    __shared__ __align__(16) T kt[kKeys * L::PITCH];
    __shared__ __align__(16) T vt[kKeys * L::PITCH];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5;
    const HeadBlock at = head_block(p.kv_heads, p.batch * p.kv_heads);
    const int n_blocks = (int)(((int64_t)p.len_q * p.group + kRows - 1) / kRows);
    const int64_t first = (int64_t)(n_blocks - 1 - at.block) * kRows;  // causal: the longest first
    const int qlen = seq_len(p.q_lens, at.b, p.len_q), klen = seq_len(p.k_lens, at.b, p.len_k);

    const int64_t row = first + wave * 32 + (lane & 31);
    const int i = (int)(row / p.group), hq = at.h * p.group + (int)(row % p.group);
    const bool exists = i < p.len_q, live = i < qlen;
    const int wave_first = (int)((first + wave * 32) / p.group), wave_last = (int)((first + wave * 32 + 31) / p.group);
    const int block_last = (int)((first + kRows - 1) / p.group);
    const bool any = (int)(first / p.group) < qlen;
    const int lim = key_limit(min(i, qlen - 1), qlen, klen, p.causal);
    const int wave_all = key_limit(min(wave_first, qlen - 1), qlen, klen, p.causal);  // keys that every row sees
    const int wave_any = wave_first < qlen ? key_limit(min(wave_last, qlen - 1), qlen, klen, p.causal) : 0;
    const int end = any ? key_limit(min(block_last, qlen - 1), qlen, klen, p.causal) : 0;

    const T* q = (const T*)p.q.p + at.b * p.q.sb + hq * p.q.sh + i * p.q.sl;
    const T* k = (const T*)p.k.p + at.b * p.k.sb + at.h * p.k.sh;
    const T* v = (const T*)p.v.p + at.b * p.v.sb + at.h * p.v.sh;
    frag_t<DT> qf[DP / 16];
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) qf[c] = load_frag<DT>(q, c, g, p.dim, live);

    const float to_log2 = p.scale * kLog2e;
    f32x16 acc[DP / 32] = {};
    float m = -INFINITY, l = 0.f;
    for (int j0 = 0; j0 < end; j0 += kKeys) {
        __syncthreads();
        stage<DT, DP, kKeys, kThreads>(kt, k, p.k.sl, j0, klen, p.dim);
        stage<DT, DP, kKeys, kThreads>(vt, v, p.v.sl, j0, klen, p.dim);
        __syncthreads();
        if (j0 >= wave_any) continue;
        f32x16 s[2] = {};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) s[t] = mma(row_frag<DT, DP>(kt, 32 * t + (lane & 31), c, g), qf[c], s[t]);
        const bool part = j0 + kKeys > wave_all;
        if (part) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (j0 + 32 * t + 8 * (r >> 2) + 4 * g + (r & 3) >= lim) s[t][r] = -INFINITY;
        }
        float top = m;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
        top = fmaxf(top, other_half(top));
        // the difference before the scale: the largest term is 1 exactly
        const float shift = top == -INFINITY ? 0.f : top;  // nothing seen yet: every term is 0
        const float alpha = __builtin_amdgcn_exp2f((m - shift) * to_log2);
        m = top;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f((s[t][r] - shift) * to_log2);
                l += s[t][r];
            }
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const frag_t<DT> b[2] = {narrow<DT>(s[t], 0), narrow<DT>(s[t], 1)};
            mma_rows<DT, DP>(acc, vt, 32 * t, b, part, 0, lim - j0, lane);
        }
    }
    if (!exists) return;
    l += other_half(l);
    const bool some = live && l != 0.f;  // NaN too: it goes on to o
    store_column<DT, DP>((T*)p.o.p + at.b * p.o.sb + hq * p.o.sh + i * p.o.sl, acc, 1.f / l, some, p.dim, g);
    if (g == 0)
        p.lse[((int64_t)at.b * p.heads + hq) * p.len_q + i] =
            some ? fmaf(m, p.scale, kLn2 * __builtin_amdgcn_logf(l)) : -INFINITY;
}

template <int DT, int DP>
hipError_t forward(const AttnParams& p, hipStream_t stream) {
    const int64_t blocks = ((int64_t)p.len_q * p.group + kRows - 1) / kRows * p.batch * p.kv_heads;
    attn_forward_kernel<DT, DP><<<dim3((unsigned)blocks), kThreads, 0, stream>>>(p);
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
