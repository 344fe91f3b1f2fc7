// kb_ops.hpp -- the reference operators (layer norm, attention): parameters
// that the host fills in, launchers, and the device helpers they share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kb_device.hpp"

namespace kb {

// ------------------------------------------------------------- layer norm --

// A [rows][cols] view with contiguous rows; stride in elements.
struct RowView {
    const void* p;
    int64_t stride;
};

struct NormForwardParams {
    RowView x, y;
    const void* w;  // NULL: 1
    const void* b;  // NULL: 0
    float* mean;    // each may be NULL
    float* rstd;
    int64_t rows;
    int cols;
    float eps;
};

struct NormBackwardParams {
    RowView dy, x, dx;  // dx.p may be NULL
    const void* w;      // NULL: 1
    const float* mean;
    const float* rstd;
    void* dw;  // each may be NULL
    void* db;
    float* part;  // partial column sums: [parts][2][cols] (dw, db)
    int64_t rows;
    int cols;
};

// Row stripes whose column sums are kept apart (NormBackwardParams::part): one
// for each work-group.  Rows of more than 128 columns and at most 768 bytes get
// twice as many, as a work-group of four such rows has few bytes on their way
// (65,536 rows, with 1024 / 512 parts: 136 x bf16 29 / 34 us, 256 31 / 37, 264 32 / 38,
// 384 38 / 40, 512 45 / 44, 1024 92 / 77; f32 136 31 / 37, 192 37 / 39, 256 45 / 42;
// sixteen rows a work-group: 64 x bf16 14.6 / 13.9, f32 128 24 / 23).
constexpr int64_t kNormParts = 512;
inline int norm_parts(int64_t groups, int64_t cols, int64_t element_bytes) {
    const int64_t most = cols > 128 && cols * element_bytes <= 768 ? 2 * kNormParts : kNormParts;
    return (int)(groups < most ? groups : most);
}
// Enough for every type.
inline size_t norm_part_bytes(int64_t rows, int64_t cols) {
    const size_t parts = (size_t)norm_parts(rows, cols, 2);
    return (parts * 2 * (size_t)cols * sizeof(float) + 15) & ~(size_t)15;
}

// dtype: x's and y's; wdtype: w's, b's, dw's and db's (dtype or DT_F32).
hipError_t launch_norm_forward(int dtype, int wdtype, const NormForwardParams& p, hipStream_t stream);
hipError_t launch_norm_backward(int dtype, int wdtype, const NormBackwardParams& p, hipStream_t stream);

// -------------------------------------------------------------- attention --

// A [batch][heads][len][dim] view; strides in elements, dim contiguous.
struct HeadView {
    const void* p;
    int64_t sb, sh, sl;
};

struct AttnParams {
    HeadView q, k, v, o;
    HeadView dout, dq, dk, dv;  // backward
    float* lse;                 // [batch][heads][len_q]
    const int32_t* q_lens;      // each may be NULL
    const int32_t* k_lens;
    int batch, heads, kv_heads, group;  // group = heads / kv_heads
    int len_q, len_k, dim;
    float scale;
    int causal;
    int f32;        // binary32 elements, whose products take eight times as long
    int parts;      // forward, dq: parts of the keys
    int key_parts;  // dk, dv: parts of the queries
    int whole;  // rows of q, k, v (and o, dout) are aligned to 16 bytes and made of 16-byte chunks
    float* ws;
};

// Tiles: query rows of a work-group and keys that pass it at a time (forward, dq),
// keys of a work-group and queries that pass it at a time (dk, dv).
constexpr int kAttnRows = 128;
constexpr int kAttnKeys = 64;
constexpr int kAttnKeyRows = 128;
constexpr int kAttnQueries = 32;
// Rows that one buffer descriptor of 2^31 bytes has to reach (AttnParams::whole
// bounds their stride); what is longer is filled piece by piece.
constexpr int kAttnReach = 64;

// What passes a work-group is split into parts, each with work-groups of its own
// and joined afterwards, so that a few rows still fill the device: `fill`
// work-groups, of `least` rows to pass or more.
inline int attn_parts(int64_t work_groups, int64_t passing, int64_t fill, int64_t least) {
    if (work_groups == 0 || 2 * work_groups > fill) return 1;
    const int64_t want = fill / work_groups, most = passing / least;
    return (int)(want < most ? want : most > 1 ? most : 1);
}
// Blocks of query rows for each (batch, key head) pair: fewer than 2^24 over all
// pairs, so that rows within one are numbered in 32 bits.
__host__ __device__ inline int pair_blocks(const AttnParams& p) {
    return (int)(((int64_t)p.len_q * p.group + kAttnRows - 1) / kAttnRows);
}
inline int64_t row_blocks(const AttnParams& p) { return (int64_t)p.batch * p.kv_heads * pair_blocks(p); }
inline int64_t key_blocks(const AttnParams& p) {
    return (int64_t)p.batch * p.kv_heads * (((int64_t)p.len_k + kAttnKeyRows - 1) / kAttnKeyRows);
}
// Forward: two work-groups for each of 256 CUs; for sequences of different
// lengths, whose parts end at different times, as many again (512 queries on
// 16,384 keys of one sequence: 8 parts cost 15 us to join).  In 32 bits parts may
// be shorter (8 heads x 100 queries on 1000 keys: 43 us, 146 with parts of 512).
inline int forward_parts(const AttnParams& p) {
    return attn_parts(row_blocks(p), p.len_k, p.q_lens || p.k_lens ? 1024 : 512, p.f32 ? 128 : 512);
}
// Backward: the work-groups that the CUs hold at once, one each in 32 bits and two
// in 16, and as many again under a causal mask, whose blocks are long and short (2 x
// 32 heads on 8 x 4096 bf16: 854 us with dk and dv in two parts, 1005 in one).  In
// 32 bits a few work-groups over a round cost a second one (256 / 320 at most: 2 x 12
// heads x 384 59 / 84 us, the same of different lengths 60 / 79, 8 heads on 2 x 700
// 157 / 214; 2 x 12 heads, 513 x 257 of different lengths 103 / 100; 512 at most: 71,
// 170 and 115).  But parts may be shorter, a tile taking 6 us (8 heads x 300: 48 us,
// 62 with parts of 128).
inline int64_t backward_fill(const AttnParams& p) { return (p.f32 ? 256 : 512) * (p.causal ? 2 : 1); }
inline int row_parts(const AttnParams& p) {
    return attn_parts(row_blocks(p), p.len_k, backward_fill(p), (p.f32 ? 1 : 2) * kAttnKeys);
}
inline int key_parts(const AttnParams& p) {
    return attn_parts(key_blocks(p), (int64_t)p.len_q * p.group, backward_fill(p), (p.f32 ? 2 : 4) * kAttnQueries);
}

// Workspace of the forward pass in parts, in floats: for each query row and part
// the sums over its keys (dim rounded up to 4), then m, l and the rounded l.
__host__ __device__ inline int64_t part_dim(const AttnParams& p) { return (p.dim + 3) / 4 * 4; }
inline int64_t forward_floats(const AttnParams& p, int parts) {
    return parts > 1 ? (int64_t)p.batch * p.heads * p.len_q * parts * (part_dim(p) + 4) : 0;
}

// Workspace of the backward pass, in floats: D_i and lse_i for every query row;
// (F16) the largest squared norm of the rows of dout in each work-group of rows,
// and of each block of kNormBlock rows of v; a word for each work-group of keys;
// then, each where it is in parts, dq of every query row and part, and dk and dv of
// every key and part.
constexpr int kNormBlock = 64;
struct BackwardLayout {
    int64_t lse, dout_norms, v_norms, marks, dq, dkv, total;
};
inline BackwardLayout backward_layout(const AttnParams& p) {
    const int64_t heads = (int64_t)p.batch * p.heads, pairs = (int64_t)p.batch * p.kv_heads;
    BackwardLayout l;
    l.lse = heads * p.len_q;
    l.dout_norms = 2 * l.lse;
    l.v_norms = l.dout_norms + row_blocks(p);
    l.marks = l.v_norms + pairs * ((p.len_k + (int64_t)kNormBlock - 1) / kNormBlock);
    l.dq = (l.marks + key_blocks(p) * key_parts(p) + 3) / 4 * 4;
    l.dkv = l.dq + (row_parts(p) > 1 ? heads * p.len_q * row_parts(p) * part_dim(p) : 0);
    l.total = l.dkv + (key_parts(p) > 1 ? 2 * pairs * p.len_k * key_parts(p) * part_dim(p) : 0);
    return l;
}

hipError_t launch_attn_forward(int dtype, const AttnParams& p, hipStream_t stream);
hipError_t launch_attn_backward(int dtype, const AttnParams& p, hipStream_t stream);

// ------------------------------------------------------- storage <-> float --

template <int DT>
struct Storage;
template <>
struct Storage<DT_F32> {
    using type = float;
};
template <>
struct Storage<DT_F16> {
    using type = _Float16;
};
template <>
struct Storage<DT_BF16> {
    using type = __bf16;
};
template <int DT>
using storage_t = typename Storage<DT>::type;

typedef uint32_t u32v4 __attribute__((ext_vector_type(4)));

// 16 bytes of elements, readable at any element's alignment (gfx950 loads
// and stores dwords at any byte address).
template <typename T>
struct Vec16 {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// 16 bytes without the first `drop` elements, zeros after the others.
template <typename T>
__device__ __forceinline__ u32v4 drop_elements(u32v4 v, int drop) {
    const int bits = drop * 8 * (int)sizeof(T);
    if (bits & 64) v = u32v4{v[2], v[3], 0, 0};
    if (bits & 32) v = u32v4{v[1], v[2], v[3], 0};
    if (sizeof(T) == 2) {
        const uint32_t s = bits & 16;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __builtin_amdgcn_alignbit(k < 3 ? v[k + 1] : 0, v[k], s);
    }
    return v;
}

// 16 bytes of a row of n elements from element c < n on, zeros past its end.
// The last ones of a row that is no multiple are read with the elements before
// them, in the same instruction as every other lane's, and then moved down
// (settle_vec, apart from the load so that nothing waits for one that is wanted
// later): loads of single elements at the end of each row took a third of a
// whole backward pass at 4095 columns of 2 bytes.
template <typename T>
__device__ __forceinline__ typename Vec16<T>::type fetch_vec(const T* row, int c, int n) {
    using V = typename Vec16<T>::type;
    constexpr int N = Vec16<T>::N;
    if (n >= N) return *(const V*)(row + min(c, n - N));
    V v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = c + e < n ? row[c + e] : (T)0.f;
    return v;
}
template <typename T>
__device__ __forceinline__ typename Vec16<T>::type settle_vec(typename Vec16<T>::type v, int c, int n) {
    using V = typename Vec16<T>::type;
    constexpr int N = Vec16<T>::N;
    if (n >= N && c > n - N) v = __builtin_bit_cast(V, drop_elements<T>(__builtin_bit_cast(u32v4, v), c - (n - N)));
    return v;
}
template <typename T>
__device__ __forceinline__ typename Vec16<T>::type load_vec(const T* row, int c, int n) {
    return settle_vec<T>(fetch_vec(row, c, n), c, n);
}

// The first n (at most N) of N elements, in at most three pieces.
template <typename T>
__device__ __forceinline__ void store_vec(T* p, int n, const float (&in)[Vec16<T>::N]) {
    using V = typename Vec16<T>::type;
    constexpr int N = Vec16<T>::N;
    V v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (T)in[e];
    if (n >= N) {
        *(V*)p = v;
        return;
    }
    u32v4 u = __builtin_bit_cast(u32v4, v);
    typedef T half __attribute__((ext_vector_type(N / 2), aligned(sizeof(T))));
    typedef uint32_t u32v2 __attribute__((ext_vector_type(2)));
    if (n & (N / 2)) {
        *(half*)p = __builtin_bit_cast(half, u32v2{u[0], u[1]});
        u = u32v4{u[2], u[3], 0, 0};
        p += N / 2;
    }
    if constexpr (N == 8) {
        typedef T two __attribute__((ext_vector_type(2), aligned(sizeof(T))));
        if (n & 2) {
            *(two*)p = __builtin_bit_cast(two, u[0]);
            u[0] = u[1];
            p += 2;
        }
    }
    if (n & 1) {
        typedef T any __attribute__((ext_vector_type(4 / sizeof(T))));
        *p = __builtin_bit_cast(any, u[0])[0];
    }
}

// Sum over the 64 lanes, the same bits in every lane.
__device__ __forceinline__ float wave_sum_f32(float v) {
    const auto step = [](float a, uint32_t b) { return a + __uint_as_float(b); };
    v = step(v, dpp_u32<DPP_QUAD_XOR1>(__float_as_uint(v)));
    v = step(v, dpp_u32<DPP_QUAD_XOR2>(__float_as_uint(v)));
    v = step(v, dpp_u32<DPP_ROW_HALF_MIRROR>(__float_as_uint(v)));
    v = step(v, dpp_u32<DPP_ROW_MIRROR>(__float_as_uint(v)));
    const uint32_t u = __float_as_uint(v);
    return (__uint_as_float(readlane_u32(u, 0)) + __uint_as_float(readlane_u32(u, 16))) +
           (__uint_as_float(readlane_u32(u, 32)) + __uint_as_float(readlane_u32(u, 48)));
}

}  // namespace kb
