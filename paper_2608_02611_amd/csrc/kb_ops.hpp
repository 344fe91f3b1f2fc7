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

// Row stripes whose column sums are kept apart (NormBackwardParams::part).
constexpr int kNormMaxParts = 512;
inline size_t norm_part_bytes(int64_t rows, int64_t cols) {
    const int64_t parts = rows < kNormMaxParts ? rows : (int64_t)kNormMaxParts;
    return ((size_t)parts * 2 * (size_t)cols * sizeof(float) + 15) & ~(size_t)15;
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
    int splits; // forward: parts of the keys
    int whole;  // rows of q, k, v (and dout) are aligned to 16 bytes and made of 16-byte chunks
    float* ws;
};

// Forward: query rows of a work-group and keys of a tile, and into how many parts
// the keys are split so that few query rows still fill the device: up to kFill
// work-groups (two for each of 256 CUs, and as many again, as parts of a ragged
// batch end at different times), of no less than kSplitKeys keys each.
constexpr int kAttnRows = 128;
constexpr int kAttnKeys = 64;
constexpr int64_t kFill = 1024;
constexpr int64_t kSplitKeys = 512;
inline int attn_splits(const AttnParams& p) {
    const int64_t work_groups =
        (int64_t)p.batch * p.kv_heads * (((int64_t)p.len_q * p.group + kAttnRows - 1) / kAttnRows);
    if (work_groups == 0 || 2 * work_groups > kFill) return 1;
    const int64_t want = kFill / work_groups, most = p.len_k / kSplitKeys;
    return (int)(want < most ? want : most > 1 ? most : 1);
}
// Workspace of a split forward pass, in floats: for each query row and part the
// sums over its keys (dim rounded up to 4), then m, l and the rounded l.
__host__ __device__ inline int64_t split_row(const AttnParams& p) { return (p.dim + 3) / 4 * 4 + 4; }
inline int64_t split_floats(const AttnParams& p, int splits) {
    return splits > 1 ? (int64_t)p.batch * p.heads * p.len_q * splits * split_row(p) : 0;
}

// Workspace of the backward pass, in floats: D_i and lse_i for every query row, then
// (F16) the largest squared norm of each block of kNormBlock rows of dout and
// of v, then a word for each work-group of kAttnKeyRows keys.
constexpr int kNormBlock = 64;
constexpr int kAttnKeyRows = 128;
inline int64_t norm_blocks(int64_t len) { return (len + kNormBlock - 1) / kNormBlock; }

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

// 16 bytes of elements, readable at any element's alignment (gfx950 loads
// and stores dwords at any byte address).
template <typename T>
struct Vec16 {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// Elements [0, n) of p as floats, 0 past them (n >= N: all).
template <typename T>
__device__ __forceinline__ void load_vec(const T* p, int n, float (&out)[Vec16<T>::N]) {
    constexpr int N = Vec16<T>::N;
    if (n >= N) {
        const typename Vec16<T>::type v = *(const typename Vec16<T>::type*)p;
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = e < n ? (float)p[e] : 0.f;
    }
}

template <typename T>
__device__ __forceinline__ void store_vec(T* p, int n, const float (&in)[Vec16<T>::N]) {
    constexpr int N = Vec16<T>::N;
    if (n >= N) {
        typename Vec16<T>::type v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)in[e];
        *(typename Vec16<T>::type*)p = v;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < n) p[e] = (T)in[e];
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
