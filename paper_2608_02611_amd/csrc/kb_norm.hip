// kb_norm.hip -- layer norm, forward and backward.
//
// Forward, per row:   mean = S(x)/C, rstd = 1/sqrt(S((x-mean)^2)/C + eps),
//                     y = (x - mean) rstd w + b.
// Backward, per row:  z = (x - mean) rstd, g = dy w,
//                     dx = rstd (g - S(g)/C - z S(g z)/C);
// over the rows:      dw = S_rows(dy z), db = S_rows(dy).
// Both move bytes: forward reads x and writes y, backward reads dy and x and
// writes dx; the arithmetic is 8 to 14 operations an element.
#include "kb_ops.hpp"

namespace kb {
namespace {

constexpr int kThreads = 256;

// Sums over the work-group, the same bits in every thread; s: one float per
// wave and value.
template <int K>
__device__ __forceinline__ void block_sum(float (&v)[K], float* s) {
    constexpr int W = kThreads / 64;
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wave_sum_f32(v[k]);
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) s[k * W + wave] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] = s[k * W];
#pragma unroll
        for (int w = 1; w < W; ++w) v[k] += s[k * W + w];
    }
    __syncthreads();
}

// A row per work-group, read once for the mean, once for the deviations and
// once for the result.
template <int DT, int WDT>
__global__ void __launch_bounds__(kThreads) norm_forward_kernel(NormForwardParams p) {
    using T = storage_t<DT>;
    using W = storage_t<WDT>;
    constexpr int N = Vec16<T>::N;
    __shared__ float s[kThreads / 64];
    const int64_t row = blockIdx.x;
    const T* x = (const T*)p.x.p + row * p.x.stride;
    T* y = (T*)p.y.p + row * p.y.stride;
    const float inv = 1.f / (float)p.cols;
    float acc[1] = {0.f}, v[N];
    for (int c = threadIdx.x * N; c < p.cols; c += kThreads * N) {
        load_vec(x + c, p.cols - c, v);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[0] += v[e];
    }
    block_sum(acc, s);
    const float mean = acc[0] * inv;
    acc[0] = 0.f;
    for (int c = threadIdx.x * N; c < p.cols; c += kThreads * N) {
        load_vec(x + c, p.cols - c, v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = c + e < p.cols ? v[e] - mean : 0.f;
            acc[0] = fmaf(d, d, acc[0]);
        }
    }
    block_sum(acc, s);
    const float rstd = 1.f / sqrtf(fmaf(acc[0], inv, p.eps));
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
    }
    for (int c = threadIdx.x * N; c < p.cols; c += kThreads * N) {
        load_vec(x + c, p.cols - c, v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int col = min(c + e, p.cols - 1);
            const float w = p.w ? (float)((const W*)p.w)[col] : 1.f;
            const float b = p.b ? (float)((const W*)p.b)[col] : 0.f;
            v[e] = fmaf((v[e] - mean) * rstd, w, b);
        }
        store_vec(y + c, p.cols - c, v);
    }
}

// dx: a row per work-group, read for the two sums and again for the result.
template <int DT, int WDT>
__global__ void __launch_bounds__(kThreads) norm_backward_dx_kernel(NormBackwardParams p) {
    using T = storage_t<DT>;
    using W = storage_t<WDT>;
    constexpr int N = Vec16<T>::N;
    __shared__ float s[2 * kThreads / 64];
    const int64_t row = blockIdx.x;
    const T* dy = (const T*)p.dy.p + row * p.dy.stride;
    const T* x = (const T*)p.x.p + row * p.x.stride;
    T* dx = (T*)p.dx.p + row * p.dx.stride;
    const float mean = p.mean[row], rstd = p.rstd[row], inv = 1.f / (float)p.cols;
    float acc[2] = {0.f, 0.f}, a[N], v[N];
    for (int c = threadIdx.x * N; c < p.cols; c += kThreads * N) {
        load_vec(dy + c, p.cols - c, a);
        load_vec(x + c, p.cols - c, v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const bool in = c + e < p.cols;
            const float g = in ? a[e] * (p.w ? (float)((const W*)p.w)[c + e] : 1.f) : 0.f;
            const float z = in ? (v[e] - mean) * rstd : 0.f;
            acc[0] += g;
            acc[1] = fmaf(g, z, acc[1]);
        }
    }
    block_sum(acc, s);
    const float mg = acc[0] * inv, mgz = acc[1] * inv;
    for (int c = threadIdx.x * N; c < p.cols; c += kThreads * N) {
        load_vec(dy + c, p.cols - c, a);
        load_vec(x + c, p.cols - c, v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float g = a[e] * (p.w ? (float)((const W*)p.w)[min(c + e, p.cols - 1)] : 1.f);
            const float z = (v[e] - mean) * rstd;
            v[e] = rstd * (g - mg - z * mgz);
        }
        store_vec(dx + c, p.cols - c, v);
    }
}

// Partial column sums: work-group (strip, part) adds the rows of its part over
// a strip of kThreads vectors of columns.
template <int DT>
__global__ void __launch_bounds__(kThreads) norm_backward_part_kernel(NormBackwardParams p, int parts) {
    using T = storage_t<DT>;
    constexpr int N = Vec16<T>::N;
    const int c = (blockIdx.x * kThreads + threadIdx.x) * N;
    if (c >= p.cols) return;
    float dw[N], db[N], a[N], v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) dw[e] = db[e] = 0.f;
    for (int64_t row = blockIdx.y; row < p.rows; row += parts) {
        load_vec((const T*)p.dy.p + row * p.dy.stride + c, p.cols - c, a);
        load_vec((const T*)p.x.p + row * p.x.stride + c, p.cols - c, v);
        const float mean = p.mean[row], rstd = p.rstd[row];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            dw[e] = fmaf(a[e], (v[e] - mean) * rstd, dw[e]);
            db[e] += a[e];
        }
    }
    float* out = p.part + (int64_t)blockIdx.y * 2 * p.cols;
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (c + e < p.cols) {
            out[c + e] = dw[e];
            out[p.cols + c + e] = db[e];
        }
}

// dw and db: column sums of the partial sums, in the order of the parts.
template <int WDT>
__global__ void __launch_bounds__(kThreads) norm_backward_join_kernel(NormBackwardParams p, int parts) {
    using W = storage_t<WDT>;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= 2 * (int64_t)p.cols) return;
    float sum = 0.f;
    for (int k = 0; k < parts; ++k) sum += p.part[(int64_t)k * 2 * p.cols + i];
    W* out = (W*)(i < p.cols ? p.dw : p.db);
    if (out) out[i < p.cols ? i : i - p.cols] = (W)sum;
}

template <int DT, int WDT>
hipError_t norm_forward(const NormForwardParams& p, hipStream_t stream) {
    norm_forward_kernel<DT, WDT><<<dim3((unsigned)p.rows), kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

template <int DT, int WDT>
hipError_t norm_backward(const NormBackwardParams& p, hipStream_t stream) {
    if (p.dx.p && p.rows > 0) norm_backward_dx_kernel<DT, WDT><<<dim3((unsigned)p.rows), kThreads, 0, stream>>>(p);
    if (p.dw || p.db) {
        const int parts = (int)(p.rows < kNormMaxParts ? p.rows : (int64_t)kNormMaxParts);
        constexpr int strip = kThreads * Vec16<storage_t<DT>>::N;
        if (parts > 0)
            norm_backward_part_kernel<DT>
                <<<dim3((unsigned)((p.cols + (int64_t)strip - 1) / strip), (unsigned)parts), kThreads, 0, stream>>>(p, parts);
        norm_backward_join_kernel<WDT>
            <<<dim3((unsigned)((2 * (int64_t)p.cols + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(p, parts);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_forward(int dtype, int wdtype, const NormForwardParams& p, hipStream_t stream) {
    if (dtype == DT_F32) return norm_forward<DT_F32, DT_F32>(p, stream);
    if (dtype == DT_F16)
        return wdtype == DT_F32 ? norm_forward<DT_F16, DT_F32>(p, stream) : norm_forward<DT_F16, DT_F16>(p, stream);
    return wdtype == DT_F32 ? norm_forward<DT_BF16, DT_F32>(p, stream) : norm_forward<DT_BF16, DT_BF16>(p, stream);
}

hipError_t launch_norm_backward(int dtype, int wdtype, const NormBackwardParams& p, hipStream_t stream) {
    if (dtype == DT_F32) return norm_backward<DT_F32, DT_F32>(p, stream);
    if (dtype == DT_F16)
        return wdtype == DT_F32 ? norm_backward<DT_F16, DT_F32>(p, stream) : norm_backward<DT_F16, DT_F16>(p, stream);
    return wdtype == DT_F32 ? norm_backward<DT_BF16, DT_F32>(p, stream) : norm_backward<DT_BF16, DT_BF16>(p, stream);
}

}  // namespace kb
