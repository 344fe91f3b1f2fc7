// kb_norm.hip -- layer norm, forward and backward.
//
// Forward, per row:   mean = S(x)/C, rstd = 1/sqrt(S((x-mean)^2)/C + eps),
//                     y = (x - mean) rstd w + b.
// Backward, per row:  z = (x - mean) rstd, g = dy w,
//                     dx = rstd (g - S(g)/C - z S(g z)/C);
// over the rows:      dw = S_rows(dy z), db = S_rows(dy).
// Both move bytes: forward reads x and writes y, backward reads dy and x and
// writes dx; the arithmetic is 8 to 14 operations an element.
//
// Measured on an MI355X, where a copy of 4 GB moves 4.8 TB/s: forward of 16,384 x
// 4096 f16 53 us, 5.0 TB/s; backward of the same in bf16 81 us, 5.0 TB/s (part of it
// from the 256 MB last-level cache); backward of 4095 x 4097 f32 47 us, 4.3 TB/s; 16
// rows of 4096, a call's own time, 7 us.
#include "kb_ops.hpp"

namespace kb {
namespace {

constexpr int kThreads = 256;

// Sums over the TPR threads of a row, the same bits in each of them; s: LDS for
// one float per wave and value (rows of more than a wave).  The work-group meets
// once, before the sums are read, so a call may not write the s of the call
// before: the callers take two in turn.
template <int TPR, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float* s) {
    if constexpr (TPR <= 16) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] += __uint_as_float(dpp_u32<DPP_QUAD_XOR1>(__float_as_uint(v[k])));
            v[k] += __uint_as_float(dpp_u32<DPP_QUAD_XOR2>(__float_as_uint(v[k])));
            v[k] += __uint_as_float(dpp_u32<DPP_ROW_HALF_MIRROR>(__float_as_uint(v[k])));
            v[k] += __uint_as_float(dpp_u32<DPP_ROW_MIRROR>(__float_as_uint(v[k])));
        }
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = wave_sum_f32(v[k]);
    }
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;  // waves of a row
        const int wave = (int)threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) s[wave * K + k] = v[k];
        }
        __syncthreads();
        const float* mine = s + wave / W * W * K;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float sum = mine[k];
#pragma unroll
            for (int w = 1; w < W; ++w) sum += mine[w * K + k];
            v[k] = sum;
        }
    }
}

// A row in the registers of TPR threads, E elements each: vector i of a thread
// is at column (i TPR + t) N.  Columns past the row are 0.
template <int DT, int TPR, int E>
struct RowRegs {
    using T = storage_t<DT>;
    static constexpr int N = Vec16<T>::N;
    static constexpr int NV = E / N;
    typename Vec16<T>::type v[NV];

    __device__ __forceinline__ void load(const T* row, int t, int cols) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * N;
            if (c < cols) v[i] = fetch_vec(row, c, cols);
            else v[i] = typename Vec16<T>::type{};
        }
    }
    __device__ __forceinline__ void settle(int t, int cols) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * N;
            if (c < cols) v[i] = settle_vec<T>(v[i], c, cols);
        }
    }
    __device__ __forceinline__ float at(int e) const { return (float)v[e / N][e % N]; }
};

// Elements c .. c + N - 1 of a weight [n], `other` past its end or without one.
template <int N, typename W>
__device__ __forceinline__ void load_weight(const W* w, int c, int n, float other, float* out) {
    constexpr int M = Vec16<W>::N;
#pragma unroll
    for (int k = 0; k < N; k += M) {
        if (w != nullptr && k < n - c) {
            const typename Vec16<W>::type v = load_vec(w, c + k, n);
#pragma unroll
            for (int e = 0; e < M; ++e) out[k + e] = (float)v[e];
        } else {
#pragma unroll
            for (int e = 0; e < M; ++e) out[k + e] = other;
        }
    }
}

// Threads of a row and elements of a thread: the fewest threads that hold the
// row at 16 elements each (8 up to 512 columns), so that a wave or less has a
// row where that is possible and its sums need no meeting.  More elements a
// thread leave too few waves on a CU to cover HBM's latency (backward makes one
// exception, norm_backward).
#define KB_NORM_DISPATCH(COLS, CALL, LONGER)      \
    ((COLS) <= 128    ? CALL<DT, WDT, 16, 8>      \
     : (COLS) <= 512  ? CALL<DT, WDT, 64, 8>      \
     : (COLS) <= 1024 ? CALL<DT, WDT, 64, 16>     \
     : (COLS) <= 2048 ? CALL<DT, WDT, 128, 16>    \
     : (COLS) <= 4096 ? CALL<DT, WDT, 256, 16>    \
     : LONGER)

constexpr int block_of(int tpr) { return tpr > kThreads ? tpr : kThreads; }

// Work-groups of a launch that goes over the rows in strides.
constexpr int64_t kForwardGroups = 2048;

// Forward: the row stays in registers between its two sums and the result; the
// next row is on its way meanwhile.
template <int DT, int WDT, int TPR, int E>
__global__ void __launch_bounds__(block_of(TPR)) norm_forward_rows_kernel(NormForwardParams p) {
    using T = storage_t<DT>;
    using W = storage_t<WDT>;
    using R = RowRegs<DT, TPR, E>;
    constexpr int N = R::N, ROWS = block_of(TPR) / TPR;
    __shared__ float s[2][block_of(TPR) / 64];
    const int t = (int)threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + (int)threadIdx.x / TPR;
    const int64_t last = p.rows - 1;
    const float inv = 1.f / (float)p.cols;
    const auto column = [&](int e) { return (e / N * TPR + t) * N + e % N; };
    float wf[E], bf[E];
#pragma unroll
    for (int i = 0; i < R::NV; ++i) {
        load_weight<N>((const W*)p.w, (i * TPR + t) * N, p.cols, 1.f, wf + i * N);
        load_weight<N>((const W*)p.b, (i * TPR + t) * N, p.cols, 0.f, bf + i * N);
    }
    R next;
    next.load((const T*)p.x.p + min(row, last) * p.x.stride, t, p.cols);
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < p.rows; base += step, row += step) {
        R x = next;
        if (base + step < p.rows) next.load((const T*)p.x.p + min(row + step, last) * p.x.stride, t, p.cols);
        x.settle(t, p.cols);
        float sum[1] = {0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) sum[0] += x.at(e);
        row_sum<TPR>(sum, s[0]);
        const float mean = sum[0] * inv;
        sum[0] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = column(e) < p.cols ? x.at(e) - mean : 0.f;
            sum[0] = fmaf(d, d, sum[0]);
        }
        row_sum<TPR>(sum, s[1]);
        const float rstd = 1.f / sqrtf(fmaf(sum[0], inv, p.eps));
        if (row > last) continue;
        if (t == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
        T* y = (T*)p.y.p + row * p.y.stride;
#pragma unroll
        for (int i = 0; i < R::NV; ++i) {
            float out[N];
#pragma unroll
            for (int e = 0; e < N; ++e) out[e] = fmaf((x.at(i * N + e) - mean) * rstd, wf[i * N + e], bf[i * N + e]);
            const int c = (i * TPR + t) * N;
            if (c < p.cols) store_vec(y + c, p.cols - c, out);
        }
    }
}

template <int DT, int WDT, int TPR, int E>
hipError_t norm_forward_rows(const NormForwardParams& p, hipStream_t stream) {
    constexpr int ROWS = block_of(TPR) / TPR;
    const int64_t groups = (p.rows + ROWS - 1) / ROWS;
    norm_forward_rows_kernel<DT, WDT, TPR, E>
        <<<dim3((unsigned)(groups < kForwardGroups ? groups : kForwardGroups)), block_of(TPR), 0, stream>>>(p);
    return hipGetLastError();
}

// Backward: dy and x of a row in registers for the two sums and dx; dw and db of
// the thread's columns add up over the rows that it sees.  At the end the row
// groups of a work-group meet in LDS and are added in their order, a column a
// thread, as one part.
// SUMS: with dw and db.  They take two registers a column, too many for rows of
// more than 8192 (spilled, 4096 x 16,384 f32 took 290 us): there a pass of its
// own over dy and x adds the columns.
template <int DT, int WDT, int TPR, int E, bool SUMS>
__global__ void __launch_bounds__(block_of(TPR)) norm_backward_rows_kernel(NormBackwardParams p) {
    using T = storage_t<DT>;
    using W = storage_t<WDT>;
    using R = RowRegs<DT, TPR, E>;
    constexpr int N = R::N, ROWS = block_of(TPR) / TPR;
    __shared__ float s[2][2 * block_of(TPR) / 64];
    const int t = (int)threadIdx.x % TPR, group = (int)threadIdx.x / TPR;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + group;
    const int64_t last = p.rows - 1;
    const float inv = 1.f / (float)p.cols;
    const auto column = [&](int e) { return (e / N * TPR + t) * N + e % N; };
    float wf[E], dw[SUMS ? E : 1], db[SUMS ? E : 1];
#pragma unroll
    for (int i = 0; i < R::NV; ++i) load_weight<N>((const W*)p.w, (i * TPR + t) * N, p.cols, 1.f, wf + i * N);
#pragma unroll
    for (int e = 0; e < (SUMS ? E : 1); ++e) dw[e] = db[e] = 0.f;
    R next_dy, next_x;
    next_dy.load((const T*)p.dy.p + min(row, last) * p.dy.stride, t, p.cols);
    next_x.load((const T*)p.x.p + min(row, last) * p.x.stride, t, p.cols);
    float next_mean = p.mean[min(row, last)], next_rstd = p.rstd[min(row, last)];
    int turn = 0;
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < p.rows; base += step, row += step, turn ^= 1) {
        R dy = next_dy, x = next_x;
        const float mean = next_mean, rstd = next_rstd;
        if (base + step < p.rows) {
            const int64_t r = min(row + step, last);
            next_dy.load((const T*)p.dy.p + r * p.dy.stride, t, p.cols);
            next_x.load((const T*)p.x.p + r * p.x.stride, t, p.cols);
            next_mean = p.mean[r];
            next_rstd = p.rstd[r];
        }
        dy.settle(t, p.cols);
        x.settle(t, p.cols);
        const bool live = row <= last;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = dy.at(e), g = d * wf[e];
            // past the row dy is 0; z there is not, and may not be finite
            const float z = column(e) < p.cols ? (x.at(e) - mean) * rstd : 0.f;
            sum[0] += g;
            sum[1] = fmaf(g, z, sum[1]);
            if (SUMS && live) {
                dw[SUMS ? e : 0] = fmaf(d, z, dw[SUMS ? e : 0]);
                db[SUMS ? e : 0] += d;
            }
        }
        if (!p.dx.p) continue;
        row_sum<TPR>(sum, s[turn]);
        if (!live) continue;
        const float mg = sum[0] * inv, mgz = sum[1] * inv;
        T* dx = (T*)p.dx.p + row * p.dx.stride;
#pragma unroll
        for (int i = 0; i < R::NV; ++i) {
            float out[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int e = i * N + k;
                const float z = (x.at(e) - mean) * rstd;
                out[k] = rstd * (fmaf(dy.at(e), wf[e], -mg) - z * mgz);
            }
            const int c = (i * TPR + t) * N;
            if (c < p.cols) store_vec(dx + c, p.cols - c, out);
        }
    }
    if constexpr (SUMS) {
        if (!p.dw && !p.db) return;
        float* part = p.part + (int64_t)blockIdx.x * 2 * p.cols;
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        if constexpr (ROWS > 1) {
            __shared__ __align__(16) float sums[2][ROWS][TPR * E];
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const int c = (e / N * TPR + t) * N + e % N;
                *(f32x4*)&sums[0][group][c] = f32x4{dw[e], dw[e + 1], dw[e + 2], dw[e + 3]};
                *(f32x4*)&sums[1][group][c] = f32x4{db[e], db[e + 1], db[e + 2], db[e + 3]};
            }
            __syncthreads();
            for (int c = (int)threadIdx.x; c < p.cols; c += block_of(TPR)) {
                float w = sums[0][0][c], b = sums[1][0][c];
#pragma unroll
                for (int k = 1; k < ROWS; ++k) {
                    w += sums[0][k][c];
                    b += sums[1][k][c];
                }
                part[c] = w;
                part[p.cols + c] = b;
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const int c = (e / N * TPR + t) * N + e % N;
                const float w[4] = {dw[e], dw[e + 1], dw[e + 2], dw[e + 3]}, b[4] = {db[e], db[e + 1], db[e + 2], db[e + 3]};
                if (c < p.cols) {
                    store_vec(part + c, p.cols - c, w);
                    store_vec(part + p.cols + c, p.cols - c, b);
                }
            }
        }
    }
}

// dw and db from the parts: a column a lane, the parts dealt out to 16 waves,
// whose sums are added in their order.  A launch has fewer than 2^32 threads, so
// its work-groups are limited and go over longer rows in strides.
constexpr int kJoinWaves = 16;
constexpr int64_t kJoinGroups = (int64_t)1 << 21;
template <int WDT>
__global__ void __launch_bounds__(64 * kJoinWaves) norm_backward_join_kernel(NormBackwardParams p, int parts) {
    using W = storage_t<WDT>;
    __shared__ float s[kJoinWaves][64];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int64_t n = 2 * (int64_t)p.cols, step = (int64_t)gridDim.x * 64;
    for (int64_t first = (int64_t)blockIdx.x * 64; first < n; first += step) {
        const int64_t i = first + lane;
        float sum = 0.f;
        if (i < n) {
#pragma unroll 8
            for (int k = wave; k < parts; k += kJoinWaves) sum += p.part[(int64_t)k * n + i];
        }
        s[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && i < n) {
#pragma unroll
            for (int k = 1; k < kJoinWaves; ++k) sum += s[k][lane];
            W* out = (W*)(i < p.cols ? p.dw : p.db);
            if (out) out[i < p.cols ? i : i - p.cols] = (W)sum;
        }
        if (first + step < n) __syncthreads();  // (the sums are read)
    }
}

template <int WDT>
hipError_t norm_backward_join(const NormBackwardParams& p, int parts, hipStream_t stream) {
    const int64_t groups = (2 * (int64_t)p.cols + 63) / 64;
    norm_backward_join_kernel<WDT>
        <<<dim3((unsigned)(groups < kJoinGroups ? groups : kJoinGroups)), 64 * kJoinWaves, 0, stream>>>(p, parts);
    return hipGetLastError();
}

template <int DT, int WDT, int TPR, int E>
hipError_t norm_backward_rows(const NormBackwardParams& p, hipStream_t stream) {
    constexpr int ROWS = block_of(TPR) / TPR;
    const int64_t groups = (p.rows + ROWS - 1) / ROWS;
    const int parts = norm_parts(groups, p.cols, sizeof(storage_t<DT>));
    if (parts > 0)
        norm_backward_rows_kernel<DT, WDT, TPR, E, true><<<dim3((unsigned)parts), block_of(TPR), 0, stream>>>(p);
    return p.dw || p.db ? norm_backward_join<WDT>(p, parts, stream) : hipGetLastError();
}

// ------------------------------------- rows that do not fit in the registers --
// A column is a uint32_t: the step past the last one may pass 2^31.

template <typename V, int N>
__device__ __forceinline__ void widen(V v, float (&out)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = (float)v[e];
}

// Sums over a work-group of kThreads.
template <int K>
__device__ __forceinline__ void block_sum(float (&v)[K], float* s) {
    row_sum<kThreads>(v, s);
    __syncthreads();
}

// A row per work-group, read once for the mean, once for the deviations and
// once for the result.
template <int DT, int WDT>
__global__ void __launch_bounds__(kThreads) norm_forward_long_kernel(NormForwardParams p) {
    using T = storage_t<DT>;
    using W = storage_t<WDT>;
    constexpr int N = Vec16<T>::N;
    __shared__ float s[kThreads / 64];
    const int64_t row = blockIdx.x;
    const T* x = (const T*)p.x.p + row * p.x.stride;
    T* y = (T*)p.y.p + row * p.y.stride;
    const float inv = 1.f / (float)p.cols;
    float acc[1] = {0.f}, v[N];
    for (uint32_t c = threadIdx.x * N; c < (uint32_t)p.cols; c += kThreads * N) {
        widen(load_vec(x, c, p.cols), v);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[0] += v[e];
    }
    block_sum(acc, s);
    const float mean = acc[0] * inv;
    acc[0] = 0.f;
    for (uint32_t c = threadIdx.x * N; c < (uint32_t)p.cols; c += kThreads * N) {
        widen(load_vec(x, c, p.cols), v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = e < p.cols - (int)c ? v[e] - mean : 0.f;
            acc[0] = fmaf(d, d, acc[0]);
        }
    }
    block_sum(acc, s);
    const float rstd = 1.f / sqrtf(fmaf(acc[0], inv, p.eps));
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
    }
    for (uint32_t c = threadIdx.x * N; c < (uint32_t)p.cols; c += kThreads * N) {
        widen(load_vec(x, c, p.cols), v);
        float w[N], b[N];
        load_weight<N>((const W*)p.w, c, p.cols, 1.f, w);
        load_weight<N>((const W*)p.b, c, p.cols, 0.f, b);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = fmaf((v[e] - mean) * rstd, w[e], b[e]);
        store_vec(y + c, p.cols - c, v);
    }
}

// dx: a row per work-group, read for the two sums and again for the result.
template <int DT, int WDT>
__global__ void __launch_bounds__(kThreads) norm_backward_dx_long_kernel(NormBackwardParams p) {
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
    for (uint32_t c = threadIdx.x * N; c < (uint32_t)p.cols; c += kThreads * N) {
        widen(load_vec(dy, c, p.cols), a);
        widen(load_vec(x, c, p.cols), v);
        float w[N];
        load_weight<N>((const W*)p.w, c, p.cols, 1.f, w);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float g = a[e] * w[e], z = e < p.cols - (int)c ? (v[e] - mean) * rstd : 0.f;
            acc[0] += g;
            acc[1] = fmaf(g, z, acc[1]);
        }
    }
    block_sum(acc, s);
    const float mg = acc[0] * inv, mgz = acc[1] * inv;
    for (uint32_t c = threadIdx.x * N; c < (uint32_t)p.cols; c += kThreads * N) {
        widen(load_vec(dy, c, p.cols), a);
        widen(load_vec(x, c, p.cols), v);
        float w[N];
        load_weight<N>((const W*)p.w, c, p.cols, 1.f, w);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float g = a[e] * w[e], z = (v[e] - mean) * rstd;
            v[e] = rstd * (g - mg - z * mgz);
        }
        store_vec(dx + c, p.cols - c, v);
    }
}

// Partial column sums: work-group (strip, part) adds the rows of its part over
// a strip of kThreads vectors of columns.
template <int DT>
__global__ void __launch_bounds__(kThreads) norm_backward_part_long_kernel(NormBackwardParams p, int parts) {
    using T = storage_t<DT>;
    constexpr int N = Vec16<T>::N;
    const uint32_t c = (blockIdx.x * kThreads + threadIdx.x) * N;
    if (c >= (uint32_t)p.cols) return;
    float dw[N], db[N], a[N], v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) dw[e] = db[e] = 0.f;
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < p.rows; row += parts) {
        widen(load_vec((const T*)p.dy.p + row * p.dy.stride, c, p.cols), a);
        widen(load_vec((const T*)p.x.p + row * p.x.stride, c, p.cols), v);
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
        if (e < p.cols - (int)c) {
            out[c + e] = dw[e];
            out[(int64_t)p.cols + c + e] = db[e];
        }
}

template <int DT, int WDT>
hipError_t norm_forward_rows_long(const NormForwardParams& p, hipStream_t stream) {
    norm_forward_long_kernel<DT, WDT><<<dim3((unsigned)p.rows), kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

template <int DT, int WDT>
hipError_t norm_backward_rows_long(const NormBackwardParams& p, hipStream_t stream) {
    if (p.dx.p && p.rows > 0) {
        if (p.cols <= 16384)
            norm_backward_rows_kernel<DT, WDT, 1024, 16, false>
                <<<dim3((unsigned)(p.rows < kForwardGroups ? p.rows : kForwardGroups)), 1024, 0, stream>>>(p);
        else
            norm_backward_dx_long_kernel<DT, WDT><<<dim3((unsigned)p.rows), kThreads, 0, stream>>>(p);
    }
    if (!p.dw && !p.db) return hipGetLastError();
    const int parts = norm_parts(p.rows, p.cols, sizeof(storage_t<DT>));
    constexpr int strip = kThreads * Vec16<storage_t<DT>>::N;
    if (parts > 0)
        norm_backward_part_long_kernel<DT>
            <<<dim3((unsigned)((p.cols + (int64_t)strip - 1) / strip), (unsigned)parts), kThreads, 0, stream>>>(p, parts);
    return norm_backward_join<WDT>(p, parts, stream);
}

template <int DT, int WDT>
hipError_t norm_forward(const NormForwardParams& p, hipStream_t stream) {
    return KB_NORM_DISPATCH(p.cols, norm_forward_rows, (p.cols <= 8192 ? norm_forward_rows<DT, WDT, 512, 16> : p.cols <= 16384 ? norm_forward_rows<DT, WDT, 1024, 16> : norm_forward_rows_long<DT, WDT>))(p, stream);
}

template <int DT, int WDT>
hipError_t norm_backward(const NormBackwardParams& p, hipStream_t stream) {
    // Rows of 16 bits of up to 5120 columns: 24 elements a thread leave fewer threads
    // idle than 512 threads would (4096 x 4224 bf16: 33 us, 38 with 512 threads; x
    // 5120: 36, 38; x 6144: 43, 41; 4096 x 4100 f32: 51, 48).
    if constexpr (DT != DT_F32) {
        if (p.cols > 4096 && p.cols <= 5120) return norm_backward_rows<DT, WDT, 256, 24>(p, stream);
    }
    return KB_NORM_DISPATCH(p.cols, norm_backward_rows, (p.cols <= 8192 ? norm_backward_rows<DT, WDT, 512, 16> : norm_backward_rows_long<DT, WDT>))(p, stream);
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
