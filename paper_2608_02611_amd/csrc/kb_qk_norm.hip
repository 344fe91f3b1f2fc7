// kb_qk_norm.hip -- norms of query and key heads with the position rotation,
// forward and backward.
//
// Forward, for each head row x of a token:  r = 1 / sqrt(S(x^2) / D + eps),
//   g = x r w, and of the first `rot` elements each pair (a, b) becomes
//   (a cos - b sin, b cos + a sin) of the token's angle for that pair.
// Backward:  g = dy turned the other way, z = x r, u = g w,
//   dx = r (u - z S(u z) / D), dw = S(g z) over tokens and heads.
// Both move bytes: forward reads x and writes y, backward reads dy and x and
// writes dx.  A token's angles are the same for all of its heads, so a wave takes
// the head rows of one token and works the angles out once, one a lane.
//
// Measured on an MI355X, where a copy of 4 GB moves 4.8 TB/s: forward of 16,384
// tokens of 32 + 8 heads of 128, f16, 72 us, 4.7 TB/s (with the weights read element
// by element 89); backward of the same in bf16 119 us, 4.2 TB/s, 4 of it the second
// kernel.  16 tokens, a call's own time, 9 us, of which the kernel has 4.7.
#include "kb_ops.hpp"

namespace kb {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxPairs = KB_QK_MAX_DIM / 2;

// cos and sin of position * freq.  The angle is exact: the binary64 product of a
// 31-bit and a 24-bit number, and what its rounding left.  In turns, less the
// nearest quarter, it is off by less than 2^-56 up to angles of 2^50 (1 / (2 pi) in
// two parts, the first product's rounding taken back by the fma); then Taylor's
// series on [-pi/4, pi/4], whose first term left out is under 2^-28.
__device__ __forceinline__ void turn_of(int position, float freq, float* cos_out, float* sin_out) {
    constexpr double kInv = 0.15915494309189535, kInvLow = -9.8393350380770985e-18;  // 1 / (2 pi)
    constexpr double kTwoPi = 6.283185307179586;
    const double n = (double)position, f = (double)freq;
    const double angle = n * f, left = fma(n, f, -angle);
    const double quarters = rint(4.0 * (angle * kInv));
    double t = fma(angle, kInv, -0.25 * quarters);
    t = fma(angle, kInvLow, t);
    t = fma(left, kInv, t);
    const float r = (float)(t * kTwoPi), q = r * r;
    float s = fmaf(q, 2.7557319e-6f, -1.9841270e-4f);
    s = fmaf(q, s, 8.3333333e-3f);
    s = fmaf(q, s, -1.6666667e-1f);
    s = fmaf(r * q, s, r);
    float c = fmaf(q, -2.7557319e-7f, 2.4801587e-5f);
    c = fmaf(q, c, -1.3888889e-3f);
    c = fmaf(q, c, 4.1666667e-2f);
    c = fmaf(q, c, -0.5f);
    c = fmaf(q, c, 1.f);
    const int k = (int)(quarters - 4.0 * floor(quarters * 0.25));
    const float a = k & 1 ? s : c, b = k & 1 ? c : s;
    *cos_out = (k + 1) & 2 ? -a : a;
    *sin_out = k & 2 ? -b : b;
}

// What a lane has of each head row: a unit of two vectors of V elements, at
// `first` and `second`, that make V rotating pairs: elements i and V + i of the
// unit, or 2i and 2i + 1 (NEAR).  Behind the rotating units come units of the
// other elements; the last of them may lack its second vector.  A row is held by
// `lanes` lanes, a power of two, so a wave has 64 / lanes rows at a time.
template <int DT, int V>
struct Vec {
    typedef storage_t<DT> type __attribute__((ext_vector_type(V), aligned(sizeof(storage_t<DT>))));
};

template <int DT, int V, bool NEAR>
struct Unit {
    using T = storage_t<DT>;
    using VT = typename Vec<DT, V>::type;
    int first, second, pair;  // pair: the first of its V pairs
    bool in, two, rotates;

    __device__ __forceinline__ void set(int u, int dim, int rot) {
        const int rotating = rot / (2 * V);
        rotates = u < rotating;
        pair = rotates ? V * u : 0;
        if (rotates) {
            first = NEAR ? 2 * V * u : V * u;
            second = NEAR ? first + V : rot / 2 + V * u;
        } else {
            first = rot + 2 * V * (u - rotating);
            second = first + V;
        }
        in = first < dim;
        two = second < dim;
    }
    __device__ __forceinline__ void load(const T* row, bool live, VT (&v)[2]) const {
        v[0] = v[1] = VT{};
        if (live && in) v[0] = *(const VT*)(row + first);
        if (live && two && in) v[1] = *(const VT*)(row + second);
    }
    __device__ __forceinline__ void store(T* row, bool live, const float (&x)[2 * V]) const {
        VT v[2];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[0][e] = (T)x[e];
            v[1][e] = (T)x[V + e];
        }
        if (live && in) *(VT*)(row + first) = v[0];
        if (live && two && in) *(VT*)(row + second) = v[1];
    }
    // The pairs turned by (cos, sin); sign -1: the other way.
    __device__ __forceinline__ void turn(float (&x)[2 * V], const float (&c)[V], const float (&s)[V], float sign) const {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int ia = NEAR ? 2 * i : i, ib = NEAR ? 2 * i + 1 : V + i;
            const float a = x[ia], b = x[ib], si = sign * s[i];
            x[ia] = rotates ? fmaf(a, c[i], -(b * si)) : a;
            x[ib] = rotates ? fmaf(b, c[i], a * si) : b;
        }
    }
    template <typename W>
    __device__ __forceinline__ void weight_as(const W* w, float (&out)[2 * V]) const {
        typedef W vec __attribute__((ext_vector_type(V), aligned(sizeof(W))));
        vec v[2];
#pragma unroll
        for (int e = 0; e < V; ++e) v[0][e] = v[1][e] = (W)1.f;
        if (w != nullptr && in) v[0] = *(const vec*)(w + first);
        if (w != nullptr && in && two) v[1] = *(const vec*)(w + second);
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) out[e] = (float)v[e / V][e % V];
    }
    __device__ __forceinline__ void weight(const void* w, int w_f32, float (&out)[2 * V]) const {
        if (DT == DT_F32 || w_f32) weight_as((const float*)w, out);
        else weight_as((const T*)w, out);
    }
};

// Sum over the lanes of a row, the same bits in each.
__device__ __forceinline__ float row_sum(float v, int lanes) {
    if (lanes > 1) v += __uint_as_float(dpp_u32<DPP_QUAD_XOR1>(__float_as_uint(v)));
    if (lanes > 2) v += __uint_as_float(dpp_u32<DPP_QUAD_XOR2>(__float_as_uint(v)));
    if (lanes > 4) v += __uint_as_float(dpp_u32<DPP_ROW_HALF_MIRROR>(__float_as_uint(v)));
    if (lanes > 8) v += __uint_as_float(dpp_u32<DPP_ROW_MIRROR>(__float_as_uint(v)));
    if (lanes > 16) v += __shfl_xor(v, 16);
    if (lanes > 32) v += __shfl_xor(v, 32);
    return v;
}

// The token's angles, by all lanes of a wave into its own LDS.
__device__ __forceinline__ void token_turns(const QkParams& p, int64_t token, int lane, float (*turns)[kMaxPairs]) {
    const int position = p.positions[token];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int i = lane; i < p.rot / 2; i += 64) turn_of(position, p.freqs[i], &turns[0][i], &turns[1][i]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// Those of the lane's units.
template <int V, int E>
__device__ __forceinline__ void unit_turns(const float (*turns)[kMaxPairs], const int (&pair)[E], const bool (&rotates)[E],
                                           float (&c)[E][V], float (&s)[E][V]) {
#pragma unroll
    for (int n = 0; n < E; ++n)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            c[n][i] = rotates[n] ? turns[0][pair[n] + i] : 1.f;
            s[n][i] = rotates[n] ? turns[1][pair[n] + i] : 0.f;
        }
}

// Backward: lanes of a row, passes over a token that a wave makes at a time, and the
// work-groups of q and of k.
struct BackwardPlan {
    int lanes, passes_each, parts[2];
};

// A wave's passes over a token: `per` rows of q, or of k, in each.
struct Passes {
    int per, of_q, all;
    __device__ __forceinline__ Passes(const QkParams& p, int lanes) {
        per = 64 / lanes;
        of_q = (p.heads[0] + per - 1) / per;
        all = of_q + (p.heads[1] + per - 1) / per;
    }
};

template <int DT, int V, int E, bool NEAR>
__global__ void __launch_bounds__(kThreads) qk_forward_kernel(QkParams p, int lanes, int passes_each) {
    using T = storage_t<DT>;
    using U = Unit<DT, V, NEAR>;
    __shared__ __align__(16) float turns[kWaves][2][kMaxPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const Passes ps(p, lanes);
    const int in_row = lane & (lanes - 1), row0 = lane / lanes;
    const int from = (int)blockIdx.y * passes_each, to = min(ps.all, from + passes_each);
    const float inv = 1.f / (float)p.dim;
    U unit[E];
#pragma unroll
    for (int n = 0; n < E; ++n) unit[n].set(in_row + n * lanes, p.dim, p.rot);
    int pair[E];
    bool rotates[E];
    float w[2][E][2 * V];
#pragma unroll
    for (int n = 0; n < E; ++n) {
        pair[n] = unit[n].pair;
        rotates[n] = unit[n].rotates;
        unit[n].weight(p.w[0], p.w_f32, w[0][n]);
        unit[n].weight(p.w[1], p.w_f32, w[1][n]);
    }
    const int64_t step = (int64_t)gridDim.x * kWaves;
    for (int64_t token = (int64_t)blockIdx.x * kWaves + wave; token < p.tokens; token += step) {
        typename U::VT next[E][2];
        const auto fetch = [&](int pass) {
            const int t = pass >= ps.of_q, row = (t ? pass - ps.of_q : pass) * ps.per + row0;
            const T* x = (const T*)p.x[t].p + token * p.x[t].st + row * p.x[t].sh;
#pragma unroll
            for (int n = 0; n < E; ++n) unit[n].load(x, row < p.heads[t], next[n]);
        };
        fetch(from);
        float c[E][V], s[E][V];
        if (p.rot > 0) {
            token_turns(p, token, lane, turns[wave]);
            unit_turns<V, E>(turns[wave], pair, rotates, c, s);
        }
        for (int pass = from; pass < to; ++pass) {
            float x[E][2 * V], sum = 0.f;
#pragma unroll
            for (int n = 0; n < E; ++n)
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    x[n][e] = (float)next[n][e / V][e % V];
                    sum = fmaf(x[n][e], x[n][e], sum);
                }
            if (pass + 1 < to) fetch(pass + 1);
            const float r = 1.f / sqrtf(fmaf(row_sum(sum, lanes), inv, p.eps));
            const int t = pass >= ps.of_q, row = (t ? pass - ps.of_q : pass) * ps.per + row0;
            T* y = (T*)p.y[t].p + token * p.y[t].st + row * p.y[t].sh;
#pragma unroll
            for (int n = 0; n < E; ++n) {
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) x[n][e] = x[n][e] * r * (t ? w[1][n][e] : w[0][n][e]);
                if (p.rot > 0) unit[n].turn(x[n], c[n], s[n], 1.f);
                unit[n].store(y, row < p.heads[t], x[n]);
            }
        }
    }
}

// Backward: a work-group has rows of q alone, or of k, so that its waves hold one
// weight and the sums of one gradient, and the angles are read from LDS where they
// are used: 126 registers and four waves a SIMD (16,384 tokens, bf16: 121 us; both
// weights and sums, 170 registers, 137; one of each with the angles in registers, 144,
// 147).  The next token's rows are not asked for ahead: 138 us, for 136 registers.
template <int DT, int V, int E, bool NEAR>
__global__ void __launch_bounds__(kThreads) qk_backward_kernel(QkParams p, BackwardPlan plan) {
    using T = storage_t<DT>;
    using U = Unit<DT, V, NEAR>;
    __shared__ __align__(16) float turns[kWaves][2][kMaxPairs];
    __shared__ float sums[kWaves][KB_QK_MAX_DIM];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int t = (int)blockIdx.x >= plan.parts[0];
    const int part = (int)blockIdx.x - t * plan.parts[0], parts = t ? plan.parts[1] : plan.parts[0];
    const int heads = t ? p.heads[1] : p.heads[0], lanes = plan.lanes, per = 64 / lanes;
    const int all = (heads + per - 1) / per, each = min(all, plan.passes_each), chunks = (all + each - 1) / each;
    const int in_row = lane & (lanes - 1), row0 = lane / lanes;
    const float inv = 1.f / (float)p.dim;
    const TokenView vx = t ? p.x[1] : p.x[0], vdy = t ? p.dy[1] : p.dy[0], vdx = t ? p.y[1] : p.y[0];
    U unit[E];
    int pair[E];
    bool rotates[E];
    float w[E][2 * V], dw[E][2 * V];
#pragma unroll
    for (int n = 0; n < E; ++n) {
        unit[n].set(in_row + n * lanes, p.dim, p.rot);
        pair[n] = unit[n].pair;
        rotates[n] = unit[n].rotates;
        unit[n].weight(t ? p.w[1] : p.w[0], p.w_f32, w[n]);
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) dw[n][e] = 0.f;
    }
    const int64_t step = (int64_t)parts * kWaves, items = p.tokens * chunks;
    for (int64_t item = (int64_t)part * kWaves + wave; item < items; item += step) {
        const int64_t token = chunks == 1 ? item : item / chunks;
        const int from = (int)(item - token * chunks) * each, to = min(all, from + each);
        typename U::VT next[E][2], next_dy[E][2];
        const auto fetch = [&](int pass) {
            const int row = pass * per + row0;
            const T* x = (const T*)vx.p + token * vx.st + row * vx.sh;
            const T* dy = (const T*)vdy.p + token * vdy.st + row * vdy.sh;
#pragma unroll
            for (int n = 0; n < E; ++n) {
                unit[n].load(x, row < heads, next[n]);
                unit[n].load(dy, row < heads, next_dy[n]);
            }
        };
        fetch(from);
        if (p.rot > 0) token_turns(p, token, lane, turns[wave]);
        for (int pass = from; pass < to; ++pass) {
            const int row = pass * per + row0;
            float x[E][2 * V], g[E][2 * V], sum = 0.f, dot = 0.f;
#pragma unroll
            for (int n = 0; n < E; ++n)
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    x[n][e] = (float)next[n][e / V][e % V];
                    g[n][e] = (float)next_dy[n][e / V][e % V];
                }
            if (pass + 1 < to) fetch(pass + 1);
#pragma unroll
            for (int n = 0; n < E; ++n) {
                if (p.rot > 0) {
                    asm volatile("" ::: "memory");  // read where they are used: 16 registers less
                    float c[V], s[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        c[i] = turns[wave][0][pair[n] + i];
                        s[i] = turns[wave][1][pair[n] + i];
                    }
                    unit[n].turn(g[n], c, s, -1.f);
                }
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    sum = fmaf(x[n][e], x[n][e], sum);
                    dot = fmaf(g[n][e] * w[n][e], x[n][e], dot);
                }
            }
            const float r = 1.f / sqrtf(fmaf(row_sum(sum, lanes), inv, p.eps));
            const float mean = row_sum(dot, lanes) * r * inv;  // S(u z) / D
            const bool live = row < heads;
            T* dx = (T*)vdx.p + token * vdx.st + row * vdx.sh;
#pragma unroll
            for (int n = 0; n < E; ++n) {
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    const float z = x[n][e] * r;
                    if (live) dw[n][e] = fmaf(g[n][e], z, dw[n][e]);
                    x[n][e] = r * (g[n][e] * w[n][e] - z * mean);
                }
                unit[n].store(dx, live && vdx.p != nullptr, x[n]);
            }
        }
    }
    if (!p.sums) return;
    // the wave's rows, then the work-group's waves, in their order
#pragma unroll
    for (int n = 0; n < E; ++n)
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
            float v = dw[n][e];
            for (int m = lanes; m < 64; m *= 2) v += __shfl_xor(v, m);
            const int d = e < V ? unit[n].first + e : unit[n].second + e - V;
            if (row0 == 0 && unit[n].in && (e < V || unit[n].two)) sums[wave][d] = v;
        }
    __syncthreads();
    for (int d = threadIdx.x; d < p.dim; d += kThreads) {
        float v = sums[0][d];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) v += sums[k][d];
        p.part[(int64_t)blockIdx.x * p.dim + d] = v;
    }
}

// The parts of dw added up: a work-group has 16 columns of q's or of k's and 64
// threads for each, whose parts it joins in a fixed order.
constexpr int kJoinColumns = 16;
constexpr int kJoinThreads = 1024;
template <int WDT>
__global__ void __launch_bounds__(kJoinThreads) qk_join_kernel(QkParams p, BackwardPlan plan) {
    constexpr int K = kJoinThreads / kJoinColumns;
    __shared__ float s[K][kJoinColumns + 1];
    const int c = threadIdx.x % kJoinColumns, k = threadIdx.x / kJoinColumns, t = (int)blockIdx.y;
    const int d = (int)blockIdx.x * kJoinColumns + c;
    const int parts = t ? plan.parts[1] : plan.parts[0];
    const float* part = p.part + (int64_t)(t ? plan.parts[0] : 0) * p.dim;
    float v = 0.f;
    if (d < p.dim) {
#pragma unroll 8
        for (int n = k; n < parts; n += K) v += part[(int64_t)n * p.dim + d];
    }
    s[k][c] = v;
    __syncthreads();
#pragma unroll
    for (int m = K / 2; m > 0; m /= 2) {
        if (k < m) s[k][c] += s[k + m][c];
        __syncthreads();
    }
    void* dw = t ? p.dw[1] : p.dw[0];
    if (k == 0 && d < p.dim && dw != nullptr) ((storage_t<WDT>*)dw)[d] = (storage_t<WDT>)s[0][c];
}

// The launch: passes that a wave makes over its token.  All of them, so that the
// angles are worked out once, where there are tokens enough for the device: sixteen
// waves a CU (4096 tokens forward 16.5 us; asked for 64 waves, which makes a pass of
// each, 24.9; asked for 4 it is 16.7, and 1024 tokens 11.1 for 10.4).
struct Plan {
    int lanes, passes_each, chunks;
};
Plan plan_of(const QkParams& p, int v, int e) {
    const int units = p.rot / (2 * v) + (p.dim - p.rot + 2 * v - 1) / (2 * v);
    Plan plan{1, 1, 1};
    while (plan.lanes * e < units) plan.lanes *= 2;
    const int per = 64 / plan.lanes;
    const int64_t all = (p.heads[0] + (int64_t)per - 1) / per + (p.heads[1] + (int64_t)per - 1) / per;
    constexpr int64_t kWavesWanted = 256 * 16;
    int64_t each = p.tokens * all / kWavesWanted;
    each = each < 1 ? 1 : each > all ? all : each;
    if ((all + each - 1) / each > 65535) each = (all + 65534) / 65535;
    plan.passes_each = (int)each;
    plan.chunks = (int)((all + each - 1) / each);
    return plan;
}

template <int DT, int V, int E, bool NEAR>
hipError_t forward(const QkParams& p, hipStream_t stream) {
    const Plan plan = plan_of(p, V, E);
    const int64_t groups = (p.tokens + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)(groups < 8192 ? groups : 8192), (unsigned)plan.chunks);
    qk_forward_kernel<DT, V, E, NEAR><<<grid, kThreads, 0, stream>>>(p, plan.lanes, plan.passes_each);
    return hipGetLastError();
}

template <int DT, int V, int E, bool NEAR>
hipError_t backward(const QkParams& p, hipStream_t stream) {
    const Plan plan = plan_of(p, V, E);
    BackwardPlan b{plan.lanes, plan.passes_each, {0, 0}};
    // work-groups in the proportion of q's and k's rows, as many as have something to do
    const int64_t per = 64 / plan.lanes;
    const int64_t passes[2] = {(p.heads[0] + per - 1) / per, (p.heads[1] + per - 1) / per};
    for (int t = 0; t < 2; ++t) {
        if (passes[t] == 0 || p.tokens == 0) continue;
        const int64_t each = passes[t] < plan.passes_each ? passes[t] : plan.passes_each;
        const int64_t groups = (p.tokens * ((passes[t] + each - 1) / each) + kWaves - 1) / kWaves;
        const int64_t share = (kQkParts - 1) * passes[t] / (passes[0] + passes[1]) + (t == 0 || passes[0] > 0);
        b.parts[t] = (int)(groups < share ? groups : share > 0 ? share : 1);
    }
    if (b.parts[0] + b.parts[1] > 0)
        qk_backward_kernel<DT, V, E, NEAR><<<dim3((unsigned)(b.parts[0] + b.parts[1])), kThreads, 0, stream>>>(p, b);
    if (p.sums) {
        const dim3 grid((unsigned)((p.dim + kJoinColumns - 1) / kJoinColumns), 2);
        if (DT == DT_F32 || p.w_f32) qk_join_kernel<DT_F32><<<grid, kJoinThreads, 0, stream>>>(p, b);
        else qk_join_kernel<DT><<<grid, kJoinThreads, 0, stream>>>(p, b);
    }
    return hipGetLastError();
}

// The widest vectors that rotating pairs and rows are made of.
template <int DT, bool FORWARD, bool NEAR>
hipError_t widest(const QkParams& p, hipStream_t stream) {
    const auto fits = [&](int v) { return p.rot % (2 * v) == 0 && p.dim % v == 0; };
    if constexpr (DT != DT_F32) {
        if (fits(8)) return FORWARD ? forward<DT, 8, 1, NEAR>(p, stream) : backward<DT, 8, 1, NEAR>(p, stream);
    }
    if (fits(4)) return FORWARD ? forward<DT, 4, 1, NEAR>(p, stream) : backward<DT, 4, 1, NEAR>(p, stream);
    if (fits(2)) return FORWARD ? forward<DT, 2, 1, NEAR>(p, stream) : backward<DT, 2, 1, NEAR>(p, stream);
    return FORWARD ? forward<DT, 1, 2, NEAR>(p, stream) : backward<DT, 1, 2, NEAR>(p, stream);
}
template <bool FORWARD>
hipError_t launch(int dtype, const QkParams& p, hipStream_t stream) {
    if (dtype == DT_F32)
        return p.interleaved ? widest<DT_F32, FORWARD, true>(p, stream) : widest<DT_F32, FORWARD, false>(p, stream);
    if (dtype == DT_F16)
        return p.interleaved ? widest<DT_F16, FORWARD, true>(p, stream) : widest<DT_F16, FORWARD, false>(p, stream);
    return p.interleaved ? widest<DT_BF16, FORWARD, true>(p, stream) : widest<DT_BF16, FORWARD, false>(p, stream);
}

}  // namespace

hipError_t launch_qk_norm_forward(int dtype, const QkParams& p, hipStream_t stream) {
    return launch<true>(dtype, p, stream);
}

hipError_t launch_qk_norm_backward(int dtype, const QkParams& p, hipStream_t stream) {
    return launch<false>(dtype, p, stream);
}

}  // namespace kb
