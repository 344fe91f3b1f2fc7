// kb_attn.hpp -- device helpers of the attention kernels: tiles of rows in
// LDS, the fragments that the matrix instructions take from them, masks.
//
// Matrix products are 32x32 tiles, 16 along the contraction at a time.  Lane l
// (c = l % 32, g = l / 32) holds for the left operand A[m = c][k = 8g .. 8g+7],
// for the right one B[k = 8g .. 8g+7][n = c], and of the result
// C[m = 8(r/4) + 4g + r%4][n = c], r = 0..15.  A result is the right operand of
// the next product without moving: its rows r = 8j .. 8j+7 are a right operand
// whose contraction index runs 16j + {4g .. 4g+3, 8+4g .. 8+4g+3}, and the left
// operand is read from LDS in that order (col_frag).  So scores are computed
// transposed where the next product runs over keys, and straight where it runs
// over queries.
#pragma once

#include "kb_ops.hpp"

namespace kb {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Eight elements along the contraction.
template <int DT>
struct Frag {
    typedef storage_t<DT> type __attribute__((ext_vector_type(8)));
};
template <int DT>
using frag_t = typename Frag<DT>::type;

__device__ __forceinline__ f32x16 mma(frag_t<DT_F16> a, frag_t<DT_F16> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(frag_t<DT_BF16> a, frag_t<DT_BF16> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// binary32: element e of the eight is one product of contraction length 2.
__device__ __forceinline__ f32x16 mma(frag_t<DT_F32> a, frag_t<DT_F32> b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// A tile of rows in LDS: DP elements a row (the head dimension rounded up,
// zeros past it) at a pitch of 64 or 128 elements, in 16-byte chunks.  Chunk
// c of row r lies at place c ^ turn(r) of its row, and 16 bytes are left free
// after every KB, so that neither the 16 rows that a row read touches at one
// chunk nor the 4 rows x 64 bytes of a transposed read fall on the same banks,
// while few bits of c are turned: the others are constants in the reads.
template <int DT, int DP>
struct Tile {
    using T = storage_t<DT>;
    static constexpr int VEC = 16 / (int)sizeof(T);
    static constexpr int PITCH = DP <= 64 ? 64 : 128;
    static constexpr int CHUNKS = DP / VEC;
    static constexpr int PITCH_BYTES = PITCH * (int)sizeof(T);
    static constexpr int KB_ROWS = 1024 / PITCH_BYTES;          // rows of a KB
    static constexpr int KB = (1024 + 16) / (int)sizeof(T);     // elements from one KB to the next

    __device__ static __forceinline__ int turn(int row) {
        if (PITCH_BYTES == 128) return (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1);
        if (PITCH_BYTES == 256) return (row & 3) << 2;
        return (row & 1) << 3;
    }
    __device__ static __forceinline__ int at(int row, int d) {
        return row / KB_ROWS * KB + row % KB_ROWS * PITCH + (((d / VEC) ^ turn(row)) * VEC) + d % VEC;
    }
    static constexpr int size(int rows) { return rows / KB_ROWS * KB; }
};

// 16 bytes of a row from element d on, zeros past dim (unaligned rows are fine).
template <typename T>
__device__ __forceinline__ u32v4 load_chunk(const T* row, int d, int dim) {
    constexpr int N = Vec16<T>::N;
    typename Vec16<T>::type v;
    if (d + N <= dim) return __builtin_bit_cast(u32v4, *(const typename Vec16<T>::type*)(row + d));
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = d + e < dim ? row[d + e] : (T)0.f;
    return __builtin_bit_cast(u32v4, v);
}

// Rows [r0, r0 + ROWS) of a view into a tile by NT threads; rows from n on are
// zeros and not read.
template <int DT, int DP, int ROWS, int NT>
__device__ __forceinline__ void stage(storage_t<DT>* tile, const storage_t<DT>* base, int64_t stride, int r0, int n,
                                      int dim) {
    using L = Tile<DT, DP>;
#pragma unroll
    for (int k = 0; k < (ROWS * L::CHUNKS + NT - 1) / NT; ++k) {
        const int idx = k * NT + (int)threadIdx.x;
        if (ROWS * L::CHUNKS % NT != 0 && idx >= ROWS * L::CHUNKS) break;
        const int row = idx / L::CHUNKS, d = idx % L::CHUNKS * L::VEC;
        u32v4 v = {0, 0, 0, 0};
        if (r0 + row < n) v = load_chunk(base + (int64_t)(r0 + row) * stride, d, dim);
        *(u32v4*)(tile + L::at(row, d)) = v;
    }
}

// Memory straight to LDS, BYTES a lane, in the order of the lanes: from the
// address, the same in all lanes, plus two offsets, one a lane's.  As buffer loads: while
// a global or flat one is under way, the compiler waits for all of a wave's LDS
// reads wherever it needs the oldest (backward of 4 x 32 heads x 2047 f16: 612 us, 638
// with global loads).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t background(const void* address) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(address), 0, 0x7FFFFFFF, 0x00020000);
}
template <int BYTES>
__device__ __forceinline__ void send(__amdgpu_buffer_rsrc_t from, uint32_t lane_offset, int offset, void* to) {
    static_assert(BYTES == 4 || BYTES == 16, "a word or a chunk");
    const auto lds = (__attribute__((address_space(3))) void*)to;
    if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds, 16, (int)lane_offset, offset, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds, 4, (int)lane_offset, offset, 0, 0);
}

// A tile filled in the background: each thread's 16-byte chunks go from memory
// straight to LDS, with no register in between, and have arrived once the
// thread has waited (tile_wait) and the work-group has met.  LDS takes a wave's
// chunks in the order of its lanes, so the tile's order (Tile::at) is made by
// what each lane reads.  For rows of whole chunks only (AttnParams::whole);
// stage() serves the others.
template <int DT, int DP, int ROWS, int NT>
struct Filler {
    using T = storage_t<DT>;
    using L = Tile<DT, DP>;
    static constexpr int SLOTS = L::PITCH / L::VEC;  // chunk places of a row
    static constexpr int STEP = NT / SLOTS;          // rows that the work-group fills at once
    static constexpr int STEPS = ROWS / STEP;
    static_assert(NT % SLOTS == 0 && ROWS % STEP == 0, "a tile is filled in whole steps");
    static_assert(STEP % 8 == 0, "turn() is the same in every step");
    static_assert(ROWS <= kAttnReach, "a tile's last row is within reach of its first");
    int row0;
    uint32_t offset;  // bytes from the step's first row to the lane's chunk
    bool in;          // the chunk lies within dim

    __device__ __forceinline__ Filler(int64_t stride, int dim) {
        row0 = (int)threadIdx.x / SLOTS;
        const int d = ((int)threadIdx.x % SLOTS ^ L::turn(row0)) * L::VEC;
        in = d < dim;
        offset = ((uint32_t)row0 * (uint32_t)stride + (uint32_t)d) * (uint32_t)sizeof(T);
    }

    // Rows [r0, r0 + ROWS) of base; those from n on are zeros.
    __device__ __forceinline__ void fill(T* tile, const T* base, int64_t stride, int r0, int n, int dim) const {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        T* to = tile + wave * L::KB;
        const auto from = background(base + (int64_t)r0 * stride);
        const int step = STEP * (int)stride * (int)sizeof(T);  // (ROWS of them are within 2^31 bytes)
        if (r0 + ROWS <= n && dim == L::PITCH) {  // the common case, without a test for each chunk
#pragma unroll
            for (int k = 0; k < STEPS; ++k) send<16>(from, offset, k * step, to + k * (STEP / L::KB_ROWS * L::KB));
        } else {
#pragma unroll 1
            for (int k = 0; k < STEPS; ++k) {
                if (in && r0 + k * STEP + row0 < n) {
                    send<16>(from, offset, k * step, to);
                } else {
                    const u32v4 zero = {0, 0, 0, 0};
                    *(u32v4*)(to + ((int)threadIdx.x & 63) * L::VEC) = zero;
                }
                to += STEP / L::KB_ROWS * L::KB;
            }
        }
    }
};

// Until the chunks that this thread has sent for have arrived.
__device__ __forceinline__ void tile_wait() { __builtin_amdgcn_s_waitcnt(0x0F70); }  // vmcnt 0

// Where a lane reads in a tile.  Its byte addresses are a few values that hold
// for the whole kernel, one for each setting of the turned bits, plus constants;
// they are kept from the compiler's sight, which would otherwise hold one
// register for each read.
template <int DT, int DP>
struct Reader {
    using T = storage_t<DT>;
    using L = Tile<DT, DP>;
    uint32_t row[4];  // row c = lane % 32, turned bits 0..3
    uint32_t col[4];
    int lane;

    __device__ __forceinline__ explicit Reader(int lane_) : lane(lane_) {
        const int c = lane & 31, g = lane >> 5;
        const uint32_t row_at = (c / L::KB_ROWS * L::KB + c % L::KB_ROWS * L::PITCH) * sizeof(T);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (DT == DT_F32) {
                // chunks 4k + 2g and the next
                if (L::PITCH_BYTES == 256) row[v] = row_at + (((v ^ (c & 3)) << 2) + 2 * g) * 16;
                else row[v] = row_at + (((v & 1) << 3 ^ L::turn(c)) + 2 * g) * 16;
                // single elements of 32 columns, rows 4g + ..
                const int q = (lane >> 4) & 1;
                if (L::PITCH_BYTES == 256) col[v] = g * L::KB * 4 + ((q ^ (v & 1)) << 2) * 16 + (lane & 15) * 4;
                else col[v] = 2 * g * L::KB * 4 + c * 4;
            } else {
                const int r = (lane & 15) >> 2, q = (lane >> 4) & 1, in = (lane & 3) >> 1;
                if (L::PITCH_BYTES == 256) {
                    row[v] = row_at + (((v ^ (c & 3)) << 2) + g) * 16;
                    col[v] = g * L::KB * 2 + r * L::PITCH * 2 + (((v ^ r) << 2) + 2 * q + in) * 16 + (lane & 1) * 8;
                } else {
                    row[v] = row_at + ((v << 1 ^ L::turn(c)) + g) * 16;
                    col[v] = (4 * g + r) * L::PITCH * 2 + ((((2 * v + q) << 1) ^ L::turn(4 * g + r)) + in) * 16 + (lane & 1) * 8;
                }
            }
            asm volatile("" : "+v"(row[v]), "+v"(col[v]));
        }
    }

    // Elements d = 16k + 8g .. +7 of row row0 + c (row0 a multiple of 32).
    __device__ __forceinline__ frag_t<DT> row_frag(const T* tile, int row0, int k) const {
        const char* base = (const char*)tile + row0 / L::KB_ROWS * L::KB * (int)sizeof(T);
        if constexpr (DT == DT_F32) {
            const char* at = L::PITCH_BYTES == 256 ? base + row[k & 3]
                                                   : base + row[(k >> 1) & 1] + ((k >> 2) * 16 + (k & 1) * 4) * 16;
            const f32x4 a = *(const f32x4*)at, b = *(const f32x4*)(at + 16);
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            const char* at = L::PITCH_BYTES == 256 ? base + row[k >> 1] + (k & 1) * 32 : base + row[k & 3];
            return *(const frag_t<DT>*)at;
        }
    }

    // Column d = 32 db + c of rows row0 + {4g .. 4g+3, 8+4g .. 8+4g+3} (row0 a
    // multiple of 16).  In 16 bits each four come from one transposed read: of 16
    // lanes, lane i gives the address of 4 elements of row i/4, columns
    // 4(i%4) .., and receives column i of the four rows.
    __device__ __forceinline__ frag_t<DT> col_frag(const T* tile, int row0, int db) const {
        const char* base = (const char*)tile + row0 / L::KB_ROWS * L::KB * (int)sizeof(T);
        if constexpr (DT == DT_F32) {
            frag_t<DT> f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = 8 * (e >> 2) + (e & 3);  // + 4g
                const char* at = base + r / L::KB_ROWS * L::KB * 4 + r % L::KB_ROWS * L::PITCH * 4;
                f[e] = *(const float*)(L::PITCH_BYTES == 256
                                           ? at + col[e & 1] + ((db ^ ((e >> 1) & 1)) * 8) * 16
                                           : at + col[0] + (((db >> 1) * 16 + ((db ^ e) & 1) * 8)) * 16);
            }
            return f;
        } else {
            using lds_ptr = __attribute__((address_space(3))) s16x4*;
            const char* at = base + col[db];
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(s16x4*)at);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(s16x4*)(at + 8 / L::KB_ROWS * L::KB * 2));
            return __builtin_bit_cast(frag_t<DT>, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Eight elements of a row in memory, d = 16c + 8g .., zeros past dim or if !in.
// WHOLE: a chunk lies within dim or past it.
template <int DT, bool WHOLE>
__device__ __forceinline__ frag_t<DT> load_frag(const storage_t<DT>* row, int c, int g, int dim, bool in) {
    using T = storage_t<DT>;
    constexpr int N = Vec16<T>::N;
    frag_t<DT> f;
#pragma unroll
    for (int k = 0; k < 8 / N; ++k) {
        const int d = 16 * c + 8 * g + k * N;
        u32v4 v = {0, 0, 0, 0};
        if (WHOLE) {
            if (in && d < dim) v = *(const u32v4*)(row + d);
        } else if (in) {
            v = load_chunk(row, d, dim);
        }
        const typename Vec16<T>::type t = __builtin_bit_cast(typename Vec16<T>::type, v);
#pragma unroll
        for (int e = 0; e < N; ++e) f[k * N + e] = t[e];
    }
    return f;
}

// Rows 8j .. 8j+7 of a result as a right operand in the storage type.
template <int DT>
__device__ __forceinline__ frag_t<DT> narrow(const f32x16& s, int j) {
    frag_t<DT> f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (storage_t<DT>)s[8 * j + e];
    return f;
}

// A product takes every row of a tile to every column, at 0 where the column
// does not see the row.  That leaves nothing behind unless the row holds a NaN or
// an infinity, which times 0 is NaN.  So a work-group whose sums end up with
// such a value, and some of whose tiles were seen in part, computes them once
// more (CAREFUL), with the rows that a column does not see cleared for it.

// acc += A B over 16 rows of a tile, column n of B seeing rows [lo, hi) of it
// (lo, hi: the lane's column's): a product for each column.
template <int DT>
__device__ void mma_seen(f32x16& acc, frag_t<DT> a, frag_t<DT> b, int row0, int lo, int hi, int lane) {
    const int g = lane >> 5;
#pragma unroll 1
    for (int n = 0; n < 32; ++n) {
        const int from = __builtin_amdgcn_readlane(lo, n), to = __builtin_amdgcn_readlane(hi, n);
        frag_t<DT> cut = a;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int row = row0 + 8 * (e >> 2) + 4 * g + (e & 3);
            if (row < from || row >= to) cut[e] = (storage_t<DT>)0.f;
        }
        f32x16 t = {};
        t = mma(cut, b, t);
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = (lane & 31) == n ? acc[r] + t[r] : acc[r];
    }
}

// acc[db] += (rows [row0, row0 + 32) of the tile)^T b, b in two halves; SEEN: by
// mma_seen.
template <int DT, int DP, bool SEEN>
__device__ __forceinline__ void mma_rows(f32x16 (&acc)[DP / 32], const storage_t<DT>* tile, const Reader<DT, DP>& rd,
                                         int row0, const frag_t<DT> (&b)[2], int lo, int hi) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
            const frag_t<DT> a = rd.col_frag(tile, row0 + 16 * j, db);
            if (SEEN) mma_seen<DT>(acc[db], a, b[j], row0 + 16 * j, lo, hi, rd.lane);
            else acc[db] = mma(a, b[j], acc[db]);
        }
}

template <int N>
__device__ __forceinline__ bool non_finite(const f32x16 (&acc)[N]) {
    float z = 0.f;  // x 0 is 0, or NaN
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) z = fmaf(acc[k][r], 0.f, z);
    return z != 0.f;
}

// Elements d = 32 db + 8 q4 + 4 g .. +3 of a row of results.
template <int DT>
__device__ __forceinline__ void store_quad(storage_t<DT>* row, int d, int dim, float a, float b, float c, float e) {
    using T = storage_t<DT>;
    typedef T quad __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const float v[4] = {a, b, c, e};
    if (d + 4 <= dim) {
        quad t;
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = (T)v[k];
        *(quad*)(row + d) = t;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (d + k < dim) row[d + k] = (T)v[k];
    }
}

// A column of transposed results (the lane's) as a row in memory, times f;
// zeros if !live (whatever the accumulators hold).
template <int DT, int DP>
__device__ __forceinline__ void store_column(storage_t<DT>* row, const f32x16 (&acc)[DP / 32], float f, bool live,
                                             int dim, int g) {
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            store_quad<DT>(row, 32 * db + 2 * r + 4 * g, dim, live ? acc[db][r] * f : 0.f,
                           live ? acc[db][r + 1] * f : 0.f, live ? acc[db][r + 2] * f : 0.f,
                           live ? acc[db][r + 3] * f : 0.f);
}

// The same as one part of a row's sums: binary32, at multiples of 4.
template <int DP>
__device__ __forceinline__ void store_part(float* row, const f32x16 (&acc)[DP / 32], int dim, int g) {
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            if (32 * db + 2 * r + 4 * g < dim)
                *(f32x4*)(row + 32 * db + 2 * r + 4 * g) = f32x4{acc[db][r], acc[db][r + 1], acc[db][r + 2], acc[db][r + 3]};
}

// Lengths of sequence b.
__device__ __forceinline__ int seq_len(const int32_t* lens, int b, int full) {
    return lens ? min(max(lens[b], 0), full) : full;
}

// Query i sees keys [0, key_limit).
__device__ __forceinline__ int key_limit(int i, int qlen, int klen, int causal) {
    return causal ? min(klen, max(0, i + 1 + klen - qlen)) : klen;
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// Work-group `id` of `blocks` blocks for each (batch, key head) pair, pair by
// pair at the same block: with a multiple of 8 pairs (the usual case) a head's
// work-groups land on one XCD, whose L2 then holds its keys.  Block 0 is to be
// the longest.  A launch of two work-groups a CU or less has no later ones to
// even out a causal mask's long and short blocks: there the second work-group
// of a CU is the shorter, the longer the first one is.
struct HeadBlock {
    int b, h, block;
};
__device__ __forceinline__ HeadBlock head_block(int id, int kv_heads, int pairs, int blocks) {
    constexpr int kCus = 256;
    const int total = pairs * blocks;
    if (total <= 2 * kCus && id >= kCus) id = total - 1 - (id - kCus);
    const int pair = id % pairs;
    return {pair / kv_heads, pair % kv_heads, id / pairs};
}

}  // namespace kb
