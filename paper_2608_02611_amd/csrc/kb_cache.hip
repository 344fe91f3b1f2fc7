// kb_cache.hip -- the new tokens' rows of k and v into the pages of their
// sequences: token t of sequence b, whose tokens end before `end`, has place
// lens[b] - end + t, in page table[b][place / page] at place % page.
//
// It moves bytes, each read and written once.  A wave has one token: its rows are
// on their way while it looks for the token's page.  Latency is what that is bound by:
// up to 64 sequences' starts and lengths are read at once, one a lane, and then the
// table (8 prompts of up to 8191 tokens, 8 heads of 128, f16: 44 us, 4.9 TB/s, where a
// copy moves 4.8; with a search of the starts, the length and the table one after the
// other 49.5, which larger batches still have: 100 prompts of up to 1000, 59 us, 4.6
// TB/s).  64 single tokens, a call's own time, 8 us, of which the kernel has 3.5.
#include "kb_paged.hpp"

namespace kb {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Elements are moved as bits, V of them at once (V divides the rows).  AHEAD: vectors
// of a lane that are on their way during the search.
template <typename B, int V, int AHEAD>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(PagedParams p) {
    typedef B VT __attribute__((ext_vector_type(V), aligned(sizeof(B))));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int chunks = p.dim / V, per_row = p.kv_heads * chunks, all = 2 * per_row;
    const int64_t step = (int64_t)gridDim.x * kWaves;
    for (int64_t token = (int64_t)blockIdx.x * kWaves + wave; token < p.tokens; token += step) {
        const auto split = [&](int i, int* t, int* head, int* d) {
            *t = i >= per_row;
            const int j = i - *t * per_row;
            *head = j / chunks;
            *d = (j - *head * chunks) * V;
        };
        const auto fetch = [&](int i) {
            int t, head, d;
            split(i, &t, &head, &d);
            const TokenView& x = t ? p.rows[1] : p.rows[0];
            return *(const VT*)((const B*)x.p + token * x.st + head * x.sh + d);
        };
        VT v[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n)
            if (n * 64 + lane < all) v[n] = fetch(n * 64 + lane);

        // its sequence, and the token after that one's last
        int b = (int)token, len;
        int64_t end = token + 1;
        if (p.starts != nullptr && p.batch <= 64) {  // a sequence a lane: all that is asked of them on its way at once
            int first = 0, last = 0, keys = 0;
            if (lane < p.batch) {
                first = p.starts[lane];
                last = p.starts[lane + 1];
                keys = paged_len(p, lane);
            }
            b = __popcll(__ballot(lane < p.batch && last <= token));
            if (b >= p.batch || token < __builtin_amdgcn_readlane(first, b)) continue;  // no sequence's
            end = min(__builtin_amdgcn_readlane(last, b), p.tokens);
            len = __builtin_amdgcn_readlane(keys, b);
        } else {
            if (p.starts != nullptr) {
                b = count_up_to(p.batch, token, lane, [&](int i) { return (int64_t)p.starts[i + 1]; });
                if (b >= p.batch || token < p.starts[b]) continue;
                end = min(p.starts[b + 1], p.tokens);
            }
            len = paged_len(p, b);
        }
        const int64_t place = (int64_t)len - end + token;
        if (place < 0 || place >= len) continue;
        const int at = page_of(p, (int)place), in_page = (int)place - at * p.page;
        const int page = p.table[b * p.table_stride + at];
        if (page < 0 || page >= p.pages) continue;  // no page

        const auto put = [&](int i, VT x) {
            int t, head, d;
            split(i, &t, &head, &d);
            const HeadView& c = t ? p.cache[1] : p.cache[0];
            *(VT*)((B*)c.p + page * c.sb + head * c.sh + in_page * c.sl + d) = x;
        };
#pragma unroll
        for (int n = 0; n < AHEAD; ++n)
            if (n * 64 + lane < all) put(n * 64 + lane, v[n]);
        for (int i = AHEAD * 64 + lane; i < all; i += 64) put(i, fetch(i));
    }
}

template <typename B, int V>
hipError_t write(const PagedParams& p, hipStream_t stream) {
    const int64_t groups = ((int64_t)p.tokens + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)(groups < 16384 ? groups : 16384));
    // tokens of a vector a lane: 52 registers instead of 98 (one key head, 8 prompts of up
    // to 8191 tokens: 10.5 us, 17 with four vectors' registers)
    if (2 * (int64_t)p.kv_heads * (p.dim / V) <= 64) cache_write_kernel<B, V, 1><<<grid, kThreads, 0, stream>>>(p);
    else cache_write_kernel<B, V, 4><<<grid, kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(int dtype, const PagedParams& p, hipStream_t stream) {
    if (dtype == DT_F32) {
        if (p.dim % 4 == 0) return write<uint32_t, 4>(p, stream);
        if (p.dim % 2 == 0) return write<uint32_t, 2>(p, stream);
        return write<uint32_t, 1>(p, stream);
    }
    if (p.dim % 8 == 0) return write<uint16_t, 8>(p, stream);
    if (p.dim % 4 == 0) return write<uint16_t, 4>(p, stream);
    if (p.dim % 2 == 0) return write<uint16_t, 2>(p, stream);
    return write<uint16_t, 1>(p, stream);
}

}  // namespace kb
