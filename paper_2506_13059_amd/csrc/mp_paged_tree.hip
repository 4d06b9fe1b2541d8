// Trees of drafted tokens over a paged cache: their ancestors and positions, and the rows of the accepted path moved together, for gfx950.
//
// Tokens of a tree are in an order in which each follows its parent.  A token's mask marks itself and its ancestors, and its position is that of its sequence's older keys and
// the length of its path.  Both kernels are a few trips to memory: 128 trees of up to 250 tokens 5.0 us, the paths of 192 of up to 60, 8 KV heads, 6.1.
#include "mp_device.h"
#include "mp_launch.h"
#include "mp_paged.h"

namespace mp {

namespace {

struct NewTokens {
    int q0, n, base;          // first row, tokens, keys that are older (negative: more tokens than keys)
};
__device__ __forceinline__ NewTokens new_tokens(const PagedKv& c, int n_tokens, int b, int most)
{
    const int s0 = c.q_start[b], s1 = c.q_start[b + 1];
    NewTokens t;
    t.q0 = min(max(s0, 0), n_tokens);
    t.n = min(min(max(s1, t.q0), n_tokens) - t.q0, most);
    t.base = c.kv_len[b] - (s1 - s0);
    return t;
}

// One workgroup a sequence, one thread a token.  Masks double the length of path that they hold from round to round, until every path has ended: as many rounds as the
// depth has binary digits.  every: rows without a result, a sequence's own and, for the first and the last one, those of no sequence, get a mask of zeros and position -1.
template <int kWords>
__global__ __launch_bounds__(64 * kWords) void paged_tree_plan_kernel(PagedKv c, const int32_t* parents, int n_tokens, int words, bool every,
                                                                      unsigned long long* mask, int32_t* positions)
{
    constexpr int kTokens = 64 * kWords;
    __shared__ unsigned long long masks[kTokens * kWords];
    __shared__ int16_t up[kTokens];
    const int b = blockIdx.x, i = threadIdx.x;
    NewTokens t = b < c.n_seqs ? new_tokens(c, n_tokens, b, 0x7fffffff) : NewTokens{};
    const int rest = b < c.n_seqs - 1 ? t.q0 + t.n : n_tokens;      // behind the last row that is the workgroup's to look after
    t.n = min(t.n, 64 * words);
    int ancestor = i < t.n ? parent_of(parents[t.q0 + i], i) : -1;
    unsigned long long own[kWords];
#pragma unroll
    for (int w = 0; w < kWords; ++w) own[w] = w == i >> 6 ? 1ull << (i & 63) : 0ull;
    while (__syncthreads_or(ancestor >= 0)) {
#pragma unroll
        for (int w = 0; w < kWords; ++w) masks[i * kWords + w] = own[w];
        up[i] = (int16_t)ancestor;
        __syncthreads();
        if (ancestor >= 0) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) own[w] |= masks[ancestor * kWords + w];
            ancestor = up[ancestor];
        }
    }
    if (i < t.n) {
        int depth = 0;
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            depth += __popcll(own[w]);
            if (w < words) mask[(long long)(t.q0 + i) * words + w] = own[w];
        }
        positions[t.q0 + i] = t.base + depth - 1;
    }
    if (!every) return;
    auto none = [&](long long row) {
        for (int w = 0; w < words; ++w) mask[row * words + w] = 0;
        positions[row] = -1;
    };
    for (long long row = t.q0 + t.n + i; row < rest; row += kTokens) none(row);
    if (b == 0)
        for (long long row = i; row < t.q0; row += kTokens) none(row);
}

constexpr int kWaves = 4, kDeep = 4, kMostWords = 16;

// One wave: keys or values of a head of a sequence.  Row i of the path goes to place i behind the older keys, which is never behind its own: rows are moved from the first
// on, some at a time, all of which are loaded before any is stored.
__global__ __launch_bounds__(64 * kWaves) void paged_tree_keep_kernel(PagedKv c, const unsigned long long* mask, int words, const int32_t* leaf, int n_tokens,
                                                                      int32_t* keep)
{
    __shared__ uint16_t paths[kWaves][64 * kMostWords];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const long long unit = (long long)blockIdx.x * kWaves + wave;
    const int b = (int)(unit / (2 * c.n_kv)), which = (int)(unit - (long long)b * 2 * c.n_kv), h = which >> 1;
    if (b >= c.n_seqs) return;
    const NewTokens t = new_tokens(c, n_tokens, b, 64 * words);
    const int last = leaf[b];
    unsigned long long m = 0;
    if (lane < words && last >= 0 && last < t.n) {
        const int in = t.n - 64 * lane;                     // tokens of this word
        m = mask[(long long)(t.q0 + last) * words + lane];
        m &= in >= 64 ? ~0ull : in > 0 ? (1ull << in) - 1ull : 0ull;
    }
    const uint32_t upto = wave_incl_scan_u32((uint32_t)__popcll(m));
    const int n = __builtin_amdgcn_readlane((int)upto, 63);
    uint16_t* const path = paths[wave];
    for (int at = (int)upto - __popcll(m); m; m &= m - 1) path[at++] = (uint16_t)(64 * lane + __builtin_ctzll(m));
    wave_lds_sync();
    if (which == 0 && lane == 0) keep[b] = max(t.base + n, 0);
    uint16_t* const pages = which & 1 ? c.V : c.K;
    const int32_t* const entries = c.table + (long long)b * c.table_stride;
    for (int r0 = 0; r0 < n; r0 += 4 * kDeep) {
        uint4 x[kDeep];
        long long to[kDeep];                                // (negative: the row stays where it is, or has no place)
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int r = r0 + 4 * i + (lane >> 4), from = r < n ? path[r] : r;
            const int page0 = page_of(entries, c.table_stride, c.n_pages, c.page_shift, t.base + from);
            const int page1 = page_of(entries, c.table_stride, c.n_pages, c.page_shift, t.base + r);
            to[i] = from == r || page0 < 0 || page1 < 0 ? -1 : row_of(page1, h, c.n_kv, c.page_shift, t.base + r) * kHeadDim;
            x[i] = make_uint4(0, 0, 0, 0);
            if (to[i] >= 0) x[i] = reinterpret_cast<const uint4*>(pages + row_of(page0, h, c.n_kv, c.page_shift, t.base + from) * kHeadDim)[lane & 15];
        }
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
            if (to[i] >= 0) reinterpret_cast<uint4*>(pages + to[i])[lane & 15] = x[i];
    }
}

}  // namespace

hipError_t launch_paged_tree_plan(const PagedKv& c, const int32_t* parents, int n_tokens, int words, bool every, uint64_t* mask, int32_t* positions, hipStream_t s)
{
    if (n_tokens <= 0 || (c.n_seqs <= 0 && !every)) return hipSuccess;
    int size = 1;
    while (size < words) size *= 2;
    const auto on = size == 1 ? Launch<paged_tree_plan_kernel<1>>::on : size == 2 ? Launch<paged_tree_plan_kernel<2>>::on : size == 4 ? Launch<paged_tree_plan_kernel<4>>::on
                  : size == 8 ? Launch<paged_tree_plan_kernel<8>>::on : Launch<paged_tree_plan_kernel<16>>::on;
    return on(dim3((unsigned)(c.n_seqs > 0 ? c.n_seqs : 1)), dim3(64 * size), s, c, parents, n_tokens, words, every, (unsigned long long*)mask, positions);
}

hipError_t launch_paged_tree_keep(const PagedKv& c, const uint64_t* mask, int words, const int32_t* leaf, int n_tokens, int32_t* keep, hipStream_t s)
{
    if (c.n_seqs <= 0) return hipSuccess;
    const long long blocks = (2ll * c.n_kv * c.n_seqs + kWaves - 1) / kWaves;
    return Launch<paged_tree_keep_kernel>::on(dim3((unsigned)blocks), dim3(64 * kWaves), s, c, (const unsigned long long*)mask, words, leaf, n_tokens, keep);
}

}  // namespace mp
