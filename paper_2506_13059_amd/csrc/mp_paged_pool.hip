// Page tables, and the maps of a step's tokens, made on the device from what sequences keep and what is to come, for gfx950.
//
// Of sequence b with `have` keys, of which stay = min(keep, have) are kept, entries [ceil(stay / P), ceil(have / P)) of its table are given back: their pages go on the
// stack of free ones, sequence after sequence, entry after entry.  Then each sequence takes ceil((stay + new) / P) - ceil(stay / P) pages from the top of the stack, sequence after
// sequence; the first that finds too few gets no tokens, and neither does any behind it that needs pages.
//
// One workgroup, for everything hangs on two running sums over the sequences: bound by its trips to memory one behind the other.  The maps of many tokens are a launch of their own.  64 sequences of up to
// eight tokens 4.8 us; 512 that give 3183 pages back, most of them 64 sequences', and take as many 8.9 to 9.2, and 3.5 for the maps of their 50 thousand rows.  A call, with eight tokens each of as many
// sequences and no maps: 1024 5.7 us; past that, in turns of 1024 without what LDS hands on, 1025 7.4, 2048 8.0, 4096 14.0.
#include "mp_device.h"
#include "mp_launch.h"
#include "mp_paged.h"

namespace mp {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kDeep = 8;

struct Shared {
    uint32_t upto[kThreads];            // of a flat list of sequences' entries: where each one's end
    int32_t left[kThreads];             // first entry
    uint32_t sums[2][kWaves];
    uint32_t counts[2][kDeep * kWaves];
    unsigned long long tokens[kWaves];
    uint32_t taken;
};

// Inclusive sum over the workgroup; *all: the sum of everything.  `which`: the two buffers in turn.
__device__ __forceinline__ uint32_t block_scan(Shared& sm, int which, uint32_t v, uint32_t* all)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t incl = wave_incl_scan_u32(v);
    if (lane == 63) sm.sums[which][wave] = incl;
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t s = sm.sums[which][w];
        before += w < wave ? s : 0u;
        sum += s;
    }
    *all = sum;
    return before + incl;
}

// The first of the sequences whose entries end behind place x of the list.
__device__ __forceinline__ int owner_of(const Shared& sm, uint32_t x)
{
    int k = 0;
#pragma unroll
    for (int step = kThreads / 2; step; step >>= 1)
        if (sm.upto[k + step - 1] <= x) k += step;
    return k;
}

struct Sequence {
    int have, stay, left, had;           // keys, keys that stay, and their pages
};
__device__ __forceinline__ Sequence sequence_at(const PagePool& p, const int32_t* keep, int b)
{
    Sequence s{0, 0, 0, 0};
    if (b < p.n_seqs) {
        const int room = p.table_stride << p.page_shift, len = p.kv_len[b];
        s.have = min(max(len, 0), room);
        s.stay = min(max(keep ? keep[b] : len, 0), s.have);
        const uint32_t up = (1u << p.page_shift) - 1u;
        s.left = (int)(((uint32_t)s.stay + up) >> p.page_shift);
        s.had = (int)(((uint32_t)s.have + up) >> p.page_shift);
    }
    return s;
}

// Rows r0 + lane of a step: their sequence, position and place in the cache.
__device__ __forceinline__ void map_rows(const PagePool& p, const StepRows& rows, int r0)
{
    const int lane = threadIdx.x & 63, r = r0 + lane;
    const int first = sequence_of(p.q_start, p.n_seqs, r0);
    int b = first >= 0 ? first : p.n_seqs;
    for (int s = first + 1; first >= 0;  s += 64) {
        const int start = s + lane <= p.n_seqs ? p.q_start[s + lane] : 0x7fffffff;
        int k = 0;                                          // how many of these starts lie at or before r
#pragma unroll
        for (int step = 32; step; step >>= 1)
            if (__shfl(start, k + step - 1, 64) <= r) k += step;
        if (__shfl(start, k, 64) <= r) ++k;                 // (63 of them: perhaps all)
        if (k > 0) b = s - 1 + k;
        if (!__any(k == 64)) break;
    }
    if (r >= rows.n_rows) return;
    int position = -1;
    long long slot = -1;
    if (b < p.n_seqs) {
        position = p.kv_len[b] - (p.q_start[b + 1] - r);
        if (rows.slots) {
            const int page = page_of(p.table + (long long)b * p.table_stride, p.table_stride, p.n_pages, p.page_shift, position);
            if (page >= 0) slot = ((long long)page << p.page_shift) + (position & ((1 << p.page_shift) - 1));
        }
    }
    if (rows.sequence) rows.sequence[r] = b < p.n_seqs ? b : -1;
    if (rows.positions) rows.positions[r] = position;
    if (rows.slots) rows.slots[r] = slot;
}

// Any number of sequences, 1024 after 1024.
__global__ __launch_bounds__(kThreads) void paged_reserve_kernel(PagePool p, const int32_t* n_new, const int32_t* keep, int32_t* granted, StepRows rows)
{
    __shared__ Shared sm;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int32_t* const stack = p.free_pages;
    uint32_t top = (uint32_t)min(max(p.n_free[0], 0), p.n_pages);
    // Pages that go back.
    int turn = 0;
    for (int s0 = 0; s0 < p.n_seqs; s0 += kThreads) {
        const Sequence seq = sequence_at(p, keep, s0 + tid);
        uint32_t all;
        const uint32_t incl = block_scan(sm, 0, (uint32_t)(seq.had - seq.left), &all);
        sm.upto[tid] = incl;
        sm.left[tid] = seq.left;
        __syncthreads();
        for (uint32_t x0 = 0; x0 < all; x0 += kDeep * kThreads, turn ^= 1) {
            int32_t page[kDeep];
            unsigned long long in[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const uint32_t x = x0 + (uint32_t)(i * kThreads + tid);
                page[i] = -1;
                if (x < all) {
                    const int k = owner_of(sm, x);
                    int32_t* const entry = p.table + (long long)(s0 + k) * p.table_stride + sm.left[k] + (int)(x - (k ? sm.upto[k - 1] : 0u));
                    page[i] = *entry;
                    *entry = -1;
                }
            }
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                in[i] = __ballot((uint32_t)page[i] < (uint32_t)p.n_pages);
                if (lane == 0) sm.counts[turn][i * kWaves + wave] = (uint32_t)__popcll(in[i]);
            }
            __syncthreads();
            const uint32_t c0 = sm.counts[turn][2 * lane], c1 = sm.counts[turn][2 * lane + 1];
            const uint32_t upto = wave_incl_scan_u32(c0 + c1);
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int at = i * kWaves + wave;
                uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)(upto - c0 - c1), at >> 1);
                if (at & 1) before += (uint32_t)__builtin_amdgcn_readlane((int)c0, at >> 1);
                const uint32_t to = top + before + (uint32_t)__popcll(in[i] & ((1ull << lane) - 1ull));
                if ((in[i] >> lane & 1) && to < (uint32_t)p.n_pages) stack[to] = page[i];      // (more than there are: a page that came twice)
            }
            top += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
        __syncthreads();
    }
    top = min(top, (uint32_t)p.n_pages);
    // Pages for the tokens to come.
    uint32_t needed = 0, taken = 0;
    unsigned long long tokens = 0;
    if (tid == 0) p.q_start[0] = 0;
    for (int s0 = 0; s0 < p.n_seqs; s0 += kThreads) {
        const int b = s0 + tid;
        const Sequence seq = sequence_at(p, keep, b);
        const int room = p.table_stride << p.page_shift;
        int come = b < p.n_seqs ? max(n_new[b], 0) : 0;
        if (come > room - seq.stay) come = 0;
        const uint32_t need = ((uint32_t)(seq.stay + come) + ((1u << p.page_shift) - 1u)) >> p.page_shift;
        const uint32_t more = come > 0 ? need - (uint32_t)seq.left : 0u;
        uint32_t all;
        const uint32_t incl = block_scan(sm, 1, more, &all);
        const bool ok = more == 0 || needed + incl <= top;
        if (!ok) come = 0;
        sm.upto[tid] = incl;
        sm.left[tid] = seq.left;
        if (tid == 0) sm.taken = 0;
        // tokens up to each one's
        unsigned long long upto = (unsigned long long)come;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const unsigned long long v = __shfl_up(upto, step, 64);
            if (lane >= step) upto += v;
        }
        if (lane == 63) sm.tokens[wave] = upto;
        __syncthreads();
        if (ok && more > 0) atomicMax(&sm.taken, incl);
        unsigned long long sum = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) upto += sm.tokens[w];
            sum += sm.tokens[w];
        }
        if (b < p.n_seqs) {
            p.kv_len[b] = seq.stay + come;
            p.q_start[b + 1] = (int32_t)min(tokens + upto, 0x7fffffffull);
            if (granted) granted[b] = come;
        }
        tokens += sum;
        __syncthreads();
        const uint32_t here = sm.taken;
        for (uint32_t x = tid; x < here; x += kThreads) {
            const int k = owner_of(sm, x);
            int32_t* const from = stack + (top - 1u - (taken + x));
            p.table[(long long)(s0 + k) * p.table_stride + sm.left[k] + (int)(x - (k ? sm.upto[k - 1] : 0u))] = *from;
            *from = -1;
        }
        taken += here;
        needed += all;
        __syncthreads();
    }
    if (tid == 0) p.n_free[0] = (int32_t)(top - taken);
    if (rows.n_rows > 0) {
        __syncthreads();
        for (int r0 = wave * 64; r0 < rows.n_rows; r0 += kThreads) map_rows(p, rows, r0);
    }
}

// Up to a thread a sequence: what the kernel below does, with what one step hands to the next in LDS, so that three trips to memory follow one another (lengths; entries that go back; the stack's top
// and entries of rows on pages that were there) instead of nine: a step of 64 sequences 9.4 -> 4.8 us on the device.
constexpr int kKept = 4096;              // pages of a step that LDS holds; where there are more, they are read back
struct SharedOnce {
    uint32_t goes[kThreads], takes[kThreads], starts[kThreads + 1];      // of the sequences: where their entries of the flat lists, and their tokens, end
    int32_t left[kThreads], stay[kThreads];
    uint32_t sums[2][kWaves], counts[2][kDeep * kWaves];
    unsigned long long tokens[kWaves];
    uint32_t taken;
    int32_t back[kKept], fresh[kKept];
};
// The first of the ascending sums that lies behind x, or the last of 2 half (half: a power of two, or 0).  (For 3183 entries, searches of several at a time, step by step, took LDS longer than they
// saved in trips to it, 11.9 us for 9.3; marks where sequences begin and a running maximum over them 10.3.)
__device__ __forceinline__ int first_behind(const uint32_t* sums, int half, uint32_t x)
{
    int k = 0;
    for (int step = half; step; step >>= 1)
        if (sums[k + step - 1] <= x) k += step;
    return k;
}

__global__ __launch_bounds__(kThreads) void paged_reserve_once_kernel(PagePool p, const int32_t* n_new, const int32_t* keep, int32_t* granted, StepRows rows)
{
    __shared__ SharedOnce sm;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int32_t* const stack = p.free_pages;
    const int room = p.table_stride << p.page_shift;
    const uint32_t up = (1u << p.page_shift) - 1u;
    const int half = p.n_seqs > 1 ? 1 << (31 - __builtin_clz((unsigned)(p.n_seqs - 1))) : 0;
    const int first_free = p.n_free[0], want = tid < p.n_seqs ? n_new[tid] : 0;
    const Sequence seq = sequence_at(p, keep, tid);
    int come = max(want, 0);
    if (come > room - seq.stay) come = 0;
    const uint32_t more = come > 0 ? (((uint32_t)(seq.stay + come) + up) >> p.page_shift) - (uint32_t)seq.left : 0u;
    uint32_t goes = wave_incl_scan_u32((uint32_t)(seq.had - seq.left)), takes = wave_incl_scan_u32(more);
    if (lane == 63) {
        sm.sums[0][wave] = goes;
        sm.sums[1][wave] = takes;
    }
    if (tid == 0) sm.taken = 0;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t n = sm.sums[0][w];
        goes += w < wave ? n : 0u;
        takes += w < wave ? sm.sums[1][w] : 0u;
        all += n;
    }
    sm.goes[tid] = goes;
    sm.takes[tid] = takes;
    sm.left[tid] = seq.left;
    sm.stay[tid] = seq.stay;
    __syncthreads();
    // Pages that go back.
    const uint32_t base = (uint32_t)min(max(first_free, 0), p.n_pages);
    uint32_t top = base;
    auto place_of = [&](const uint32_t* sums, int k, uint32_t x) { return p.table + (long long)k * p.table_stride + sm.left[k] + (int)(x - (k ? sums[k - 1] : 0u)); };
    auto push = [&](unsigned long long in, uint32_t before, int32_t page) {
        const uint32_t to = top + before + (uint32_t)__popcll(in & ((1ull << lane) - 1ull));
        if ((in >> lane & 1) && to < (uint32_t)p.n_pages) {      // (more than there are: a page that came twice)
            stack[to] = page;
            if (to - base < kKept) sm.back[to - base] = page;
        }
    };
    if (all <= kThreads) {
        int32_t page = -1;
        if ((uint32_t)tid < all) {
            int32_t* const entry = place_of(sm.goes, first_behind(sm.goes, half, (uint32_t)tid), (uint32_t)tid);
            page = *entry;
            *entry = -1;
        }
        const unsigned long long in = __ballot((uint32_t)page < (uint32_t)p.n_pages);
        if (lane == 0) sm.counts[0][wave] = (uint32_t)__popcll(in);
        __syncthreads();
        uint32_t before = 0, sum = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t n = sm.counts[0][w];
            before += w < wave ? n : 0u;
            sum += n;
        }
        push(in, before, page);
        top += sum;
    } else {
        int turn = 0;
        for (uint32_t x0 = 0; x0 < all; x0 += kDeep * kThreads, turn ^= 1) {
            int32_t page[kDeep];
            unsigned long long in[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const uint32_t x = x0 + (uint32_t)(i * kThreads + tid);
                page[i] = -1;
                if (x < all) {
                    int32_t* const entry = place_of(sm.goes, first_behind(sm.goes, half, x), x);
                    page[i] = *entry;
                    *entry = -1;
                }
            }
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                in[i] = __ballot((uint32_t)page[i] < (uint32_t)p.n_pages);
                if (lane == 0) sm.counts[turn][i * kWaves + wave] = (uint32_t)__popcll(in[i]);
            }
            __syncthreads();
            const uint32_t c0 = sm.counts[turn][2 * lane], c1 = sm.counts[turn][2 * lane + 1];
            const uint32_t upto = wave_incl_scan_u32(c0 + c1);
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int at = i * kWaves + wave;
                uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)(upto - c0 - c1), at >> 1);
                if (at & 1) before += (uint32_t)__builtin_amdgcn_readlane((int)c0, at >> 1);
                push(in[i], before, page[i]);
            }
            top += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
    }
    top = min(top, (uint32_t)p.n_pages);
    // Who gets what.
    const bool ok = more == 0 || takes <= top;
    if (!ok) come = 0;
    // (halves, so that a wave's sums of each stay within 32 bits)
    unsigned long long upto = ((unsigned long long)wave_incl_scan_u32((uint32_t)come >> 16) << 16) + wave_incl_scan_u32((uint32_t)come & 0xffffu);
    if (lane == 63) sm.tokens[wave] = upto;
    const unsigned long long got = __ballot(ok && more > 0);
    if (got && lane == 63 - __clzll((long long)got)) atomicMax(&sm.taken, takes);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) upto += w < wave ? sm.tokens[w] : 0ull;
    const uint32_t start = (uint32_t)min(upto, 0x7fffffffull);
    if (tid == 0) {
        p.q_start[0] = 0;
        sm.starts[0] = 0;
    }
    sm.starts[tid + 1] = start;
    if (tid < p.n_seqs) {
        p.kv_len[tid] = seq.stay + come;
        p.q_start[tid + 1] = (int32_t)start;
        if (granted) granted[tid] = come;
    }
    const uint32_t taken = sm.taken;
    if (tid == 0) p.n_free[0] = (int32_t)(top - taken);
    if (top - base > kKept) __syncthreads();               // (the stack is read back)
    auto popped = [&](uint32_t x) {
        const uint32_t from = top - 1u - x;
        return from >= base && top - base <= kKept ? sm.back[from - base] : stack[from];
    };
    auto take = [&](uint32_t x, int k, int32_t page) {
        *place_of(sm.takes, k, x) = page;
        stack[top - 1u - x] = -1;
        if (x < kKept) sm.fresh[x] = page;
    };
    for (uint32_t x = tid; x < taken; x += kThreads) {
        const int32_t page = popped(x);
        take(x, first_behind(sm.takes, half, x), page);
    }
    if (rows.n_rows <= 0) return;
    __syncthreads();
    for (int r = tid; r < rows.n_rows; r += kThreads) {
        const int k = first_behind(sm.starts + 1, half, (uint32_t)r);
        int position = -1;
        long long slot = -1;
        const bool there = (uint32_t)r < sm.starts[kThreads];
        if (there) {
            const int left = sm.left[k];
            position = sm.stay[k] + (r - (int)sm.starts[k]);
            const int e = position >> p.page_shift;
            const uint32_t x = (k ? sm.takes[k - 1] : 0u) + (uint32_t)(e - left);
            if (rows.slots) {
                const int32_t page = e >= left && x < kKept ? sm.fresh[x] : p.table[(long long)k * p.table_stride + e];
                if ((uint32_t)page < (uint32_t)p.n_pages) slot = ((long long)page << p.page_shift) + (position & (int)up);
            }
        }
        if (rows.sequence) rows.sequence[r] = there ? k : -1;
        if (rows.positions) rows.positions[r] = position;
        if (rows.slots) rows.slots[r] = slot;
    }
}

__global__ __launch_bounds__(256) void paged_map_kernel(PagePool p, StepRows rows)
{
    const int r0 = blockIdx.x * 256 + (threadIdx.x & ~63);
    if (r0 < rows.n_rows) map_rows(p, rows, r0);
}

// Whether the one workgroup maps the rows itself: it looks each one's sequence up by a search, as long as there are sequences, and a launch of its own costs 3.6 us whatever it does.  By itself and by
// a launch, us a call: 6000 rows of 8 sequences 7.4 and 10.3, of 64 8.5 and 10.2, of 200 9.7 and 10.2, of 1000 10.8 and 10.3; 7500 of 1000 12.0 and 10.2.
bool mapped_along(int n_rows, int n_seqs)
{
    int steps = 4;
    while (steps < 14 && 1 << (steps - 4) < n_seqs) ++steps;
    return (long long)n_rows * steps <= 1 << 16;
}

}  // namespace

hipError_t launch_paged_reserve(const PagePool& p, const int32_t* n_new, const int32_t* keep, int32_t* granted, const StepRows& rows, hipStream_t s)
{
    const bool apart = !mapped_along(rows.n_rows, p.n_seqs);
    StepRows here = rows;
    if (apart) here.n_rows = 0;
    const auto on = p.n_seqs <= kThreads ? Launch<paged_reserve_once_kernel>::on : Launch<paged_reserve_kernel>::on;
    const hipError_t e = on(dim3(1), dim3(kThreads), s, p, n_new, keep, granted, here);
    if (e != hipSuccess || !apart) return e;
    return Launch<paged_map_kernel>::on(dim3((unsigned)(((long long)rows.n_rows + 255) / 256)), dim3(256), s, p, rows);
}

}  // namespace mp
