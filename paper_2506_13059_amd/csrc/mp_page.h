// Where a key of a paged cache lies, for kernels and, so that it can be checked without a GPU, for the host.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define MP_PAGE_FN __host__ __device__ __forceinline__
#else
#define MP_PAGE_FN inline
#endif

namespace mp {

// The page of a position: -1 where it is negative, behind the table's end, or its entry names no page.  `row`: the sequence's entries.
MP_PAGE_FN int page_of(const int32_t* row, int table_stride, int n_pages, int page_shift, int position)
{
    const int entry = position >> page_shift;
    if (position < 0 || entry >= table_stride) return -1;
    const int page = row[entry];
    return page >= 0 && page < n_pages ? page : -1;
}

// Row of K and V, in rows of a head: page after page, head after head.
MP_PAGE_FN long long row_of(int page, int head, int n_kv, int page_shift, int position)
{
    return (((long long)page * n_kv + head) << page_shift) + (position & ((1 << page_shift) - 1));
}

// The entry of key unit * block + offset in a sequence's row of the table; behind its `end` keys (one at least), that of the last one.  Blocks that are asked for
// ahead may lie up to 2^31 keys behind the end, so the key is worked out in unsigned numbers.
MP_PAGE_FN int entry_of(int block, int unit, int offset, int end, int page_shift)
{
    const uint32_t key = (uint32_t)block * (uint32_t)unit + (uint32_t)offset, last = (uint32_t)end - 1u;
    return (int)((key < last ? key : last) >> page_shift);
}

// Blocks of `unit` keys that tokens [i0, i1] of a sequence attend (token i stands at position base + i): [b0, b1), one at least, so that
// rows without a key are someone's, too.  `room`: keys that the table has entries for.
MP_PAGE_FN void blocks_of(int base, int i0, int i1, int window, int room, int unit, int* b0, int* b1)
{
    const int end = base + i1 + 1 < room ? base + i1 + 1 : room;
    const int low = window > 0 && base + i0 >= window ? base + i0 - window + 1 : 0;
    *b0 = low / unit;
    *b1 = end > 0 ? (int)(((long long)end + unit - 1) / unit) : 0;
    if (*b1 <= *b0) *b1 = *b0 + 1;
}

// The lowest n of 64 bits.
MP_PAGE_FN unsigned long long below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }

// The parent of a tree's token: the number that the caller gave, if it is that of a token before it, or -1 (which, unlike any other number below zero, stays what it is in 16 bits).
MP_PAGE_FN int parent_of(int given, int token) { return given >= 0 && given < token ? given : -1; }

// A row of a tree attends the keys of its sequence that are older than the `n` new ones, `base` of them, and the new ones that its mask marks (bit i % 64 of word i / 64: the i-th); a window
// leaves it the last ones of all these.  Either way it attends the keys from a first one on, `low`, that are older or marked.
MP_PAGE_FN int tree_low(const unsigned long long* mask, int words, int base, int n, int window)
{
    if (window <= 0) return 0;
    int left = window;
    const int used = (int)(((long long)n + 63) >> 6);
    for (int w = (words < used ? words : used) - 1; w >= 0; --w) {
        unsigned long long m = mask[w] & below(n - 64 * w);
        const int marked = __builtin_popcountll(m);
        if (marked >= left) {                       // (it attends no older key)
            for (; left > 1; --left) m &= ~(1ull << (63 - __builtin_clzll(m)));
            return base + 64 * w + 63 - __builtin_clzll(m);
        }
        left -= marked;
    }
    return (base > left ? base : left) - left;
}
// Which of the 64 keys from `first` on such a row attends: a bit for each.  words: of its mask that count.
MP_PAGE_FN unsigned long long tree_keys(const unsigned long long* mask, int words, int low, int base, int first)
{
    const int at = first - base, w = at >> 6, by = at & 63;      // of the first key among the new ones
    unsigned long long marked = w >= 0 && w < words ? mask[w] >> by : 0ull;
    if (by && w + 1 >= 0 && w + 1 < words) marked |= mask[w + 1] << (64 - by);
    return (below(-at) | marked) & ~below(low - first);
}

// Work is cut into equal shares of blocks, a workgroup each, without regard to where an item (a tile of rows of a head) ends; the first
// and the last item of a share may be parts.  Which workgroup holds what of the item [x0, x1):
struct Parts {
    long long first, last;      // workgroups
};
MP_PAGE_FN Parts parts_of(long long x0, long long x1, long long share) { return Parts{x0 / share, (x1 - 1) / share}; }
// ... and in which of a workgroup's two slots: what it begins with, or what it ends with.
MP_PAGE_FN int slot_of(long long x0, long long workgroup, long long share) { return x0 > workgroup * share ? 1 : 0; }

}  // namespace mp
