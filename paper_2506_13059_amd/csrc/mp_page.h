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

}  // namespace mp
