// The paged cache as the kernels see it, and what its launches share (mp_rotary.hip, mp_paged_attn.hip, mp_paged_api.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mp_page.h"

namespace mp {

struct PagedKv {
    uint16_t* K;                 // bf16 [n_pages, n_kv, page, 128]
    uint16_t* V;
    const int32_t* table;        // [n_seqs, table_stride]
    const int32_t* kv_len;       // [n_seqs]
    const int32_t* q_start;      // [n_seqs + 1]
    int32_t n_pages, page_shift, n_kv, n_seqs, table_stride;
};

// Positions to angles, see mp_rotary_spec.  rot_dim == 0: rows stay as they are.
struct Rotation {
    const double* freqs;
    int32_t rot_dim, interleaved;
    float amplitude;
};

// Rows of n_tokens x n_heads, token after token `stride` elements apart.
struct TokenRows {
    const uint16_t* p;
    long long stride;
    int32_t n_heads;
};

hipError_t launch_rotary(const Rotation& rot, const TokenRows& x, const int32_t* positions, int n_tokens, uint16_t* out, long long out_stride,
                         uint16_t* out_lookup, int lookup_position, hipStream_t s);
hipError_t launch_paged_append(const PagedKv& c, const Rotation& rot, const TokenRows& q, uint16_t* q_out, const TokenRows& k, const TokenRows& v,
                               int n_tokens, hipStream_t s);
hipError_t launch_paged_gather(const PagedKv& c, const Rotation& rot, int first, int n, int lookup_position, uint16_t* k, uint16_t* k_lookup,
                               uint16_t* v, hipStream_t s);

struct PagedAttention {
    PagedKv c;
    const uint16_t* q;
    long long q_stride;
    int32_t n_tokens, n_q_heads, max_new, window;
    float scale_log2e;
    uint16_t* out;
    float* lse;
    float* partials;
};
size_t paged_partial_floats(int n_tokens, int n_q_heads, int n_kv_heads, int n_seqs, int max_new);
// The kernel for few tokens: sequences of up to `rows` query rows a KV head (16, 32 or 64).
size_t paged_token_floats(int rows);
hipError_t launch_paged_tokens(const PagedAttention& a, int rows, float* room, hipStream_t s);
size_t paged_chunk_floats();
hipError_t launch_paged_chunks(const PagedAttention& a, int over, float* room, hipStream_t s);     // sequences of more than `over` query rows a head
bool paged_line_fits(const PagedAttention& a);      // what the kernels count of a call's blocks stays within 32 bits
hipError_t launch_paged_attention(const PagedAttention& a, hipStream_t s);

// The sequence of token t: the last one that starts at or before it (sequences without new tokens start where the next one does), or -1
// where t lies before the first or behind the last.  All lanes of a wave ask for the same t; 64 starts are compared at a time, so a batch
// of up to 64 sequences costs one trip to memory and one of up to 4096 two.
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int n_seqs, int t)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = n_seqs + 1;                     // starts [lo, lo + n) are left; those before lo are <= t
    while (n > 0) {
        const int step = (n + 63) >> 6;
        const int at = lo + min((lane + 1) * step, n) - 1;
        const int before = __popcll(__ballot(q_start[at] <= t && lane * step < n));
        const int first = lo + min(before * step, n);
        if (step == 1) {
            lo = first;
            break;
        }
        n = min(step - 1, lo + n - first);          // (the start at the end of that step is > t)
        lo = first;
    }
    const int b = lo - 1;
    return b < n_seqs ? b : -1;
}

}  // namespace mp
