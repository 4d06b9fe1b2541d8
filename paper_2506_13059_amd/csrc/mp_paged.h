// The paged cache as the kernels see it, and what its launches share (mp_rotary.hip, mp_norm_rotary.hip, mp_paged_*.hip).
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

// Norm of a head's rows, see mp_head_norm.  weight null: rows are not normed.
struct HeadNorm {
    const uint16_t* weight;
    int32_t stride;              // elements from one head's weights to the next one's: 128, or 0 where all heads have the same
    float offset, eps;
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
hipError_t launch_norm_rotary(const Rotation& rot, const HeadNorm& norm, const TokenRows& x, const int32_t* positions, int n_tokens, uint16_t* out,
                              long long out_stride, uint16_t* out_lookup, int lookup_position, hipStream_t s);
// positions: of every token, or null: where they stand in their sequences.
hipError_t launch_paged_append_norm(const PagedKv& c, const Rotation& rot, const HeadNorm& q_norm, const HeadNorm& k_norm, const int32_t* positions,
                                    const TokenRows& q, uint16_t* q_out, const TokenRows& k, const TokenRows& v, int n_tokens, hipStream_t s);
hipError_t launch_paged_gather(const PagedKv& c, const Rotation& rot, int first, int n, int lookup_position, uint16_t* k, uint16_t* k_lookup,
                               uint16_t* v, hipStream_t s);

// Page tables and what a step's tokens are, made on the device, see mp_page_pool.
struct PagePool {
    int32_t *table, *kv_len, *q_start, *free_pages, *n_free;
    int32_t n_pages, page_shift, n_seqs, table_stride;
};
struct StepRows {
    int32_t *sequence, *positions;
    int64_t* slots;
    int32_t n_rows;
};
hipError_t launch_paged_reserve(const PagePool& p, const int32_t* n_new, const int32_t* keep, int32_t* granted, const StepRows& rows, hipStream_t s);

// Trees of drafted tokens: every token's mask of `words` 64-bit words marks tokens of its sequence.
// every: rows without a result get a mask of zeros and position -1.
hipError_t launch_paged_tree_plan(const PagedKv& c, const int32_t* parents, int n_tokens, int words, bool every, uint64_t* mask, int32_t* positions, hipStream_t s);
hipError_t launch_paged_tree_keep(const PagedKv& c, const uint64_t* mask, int words, const int32_t* leaf, int n_tokens, int32_t* keep, hipStream_t s);

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
// ... of a tree's tokens: `mask` marks which new tokens of its sequence each one attends.
struct PagedTreeAttention : PagedAttention {
    const unsigned long long* mask;      // [n_tokens, words]
    int32_t words;
};
size_t paged_partial_floats(int n_tokens, int n_q_heads, int n_kv_heads, int n_seqs, int max_new);
// The kernel for few tokens: sequences of up to `rows` query rows a KV head (16, 32 or 64).
size_t paged_token_floats(int rows);
hipError_t launch_paged_tokens(const PagedAttention& a, int rows, float* room, hipStream_t s);
hipError_t launch_paged_tokens(const PagedTreeAttention& a, int rows, float* room, hipStream_t s);
hipError_t launch_paged_token_merge(const PagedAttention& a, int groups, const float* parts, const void* cuts, hipStream_t s);
// The kernel for trees of up to `rows` query rows a KV head (64 or 128), in room for paged_token_floats(rows).
hipError_t launch_paged_tree_rows(const PagedTreeAttention& a, int rows, float* room, hipStream_t s);
size_t paged_chunk_floats();
hipError_t launch_paged_chunks(const PagedAttention& a, int over, float* room, hipStream_t s);     // sequences of more than `over` query rows a head
hipError_t launch_paged_chunks(const PagedTreeAttention& a, int over, float* room, hipStream_t s);
bool paged_line_fits(const PagedAttention& a);
bool paged_line_fits(const PagedTreeAttention& a);     // what the kernels count of a call's blocks stays within 32 bits
hipError_t launch_paged_attention(const PagedAttention& a, hipStream_t s);
hipError_t launch_paged_attention(const PagedTreeAttention& a, hipStream_t s);

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
