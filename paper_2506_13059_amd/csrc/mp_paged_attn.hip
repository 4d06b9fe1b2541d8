// Attention of new tokens over a paged cache, for gfx950.
//
// Query row i of a sequence with n new tokens and len keys (the new ones among them) stands at position p = len - n + i and attends the
// keys j with p - window < j <= p (window 0: all up to p) whose page is there:
//     o = sum_j e^(s q.k_j - m) v_j / l,   l = sum_j e^(s q.k_j - m),   lse = m + ln l,
// a row without such a key gives zeros and -inf.
#include "mp_paged.h"

namespace mp {

size_t paged_partial_floats(int n_tokens, int n_q_heads, int n_kv_heads, int n_seqs, int max_new)
{
    return n_tokens > 0 ? paged_chunk_floats() : 0;
}

hipError_t launch_paged_attention(const PagedAttention& a, hipStream_t s)
{
    if (a.n_tokens <= 0 || a.c.n_seqs <= 0) return hipSuccess;
    return launch_paged_chunks(a, 0, a.partials, s);
}

}  // namespace mp
