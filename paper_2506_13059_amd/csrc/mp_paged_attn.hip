// Attention of new tokens over a paged cache, for gfx950.
//
// Query row i of a sequence with n new tokens and len keys (the new ones among them) stands at position p = len - n + i and attends the
// keys j with p - window < j <= p (window 0: all up to p) whose page is there:
//     o = sum_j e^(s q.k_j - m) v_j / l,   l = sum_j e^(s q.k_j - m),   lse = m + ln l,
// a row without such a key gives zeros and -inf.
#include "mp_paged.h"

namespace mp {

namespace {

// Which kernels a call runs.  That for few tokens takes sequences of up to `tokens` query rows a KV head (0: it does not run): as many as any sequence can
// have, where it can (64 rows each of 8 sequences of up to 30K keys: 103 us, by that for chunks 132).  Otherwise that for chunks runs, and the former takes the sequences of up
// to 16 rows, unless none need be there (one sequence, or as many tokens in the call as its sequences can have); fifteen tokens beside 333 of a prompt: 151 us by that for chunks alone, 122 by both, when both were new.
struct Kernels {
    int tokens;
    bool chunks;
};
Kernels kernels_of(int n_tokens, int group, int n_seqs, int max_new)
{
    const long long rows = (long long)max_new * group;
    for (int most = 16; most <= 64; most *= 2)
        if (rows <= most) return Kernels{most, false};
    return Kernels{n_seqs > 1 && (long long)n_seqs * max_new > n_tokens ? 16 : 0, true};
}

}  // namespace

size_t paged_partial_floats(int n_tokens, int n_q_heads, int n_kv_heads, int n_seqs, int max_new)
{
    if (n_tokens <= 0 || n_seqs <= 0) return 0;
    const Kernels k = kernels_of(n_tokens, n_q_heads / n_kv_heads, n_seqs, max_new);
    return (k.tokens ? paged_token_floats(k.tokens) : 0) + (k.chunks ? paged_chunk_floats() : 0);
}

hipError_t launch_paged_attention(const PagedAttention& a, hipStream_t s)
{
    if (a.n_tokens <= 0 || a.c.n_seqs <= 0) return hipSuccess;
    const Kernels k = kernels_of(a.n_tokens, a.n_q_heads / a.c.n_kv, a.c.n_seqs, a.max_new);
    float* room = a.partials;
    if (k.tokens) {
        const hipError_t e = launch_paged_tokens(a, k.tokens, room, s);
        if (e != hipSuccess) return e;
        room += paged_token_floats(k.tokens);
    }
    return k.chunks ? launch_paged_chunks(a, k.tokens, room, s) : hipSuccess;
}

}  // namespace mp
