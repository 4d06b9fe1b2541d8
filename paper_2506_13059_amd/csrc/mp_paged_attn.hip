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
// have, where it can (8 sequences of up to 30K keys, 40 and 64 rows each: 95 and 107 us, by that for chunks 110 and 123; of up to 1000 keys equal).  Otherwise that
// for chunks runs, and the former takes the sequences of up to 16 rows, unless none need be there (one sequence, or as many tokens in the call as its sequences can have).
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

// Short sequences beside longer ones go to their own kernel if they can have this many rows of keys, all heads together: its two launches cost 8 to 13 us and it reads keys
// at 6.6 TB/s, where in the kernel for chunks a sequence's few rows keep one wave of eight busy.  Single tokens beside a piece of 333 tokens, 8 KV heads of four, us by both kernels
// and by that for chunks alone: 15 sequences that see 1023 keys 54 and 43, 4096 keys 94 and 97 (0.5M rows), a window of 4096 in 16K 98 and 101, up to 16K 153 and 172 (2M); 63 of up
// to 4096 keys 113 and 136, of up to 16K 326 and 438; 1 and 3 of up to 16K 136 and 123, 135 and 127.  Lengths are known on the device only: what the page table or the window allows
// stands for them, so a table with room for much more than its sequences hold costs them those 8 to 13 us.
constexpr long long kOwnKernelRows = 3 << 18;

bool short_ones_apart(const PagedAttention& a)
{
    const long long room = (long long)a.c.table_stride << a.c.page_shift;
    return (a.c.n_seqs - 1) * (a.window > 0 && a.window < room ? a.window : room) >= kOwnKernelRows / a.c.n_kv;
}

}  // namespace

size_t paged_partial_floats(int n_tokens, int n_q_heads, int n_kv_heads, int n_seqs, int max_new)
{
    if (n_tokens <= 0 || n_seqs <= 0) return 0;
    const Kernels k = kernels_of(n_tokens, n_q_heads / n_kv_heads, n_seqs, max_new);
    return (k.tokens ? paged_token_floats(k.tokens) : 0) + (k.chunks ? paged_chunk_floats() : 0);
}

// A head's blocks on the line (mp_paged_plan.h) at most, in the kernel that has the smaller tiles, blocks and more places in front; tiles: what all tokens fill, and one that is not full a sequence.
bool paged_line_fits(const PagedAttention& a)
{
    const long long tokens = 256 / (a.n_q_heads / a.c.n_kv), room = (long long)a.c.table_stride << a.c.page_shift;
    const long long keys = a.window > 0 && a.window + tokens < room ? a.window + tokens : room;
    const long long tiles = a.n_tokens / tokens + (a.c.n_seqs < a.n_tokens ? a.c.n_seqs : a.n_tokens);
    return tiles * (keys / 64 + 5) < 1ll << 32;
}

hipError_t launch_paged_attention(const PagedAttention& a, hipStream_t s)
{
    if (a.n_tokens <= 0 || a.c.n_seqs <= 0) return hipSuccess;
    Kernels k = kernels_of(a.n_tokens, a.n_q_heads / a.c.n_kv, a.c.n_seqs, a.max_new);
    if (k.chunks && !short_ones_apart(a)) k.tokens = 0;
    float* room = a.partials;
    if (k.tokens) {
        const hipError_t e = launch_paged_tokens(a, k.tokens, room, s);
        if (e != hipSuccess) return e;
        room += paged_token_floats(k.tokens);
    }
    return k.chunks ? launch_paged_chunks(a, k.tokens, room, s) : hipSuccess;
}

}  // namespace mp
