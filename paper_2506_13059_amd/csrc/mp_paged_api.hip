// C-ABI layer of rotary positions and the paged cache: argument checks and launches.  Context-free; errors go to mp_last_error(NULL).
#include "../../include/mp.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "mp_ctx.h"
#include "mp_paged.h"

using namespace mp;

namespace mp {
mp_status fail(mp_ctx* ctx, mp_status st, const char* fmt, ...);      // mp_api.hip
}

namespace {

constexpr long long kMostKeys = 0x7fffffff;
constexpr long long kMostRows = 4ll * 0x7fffffff;
constexpr long long kMostGroups = (1ll << 24) - 1;      // workgroups of 256: a launch counts its lanes in 32 bits
constexpr long long kMostTokens = 4 * kMostGroups;      // ... where every token has a wave
constexpr int kMostSequences = (1 << 22) - 1;                // ... of up to 1024 lanes each
constexpr int kMostTurns = 0x7fffffff - 1024;                // sequences are gone through up to 1024 at a time, in 32 bits

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

mp_status rotation_ok(const char* who, const mp_rotary_spec* r, Rotation* out)
{
    if (!r) return fail(nullptr, MP_EINVAL, "%s: null rotary spec", who);
    if (!r->freqs) return fail(nullptr, MP_EINVAL, "%s: null frequencies", who);
    if (r->rot_dim < 2 || r->rot_dim > kHeadDimHost || (r->rot_dim & 1))
        return fail(nullptr, MP_EINVAL, "%s: rot_dim %d is not an even number from 2 to 128", who, r->rot_dim);
    if (r->layout != MP_ROTARY_HALF && r->layout != MP_ROTARY_INTERLEAVED) return fail(nullptr, MP_EINVAL, "%s: unknown layout %d", who, r->layout);
    if (!std::isfinite(r->amplitude)) return fail(nullptr, MP_EINVAL, "%s: the amplitude is not finite", who);
    out->freqs = r->freqs;
    out->rot_dim = r->rot_dim;
    out->interleaved = r->layout == MP_ROTARY_INTERLEAVED;
    out->amplitude = r->amplitude;
    return MP_OK;
}

// norm null: rows are not normed.
mp_status norm_ok(const char* who, const char* what, const mp_head_norm* n, int32_t n_heads, HeadNorm* out)
{
    *out = HeadNorm{};
    if (!n) return MP_OK;
    if (!n->weight) return fail(nullptr, MP_EINVAL, "%s: null weights of %s", who, what);
    if (!aligned(n->weight)) return fail(nullptr, MP_EINVAL, "%s: the weights of %s do not start on 16 bytes", who, what);
    if (n->n_heads != 1 && n->n_heads != n_heads) return fail(nullptr, MP_EINVAL, "%s: weights of %d heads for %d heads of %s", who, n->n_heads, n_heads, what);
    if (!std::isfinite(n->offset)) return fail(nullptr, MP_EINVAL, "%s: the offset of %s is not finite", who, what);
    if (!(n->eps > 0.f) || !std::isfinite(n->eps)) return fail(nullptr, MP_EINVAL, "%s: eps of %s must be positive", who, what);
    out->weight = (const uint16_t*)n->weight;
    out->stride = n->n_heads == 1 ? 0 : kHeadDimHost;
    out->offset = n->offset;
    out->eps = n->eps;
    return MP_OK;
}

// Rows of n_heads heads a token, `stride` elements apart (0: densely packed).
mp_status rows_ok(const char* who, const char* what, const void* p, int64_t stride, int32_t n_heads, TokenRows* out)
{
    if (!p) return fail(nullptr, MP_EINVAL, "%s: null %s", who, what);
    if (!aligned(p)) return fail(nullptr, MP_EINVAL, "%s: %s does not start on 16 bytes", who, what);
    if (stride == 0) stride = (int64_t)n_heads * kHeadDimHost;
    if (stride < (int64_t)n_heads * kHeadDimHost || (stride & 7))
        return fail(nullptr, MP_EINVAL, "%s: token stride %lld of %s is no multiple of 8 or less than its %d rows", who, (long long)stride, what, n_heads);
    out->p = (const uint16_t*)p;
    out->stride = stride;
    out->n_heads = n_heads;
    return MP_OK;
}

mp_status cache_ok(const char* who, const mp_paged_kv* c, PagedKv* out)
{
    if (!c) return fail(nullptr, MP_EINVAL, "%s: null cache", who);
    if (c->head_dim != kHeadDimHost) return fail(nullptr, MP_EINVAL, "%s: head_dim %d is not 128", who, c->head_dim);
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_seqs < 0 || c->table_stride < 1)
        return fail(nullptr, MP_EINVAL, "%s: bad sizes n_pages=%d n_kv_heads=%d n_seqs=%d table_stride=%d", who, c->n_pages, c->n_kv_heads, c->n_seqs,
                    c->table_stride);
    if (c->page_size < 1 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
        return fail(nullptr, MP_EINVAL, "%s: page_size %d is not a power of two up to 1024", who, c->page_size);
    if ((long long)c->table_stride * c->page_size > kMostKeys)
        return fail(nullptr, MP_EINVAL, "%s: a sequence's pages hold more than 2^31 - 1 keys", who);
    if (c->n_seqs > kMostTurns) return fail(nullptr, MP_EINVAL, "%s: too many sequences", who);
    if (!c->k_pages || !c->v_pages) return fail(nullptr, MP_EINVAL, "%s: null pages", who);
    if (!aligned(c->k_pages) || !aligned(c->v_pages)) return fail(nullptr, MP_EINVAL, "%s: pages do not start on 16 bytes", who);
    if (c->n_seqs > 0 && (!c->page_table || !c->kv_len || !c->q_start)) return fail(nullptr, MP_EINVAL, "%s: null page_table, kv_len or q_start", who);
    out->K = (uint16_t*)c->k_pages;
    out->V = (uint16_t*)c->v_pages;
    out->table = c->page_table;
    out->kv_len = c->kv_len;
    out->q_start = c->q_start;
    out->n_pages = c->n_pages;
    out->page_shift = __builtin_ctz((unsigned)c->page_size);
    out->n_kv = c->n_kv_heads;
    out->n_seqs = c->n_seqs;
    out->table_stride = c->table_stride;
    return MP_OK;
}

// `count` of `bytes` each; a null pointer, or none of them, overlaps nothing.
struct Span {
    const void* p;
    long long count;
    int bytes;
};
bool overlap(const Span& a, const Span& b)
{
    const uintptr_t a0 = (uintptr_t)a.p, a1 = a0 + (uintptr_t)(a.count * a.bytes), b0 = (uintptr_t)b.p, b1 = b0 + (uintptr_t)(b.count * b.bytes);
    return a.p && b.p && a0 < a1 && b0 < b1 && a0 < b1 && b0 < a1;
}
// Whether a result lies on something that is read, or on another result.
template <int kResults, int kRead>
bool overlap(const Span (&results)[kResults], const Span (&read)[kRead])
{
    for (int i = 0; i < kResults; ++i) {
        for (const Span& r : read)
            if (overlap(results[i], r)) return true;
        for (int j = 0; j < i; ++j)
            if (overlap(results[i], results[j])) return true;
    }
    return false;
}

mp_status launched(const char* who, hipError_t e)
{
    return e == hipSuccess ? MP_OK : fail(nullptr, MP_EHIP, "%s: %s", who, hipGetErrorString(e));
}

// mp_rotary, and with a norm mp_norm_rotary.
mp_status turn_rows(const char* who, const mp_rotary_spec* rotary, const mp_head_norm* norm, const void* x, int64_t x_stride, const int32_t* positions,
                    int32_t n_tokens, int32_t n_heads, void* out, int64_t out_stride, void* out_lookup, int32_t lookup_position, void* stream)
{
    Rotation rot;
    mp_status st = rotation_ok(who, rotary, &rot);
    if (st != MP_OK) return st;
    if (n_tokens < 0 || n_heads < 1) return fail(nullptr, MP_EINVAL, "%s: bad sizes n_tokens=%d n_heads=%d", who, n_tokens, n_heads);
    HeadNorm nm;
    if ((st = norm_ok(who, "x", norm, n_heads, &nm)) != MP_OK) return st;
    if (n_tokens == 0) return MP_OK;
    if (!out && !out_lookup) return fail(nullptr, MP_EINVAL, "%s: no output", who);
    TokenRows in, to{};
    st = rows_ok(who, "x", x, x_stride, n_heads, &in);
    if (st != MP_OK) return st;
    if (out) {
        if (!positions) return fail(nullptr, MP_EINVAL, "%s: null positions", who);
        st = rows_ok(who, "out", out, out_stride, n_heads, &to);
        if (st != MP_OK) return st;
        if (out == x && to.stride != in.stride) return fail(nullptr, MP_EINVAL, "%s: in place, the strides of x and out have to be the same", who);
    }
    if (out_lookup && !aligned(out_lookup)) return fail(nullptr, MP_EINVAL, "%s: out_lookup does not start on 16 bytes", who);
    if (out_lookup && (out_lookup == out || (out_lookup == x && in.stride != (int64_t)n_heads * kHeadDimHost)))
        return fail(nullptr, MP_EINVAL, "%s: out_lookup overlaps another tensor", who);
    if (n_tokens > kMostTokens || (long long)n_tokens * n_heads > kMostRows) return fail(nullptr, MP_EINVAL, "%s: too many rows", who);
    if (norm)
        return launched(who, launch_norm_rotary(rot, nm, in, positions, n_tokens, (uint16_t*)out, to.stride, (uint16_t*)out_lookup, lookup_position,
                                                (hipStream_t)stream));
    return launched(who, launch_rotary(rot, in, positions, n_tokens, (uint16_t*)out, to.stride, (uint16_t*)out_lookup, lookup_position, (hipStream_t)stream));
}

// mp_paged_append, and with norms or positions mp_paged_append_norm.
mp_status append(const char* who, const mp_paged_kv* cache, const mp_rotary_spec* rotary, const mp_head_norm* q_norm, const mp_head_norm* k_norm,
                 const int32_t* positions, const void* q, int64_t q_stride, int32_t n_q_heads, void* q_out, const void* k, int64_t k_stride, const void* v,
                 int64_t v_stride, int32_t n_tokens, void* stream)
{
    PagedKv c;
    Rotation rot{};
    mp_status st = cache_ok(who, cache, &c);
    if (st != MP_OK) return st;
    if (rotary && (st = rotation_ok(who, rotary, &rot)) != MP_OK) return st;
    if (n_tokens < 0) return fail(nullptr, MP_EINVAL, "%s: n_tokens %d < 0", who, n_tokens);
    if ((q == nullptr) != (q_out == nullptr)) return fail(nullptr, MP_EINVAL, "%s: q and q_out go together", who);
    if (q && n_q_heads < 1) return fail(nullptr, MP_EINVAL, "%s: bad n_q_heads %d", who, n_q_heads);
    HeadNorm qn, kn;
    if ((st = norm_ok(who, "q", q ? q_norm : nullptr, n_q_heads, &qn)) != MP_OK || (st = norm_ok(who, "k", k_norm, c.n_kv, &kn)) != MP_OK) return st;
    if (n_tokens == 0) return MP_OK;
    TokenRows tq{}, tk, tv;
    if (q) {
        if ((st = rows_ok(who, "q", q, q_stride, n_q_heads, &tq)) != MP_OK) return st;
        if (!aligned(q_out)) return fail(nullptr, MP_EINVAL, "%s: q_out does not start on 16 bytes", who);
        if (q == q_out && tq.stride != (int64_t)n_q_heads * kHeadDimHost) return fail(nullptr, MP_EINVAL, "%s: in place, q has to be densely packed", who);
    }
    if ((st = rows_ok(who, "k", k, k_stride, c.n_kv, &tk)) != MP_OK) return st;
    if ((st = rows_ok(who, "v", v, v_stride, c.n_kv, &tv)) != MP_OK) return st;
    if (n_tokens > kMostTokens || n_tokens * (tq.n_heads + 2ll * c.n_kv) > kMostRows) return fail(nullptr, MP_EINVAL, "%s: too many rows", who);
    if (q_norm || k_norm || positions)
        return launched(who, launch_paged_append_norm(c, rot, qn, kn, positions, tq, (uint16_t*)q_out, tk, tv, n_tokens, (hipStream_t)stream));
    return launched(who, launch_paged_append(c, rot, tq, (uint16_t*)q_out, tk, tv, n_tokens, (hipStream_t)stream));
}

mp_status mask_ok(const char* who, const uint64_t* mask, int32_t words, int32_t n_tokens)
{
    if (n_tokens < 0) return fail(nullptr, MP_EINVAL, "%s: n_tokens %d < 0", who, n_tokens);
    if (words < 1 || words > 16) return fail(nullptr, MP_EINVAL, "%s: mask_words %d is not 1 .. 16", who, words);
    if (n_tokens > 0 && !mask) return fail(nullptr, MP_EINVAL, "%s: null mask", who);
    if ((uintptr_t)mask & 7) return fail(nullptr, MP_EINVAL, "%s: the mask does not start on 8 bytes", who);
    return MP_OK;
}

// `a` holds what the two forms of attention differ in.
template <class A>
mp_status attention(const char* who, A& a, const mp_paged_kv* cache, const void* q, int64_t q_stride, int32_t n_tokens, int32_t n_q_heads, int32_t max_new,
                    int32_t window, float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    mp_status st = cache_ok(who, cache, &a.c);
    if (st != MP_OK) return st;
    if (n_tokens < 0 || n_q_heads < 1 || n_q_heads % a.c.n_kv || max_new < 0 || window < 0)
        return fail(nullptr, MP_EINVAL, "%s: bad arguments n_tokens=%d Hq=%d Hkv=%d max_new=%d window=%d", who, n_tokens, n_q_heads, a.c.n_kv, max_new, window);
    if (n_q_heads / a.c.n_kv > 8) return fail(nullptr, MP_EINVAL, "%s: group size %d > 8 is not supported", who, n_q_heads / a.c.n_kv);
    if (!(softmax_scale >= 0.f) || !std::isfinite(softmax_scale)) return fail(nullptr, MP_EINVAL, "%s: softmax_scale must be finite and not negative", who);
    if (n_tokens == 0 || a.c.n_seqs == 0) return MP_OK;
    TokenRows rows;
    if ((st = rows_ok(who, "q", q, q_stride, n_q_heads, &rows)) != MP_OK) return st;
    if (!out || !aligned(out)) return fail(nullptr, MP_EINVAL, "%s: out is null or does not start on 16 bytes", who);
    if (max_new == 0 || max_new > n_tokens) max_new = n_tokens;
    const size_t need = mp_paged_workspace_bytes(n_tokens, n_q_heads, a.c.n_kv, a.c.n_seqs, max_new);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(nullptr, MP_EINVAL, "%s: workspace of %zu bytes, %zu are needed", who, workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned(workspace)) return fail(nullptr, MP_EINVAL, "%s: the workspace does not start on 16 bytes", who);
    // (workgroups that share a tile of query rows read them until the last of them is done)
    const uintptr_t q0 = (uintptr_t)q, q1 = q0 + 2 * ((uint64_t)(n_tokens - 1) * rows.stride + (uint64_t)n_q_heads * kHeadDimHost);
    const uintptr_t o0 = (uintptr_t)out, o1 = o0 + 2 * (uint64_t)n_tokens * n_q_heads * kHeadDimHost;
    if (o0 < q1 && q0 < o1) return fail(nullptr, MP_EINVAL, "%s: out overlaps the rows of q", who);
    a.q = rows.p;
    a.q_stride = rows.stride;
    a.n_tokens = n_tokens;
    a.n_q_heads = n_q_heads;
    a.max_new = max_new;
    a.window = window;
    const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)kHeadDimHost);
    a.scale_log2e = scale * 1.4426950408889634f;
    a.out = (uint16_t*)out;
    a.lse = lse;
    a.partials = (float*)workspace;
    if (!paged_line_fits(a)) return fail(nullptr, MP_EINVAL, "%s: too many tokens over a page table with room for so many keys", who);
    return launched(who, launch_paged_attention(a, (hipStream_t)stream));
}

}  // namespace

extern "C" {

mp_status mp_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len, double low, double high, double* freqs)
{
    const char* who = "mp_rotary_frequencies";
    if (!freqs) return fail(nullptr, MP_EINVAL, "%s: null pointer", who);
    if (rot_dim < 2 || rot_dim > kHeadDimHost || (rot_dim & 1)) return fail(nullptr, MP_EINVAL, "%s: rot_dim %d is not an even number from 2 to 128", who, rot_dim);
    if (scaling < MP_ROTARY_PLAIN || scaling > MP_ROTARY_BY_PARTS) return fail(nullptr, MP_EINVAL, "%s: unknown scaling %d", who, scaling);
    if (!(base > 0.0) || !std::isfinite(base)) return fail(nullptr, MP_EINVAL, "%s: base must be positive", who);
    if (scaling != MP_ROTARY_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return fail(nullptr, MP_EINVAL, "%s: factor must be positive", who);
    if (scaling == MP_ROTARY_BASE && rot_dim == 2) return fail(nullptr, MP_EINVAL, "%s: one pair has no base to scale", who);
    if (scaling == MP_ROTARY_BY_PARTS && (!(original_len > 0.0) || !std::isfinite(original_len) || !(low < high) || !std::isfinite(low) || !std::isfinite(high)))
        return fail(nullptr, MP_EINVAL, "%s: by parts needs original_len > 0 and low < high", who);
    if (scaling == MP_ROTARY_BASE) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot_dim);
        if (scaling == MP_ROTARY_LINEAR) f /= factor;
        if (scaling == MP_ROTARY_BY_PARTS) {
            const double turns = original_len * f / 6.283185307179586476925;
            double keep = (turns - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = f * keep + f / factor * (1.0 - keep);
        }
        freqs[i] = f;
    }
    return MP_OK;
}

mp_status mp_rotary(const mp_rotary_spec* rotary, const void* x, int64_t x_stride, const int32_t* positions, int32_t n_tokens, int32_t n_heads, void* out,
                    int64_t out_stride, void* out_lookup, int32_t lookup_position, void* stream)
{
    return turn_rows("mp_rotary", rotary, nullptr, x, x_stride, positions, n_tokens, n_heads, out, out_stride, out_lookup, lookup_position, stream);
}

mp_status mp_norm_rotary(const mp_head_norm* norm, const mp_rotary_spec* rotary, const void* x, int64_t x_stride, const int32_t* positions, int32_t n_tokens,
                         int32_t n_heads, void* out, int64_t out_stride, void* out_lookup, int32_t lookup_position, void* stream)
{
    const char* who = "mp_norm_rotary";
    if (!norm) return fail(nullptr, MP_EINVAL, "%s: null norm", who);
    return turn_rows(who, rotary, norm, x, x_stride, positions, n_tokens, n_heads, out, out_stride, out_lookup, lookup_position, stream);
}

mp_status mp_paged_append(const mp_paged_kv* cache, const mp_rotary_spec* rotary, const void* q, int64_t q_stride, int32_t n_q_heads, void* q_out, const void* k,
                          int64_t k_stride, const void* v, int64_t v_stride, int32_t n_tokens, void* stream)
{
    return append("mp_paged_append", cache, rotary, nullptr, nullptr, nullptr, q, q_stride, n_q_heads, q_out, k, k_stride, v, v_stride, n_tokens, stream);
}

mp_status mp_paged_append_norm(const mp_paged_kv* cache, const mp_rotary_spec* rotary, const mp_head_norm* q_norm, const mp_head_norm* k_norm,
                               const int32_t* positions, const void* q, int64_t q_stride, int32_t n_q_heads, void* q_out, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, int32_t n_tokens, void* stream)
{
    return append("mp_paged_append_norm", cache, rotary, q_norm, k_norm, positions, q, q_stride, n_q_heads, q_out, k, k_stride, v, v_stride, n_tokens, stream);
}

mp_status mp_paged_gather(const mp_paged_kv* cache, const mp_rotary_spec* rotary, int32_t first, int32_t n, int32_t lookup_position, void* k, void* k_lookup,
                          void* v, void* stream)
{
    const char* who = "mp_paged_gather";
    PagedKv c;
    Rotation rot{};
    mp_status st = cache_ok(who, cache, &c);
    if (st != MP_OK) return st;
    if (k_lookup && (st = rotation_ok(who, rotary, &rot)) != MP_OK) return st;
    if (first < 0 || n < 0 || (long long)first + n > kMostKeys) return fail(nullptr, MP_EINVAL, "%s: bad range first=%d n=%d", who, first, n);
    if (!k && !k_lookup && !v) return fail(nullptr, MP_EINVAL, "%s: no output", who);
    if (!aligned(k) || !aligned(k_lookup) || !aligned(v)) return fail(nullptr, MP_EINVAL, "%s: an output does not start on 16 bytes", who);
    if (((long long)n + 15) / 16 * c.n_seqs > kMostGroups) return fail(nullptr, MP_EINVAL, "%s: too many rows", who);
    return launched(who, launch_paged_gather(c, rot, first, n, lookup_position, (uint16_t*)k, (uint16_t*)k_lookup, (uint16_t*)v, (hipStream_t)stream));
}

size_t mp_paged_workspace_bytes(int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_seqs, int32_t max_new)
{
    if (n_tokens < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 8 || n_seqs < 0 || max_new < 0) return 0;
    if (max_new == 0 || max_new > n_tokens) max_new = n_tokens;
    return sizeof(float) * paged_partial_floats(n_tokens, n_q_heads, n_kv_heads, n_seqs, max_new);
}

mp_status mp_paged_attention(const mp_paged_kv* cache, const void* q, int64_t q_stride, int32_t n_tokens, int32_t n_q_heads, int32_t max_new, int32_t window,
                             float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    PagedAttention a{};
    return attention("mp_paged_attention", a, cache, q, q_stride, n_tokens, n_q_heads, max_new, window, softmax_scale, out, lse, workspace, workspace_bytes, stream);
}

mp_status mp_paged_tree_attention(const mp_paged_kv* cache, const void* q, int64_t q_stride, const uint64_t* mask, int32_t mask_words, int32_t n_tokens,
                                  int32_t n_q_heads, int32_t max_new, int32_t window, float softmax_scale, void* out, float* lse, void* workspace,
                                  size_t workspace_bytes, void* stream)
{
    const char* who = "mp_paged_tree_attention";
    PagedTreeAttention a{};
    const mp_status st = mask_ok(who, mask, mask_words, n_tokens);
    if (st != MP_OK) return st;
    const long long rows = (long long)n_tokens * n_q_heads, marks = (long long)n_tokens * mask_words;
    if (overlap(Span{out, rows, 2 * kHeadDimHost}, Span{mask, marks, 8}) || overlap(Span{lse, rows, 4}, Span{mask, marks, 8}))
        return fail(nullptr, MP_EINVAL, "%s: out or lse overlaps the mask", who);
    a.mask = (const unsigned long long*)mask;
    a.words = mask_words;
    return attention(who, a, cache, q, q_stride, n_tokens, n_q_heads, max_new, window, softmax_scale, out, lse, workspace, workspace_bytes, stream);
}

mp_status mp_paged_tree_plan(const mp_paged_kv* cache, const int32_t* parents, int32_t n_tokens, int32_t mask_words, uint64_t* mask, int32_t* positions, void* stream)
{
    const char* who = "mp_paged_tree_plan";
    PagedKv c;
    mp_status st = cache_ok(who, cache, &c);
    const bool every = mask_words > 0 && (mask_words & MP_TREE_EVERY_ROW);
    if (every) mask_words &= ~MP_TREE_EVERY_ROW;
    if (st != MP_OK || (st = mask_ok(who, mask, mask_words, n_tokens)) != MP_OK) return st;
    if (n_tokens == 0 || (c.n_seqs == 0 && !every)) return MP_OK;
    if (!parents || !positions) return fail(nullptr, MP_EINVAL, "%s: null parents or positions", who);
    if (c.n_seqs > kMostSequences) return fail(nullptr, MP_EINVAL, "%s: more than %d sequences", who, kMostSequences);
    // (other sequences' workgroups read while one writes)
    if (overlap({{mask, (long long)n_tokens * mask_words, 8}, {positions, n_tokens, 4}}, {{parents, n_tokens, 4}, {c.kv_len, c.n_seqs, 4}, {c.q_start, c.n_seqs + 1ll, 4}}))
        return fail(nullptr, MP_EINVAL, "%s: the mask or the positions overlap another argument", who);
    return launched(who, launch_paged_tree_plan(c, parents, n_tokens, mask_words, every, mask, positions, (hipStream_t)stream));
}

mp_status mp_paged_tree_keep(const mp_paged_kv* cache, const uint64_t* mask, int32_t mask_words, int32_t n_tokens, const int32_t* leaf, int32_t* keep, void* stream)
{
    const char* who = "mp_paged_tree_keep";
    PagedKv c;
    mp_status st = cache_ok(who, cache, &c);
    if (st != MP_OK || (st = mask_ok(who, mask, mask_words, n_tokens)) != MP_OK) return st;
    if (c.n_seqs == 0) return MP_OK;
    if (!leaf || !keep) return fail(nullptr, MP_EINVAL, "%s: null leaf or keep", who);
    if (2ll * c.n_kv * c.n_seqs > kMostTokens) return fail(nullptr, MP_EINVAL, "%s: too many heads of sequences", who);
    if (overlap({{keep, c.n_seqs, 4}}, {{leaf, c.n_seqs, 4}, {mask, (long long)n_tokens * mask_words, 8}, {c.kv_len, c.n_seqs, 4}, {c.q_start, c.n_seqs + 1ll, 4},
                                        {c.table, (long long)c.n_seqs * c.table_stride, 4}}))
        return fail(nullptr, MP_EINVAL, "%s: keep overlaps another argument", who);
    return launched(who, launch_paged_tree_keep(c, mask, mask_words, leaf, n_tokens, keep, (hipStream_t)stream));
}

mp_status mp_paged_reserve(const mp_page_pool* pool, const int32_t* n_new, const int32_t* keep, int32_t* granted, int32_t* sequence, int32_t* positions,
                           int64_t* slots, int32_t n_rows, void* stream)
{
    const char* who = "mp_paged_reserve";
    if (!pool) return fail(nullptr, MP_EINVAL, "%s: null pool", who);
    if (pool->n_pages < 1 || pool->n_seqs < 0 || pool->table_stride < 1)
        return fail(nullptr, MP_EINVAL, "%s: bad sizes n_pages=%d n_seqs=%d table_stride=%d", who, pool->n_pages, pool->n_seqs, pool->table_stride);
    if (pool->page_size < 1 || pool->page_size > 1024 || (pool->page_size & (pool->page_size - 1)))
        return fail(nullptr, MP_EINVAL, "%s: page_size %d is not a power of two up to 1024", who, pool->page_size);
    if ((long long)pool->table_stride * pool->page_size > kMostKeys || (long long)pool->n_pages * pool->page_size > kMostKeys)
        return fail(nullptr, MP_EINVAL, "%s: a sequence's pages, or all of them, hold more than 2^31 - 1 keys", who);
    if ((long long)pool->n_seqs * pool->table_stride > kMostKeys) return fail(nullptr, MP_EINVAL, "%s: the page table has more than 2^31 - 1 entries", who);
    if (!pool->free_pages || !pool->n_free || !pool->q_start) return fail(nullptr, MP_EINVAL, "%s: null free_pages, n_free or q_start", who);
    if (pool->n_seqs > 0 && (!pool->page_table || !pool->kv_len || !n_new)) return fail(nullptr, MP_EINVAL, "%s: null page_table, kv_len or n_new", who);
    if (n_rows < 0) return fail(nullptr, MP_EINVAL, "%s: n_rows %d < 0", who, n_rows);
    if (!sequence && !positions && !slots) n_rows = 0;
    // (rows are gone through 64 at a time; one of 2^31 - 1 would lie before no start)
    if (n_rows > kMostKeys - 64 || pool->n_seqs > kMostTurns) return fail(nullptr, MP_EINVAL, "%s: too many rows or sequences", who);
    const long long n = pool->n_seqs;
    if (overlap({{pool->page_table, n * pool->table_stride, 4}, {pool->kv_len, n, 4}, {pool->q_start, n + 1, 4}, {pool->free_pages, pool->n_pages, 4}, {pool->n_free, 1, 4},
                 {granted, n, 4}, {sequence, n_rows, 4}, {positions, n_rows, 4}, {slots, n_rows, 8}},
                {{n_new, n, 4}, {keep, n, 4}}))
        return fail(nullptr, MP_EINVAL, "%s: what is written overlaps another argument", who);
    if ((uintptr_t)slots & 7) return fail(nullptr, MP_EINVAL, "%s: slots do not start on 8 bytes", who);
    PagePool p;
    p.table = pool->page_table;
    p.kv_len = pool->kv_len;
    p.q_start = pool->q_start;
    p.free_pages = pool->free_pages;
    p.n_free = pool->n_free;
    p.n_pages = pool->n_pages;
    p.page_shift = __builtin_ctz((unsigned)pool->page_size);
    p.n_seqs = pool->n_seqs;
    p.table_stride = pool->table_stride;
    return launched(who, launch_paged_reserve(p, n_new, keep, granted, StepRows{sequence, positions, slots, n_rows}, (hipStream_t)stream));
}

}  // extern "C"
