// Norms of each head's queries and keys with the rotation in the same pass, for gfx950.
//
//     y = R(p) [ x / sqrt(mean(x^2) + eps) * (w + offset) ],
//
// the mean over the 128 dimensions of a row, R(p) as in mp_rotary.hip.  The sum of squares, the weights and the rotation are fp32, and the result is rounded to bf16 once.  The
// factor 1 / sqrt() is a row's, so it multiplies last; where all heads have the same weights these go into the cosines and sines of a token, once for all of its rows.
//
// Copies, bound by memory, or by a launch and its trips to memory where there are few tokens: a decode step's 16 tokens of 32 heads at two positions 4.5 us on the device, 16 tokens' append 5.3; five prompts' append
// (486 MB read and written, weights of each head) 97 us, 5.0 TB/s, as a large copy.  Rows by themselves: 32768 tokens of 32 heads 79 us, 6.8 TB/s, of 40 with weights of each 121, 5.5; 8191 of 32, which
// the last-level cache holds, 23.4 us, at two positions 32.6.
#include "mp_launch.h"
#include "mp_turn.h"

namespace mp {

namespace {

__device__ __forceinline__ float row_sum_f32(float v)
{
    v += dpp_f32<kDppXor1>(v);
    v += dpp_f32<kDppXor2>(v);
    v += dpp_f32<kDppHalfMirror>(v);
    v += dpp_f32<kDppMirror>(v);
    return v;
}

// 1 / sqrt(mean + eps) of the row that the lane has eight elements of.
__device__ __forceinline__ float row_factor(const float (&x)[8], float eps)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
    return rsqrtf(fmaf(row_sum_f32(s), 1.f / kHeadDim, eps));
}

// Rows whose sum of squares has passed fp32 (a factor of zero) again, scaled by 2^-70: elements reach 2^58 then, and squares of 128 of them 2^123.  All lanes take part.  Rows with an infinity
// keep their factor of zero, which meets finite numbers but for those of its pair: dims that are not turned become their own partners, for what they meet is a sine of zero, and an infinity of a
// neighbour would make NaN of it.  (Here, for where all elements are finite it makes no difference: done for every row it takes 128 us for 121, 32768 tokens of 40 heads with weights of each.)
__device__ __forceinline__ void scale_down(float (&x)[8], float (&y)[8], float& f, float eps, const Turn& t)
{
    const float by = f == 0.f ? 0x1p-70f : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] *= by;
        y[i] = i < t.n ? y[i] * by : x[i];
    }
    f = row_factor(x, eps * by * by);
}

// The weights of a lane's dims and of their partners, with the offset.
struct Weights {
    float own[8], partner[8];
};
__device__ __forceinline__ Weights weights_of(const uint4& w, float offset, const Turn& t, const Rotation& rot)
{
    Weights r;
    unpack(w, r.own);
    partners(w, t, rot, r.partner);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        r.own[i] += offset;
        r.partner[i] += offset;
    }
    return r;
}
__device__ __forceinline__ void fold(Turn& t, const Weights& w)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        t.cs[i] *= w.own[i];
        t.sn[i] *= w.partner[i];
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    bf16x2_t v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint4 scaled_turn(const float (&x)[8], const float (&y)[8], const Turn& t, float f)
{
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        u[i] = pack_bf16(fmaf(y[2 * i], t.sn[2 * i], x[2 * i] * t.cs[2 * i]) * f, fmaf(y[2 * i + 1], t.sn[2 * i + 1], x[2 * i + 1] * t.cs[2 * i + 1]) * f);
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// Rows [h0, h1) of one token and kind, `step` elements apart where they go.  Normed ones are turned by `turns` tables, the second for `also` (or null).
struct Rows {
    const uint16_t* from;
    uint16_t* to;
    long long step;
    uint16_t* also;
    int h0, h1;
};
template <bool kOnce, bool kHeads, bool kTwo>
__device__ __forceinline__ void normed_rows(const Rows& r, const HeadNorm& norm, const Rotation& rot, const float2* table, const float2* table2)
{
    const int lane = threadIdx.x & 63, c = lane & 15;
    Turn first = load_turn(table, rot), second{};
    if constexpr (kTwo) second = load_turn(table2, rot);
    if constexpr (!kHeads) {
        const Weights w = weights_of(reinterpret_cast<const uint4*>(norm.weight)[c], norm.offset, first, rot);
        fold(first, w);
        if constexpr (kTwo) fold(second, w);
    }
    for (int h0 = r.h0; h0 < r.h1; h0 += 4 * kDeep) {
        uint4 v[kDeep], w[kHeads ? kDeep : 1];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {                   // (rows past the end repeat the last one: all lanes take part in the exchange)
            const int h = min(h0 + 4 * i + (lane >> 4), r.h1 - 1);
            v[i] = reinterpret_cast<const uint4*>(r.from + (long long)h * kHeadDim)[c];
            if constexpr (kHeads) w[i] = reinterpret_cast<const uint4*>(norm.weight + (long long)h * kHeadDim)[c];
        }
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int h = h0 + 4 * i + (lane >> 4);
            if (h0 + 4 * i >= r.h1) break;
            float x[8], y[8];
            unpack(v[i], x);
            partners(v[i], first, rot, y);
            float f = row_factor(x, norm.eps);
            if (__any(f == 0.f)) scale_down(x, y, f, norm.eps, first);
            if constexpr (kHeads) {
                const Weights u = weights_of(w[i], norm.offset, first, rot);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] *= u.own[e];
                    y[e] *= u.partner[e];
                }
            }
            const uint4 a = scaled_turn(x, y, first, f);
            if (r.to && h < r.h1) store16<kOnce>(reinterpret_cast<uint4*>(r.to + h * r.step) + c, a);
            if constexpr (kTwo) {
                const uint4 b = scaled_turn(x, y, second, f);
                if (h < r.h1) store16<kOnce>(reinterpret_cast<uint4*>(r.also + (long long)h * kHeadDim) + c, b);
            }
        }
    }
}
// ... that are only turned (kTurned), or copied.
template <bool kOnce, bool kTurned>
__device__ __forceinline__ void plain_rows(const Rows& r, const Rotation& rot, const float2* table)
{
    const int lane = threadIdx.x & 63, c = lane & 15;
    Turn t{};
    if constexpr (kTurned) t = load_turn(table, rot);
    for (int h0 = r.h0; h0 < r.h1; h0 += 4 * kDeep) {
        uint4 v[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) v[i] = reinterpret_cast<const uint4*>(r.from + (long long)min(h0 + 4 * i + (lane >> 4), r.h1 - 1) * kHeadDim)[c];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int h = h0 + 4 * i + (lane >> 4);
            if (h0 + 4 * i >= r.h1) break;
            if constexpr (kTurned) {
                float y[8];
                partners(v[i], t, rot, y);
                v[i] = turned(v[i], y, t);
            }
            if (h < r.h1) store16<kOnce>(reinterpret_cast<uint4*>(r.to + h * r.step) + c, v[i]);
        }
    }
}

// One wave: `rows` rows (a multiple of four) of one token.
template <bool kOnce, bool kHeads>
__global__ __launch_bounds__(64 * kWaves) void norm_rotary_kernel(Rotation rot, HeadNorm norm, const uint16_t* x, long long x_stride, const int32_t* positions,
                                                                  uint16_t* out, long long out_stride, uint16_t* lookup, int lookup_position, int n_tokens,
                                                                  int n_heads, int rows, int parts)
{
    __shared__ float2 tables[kWaves][2][64];
    const int wave = threadIdx.x >> 6;
    const long long w = (long long)blockIdx.x * kWaves + wave;
    const int t = (int)(w / parts), part = (int)(w - (long long)t * parts);
    if (t >= n_tokens) return;
    Rows r;
    r.from = x + t * x_stride;
    r.to = out ? out + t * out_stride : lookup + (long long)t * n_heads * kHeadDim;
    r.step = kHeadDim;
    r.also = lookup + (long long)t * n_heads * kHeadDim;
    r.h0 = part * rows;
    r.h1 = min(n_heads, r.h0 + rows);
    fill_table(tables[wave][0], rot, out ? positions[t] : lookup_position);
    if (out && lookup) {
        fill_table(tables[wave][1], rot, lookup_position);
        normed_rows<kOnce, kHeads, true>(r, norm, rot, tables[wave][0], tables[wave][1]);
    } else {
        normed_rows<kOnce, kHeads, false>(r, norm, rot, tables[wave][0], nullptr);
    }
}

// One wave: `per` groups of up to four rows of one token, which are those of its query heads, then of its key heads, then of its value heads.
template <bool kOnce>
__global__ __launch_bounds__(64 * kWaves) void paged_append_norm_kernel(PagedKv cache, Rotation rot, HeadNorm q_norm, HeadNorm k_norm, const int32_t* positions,
                                                                        const uint16_t* q, long long q_stride, uint16_t* q_out, const uint16_t* k,
                                                                        long long k_stride, const uint16_t* v, long long v_stride, int n_tokens, int n_q, int per,
                                                                        int parts)
{
    __shared__ float2 tables[kWaves][64];
    const int wave = threadIdx.x >> 6;
    const long long w = (long long)blockIdx.x * kWaves + wave;
    const int t = (int)(w / parts), part = (int)(w - (long long)t * parts);
    if (t >= n_tokens) return;
    const int b = sequence_of(cache.q_start, cache.n_seqs, t);
    if (b < 0) return;
    const int place = cache.kv_len[b] - (cache.q_start[b + 1] - t);
    const int page = page_of(cache.table + (long long)b * cache.table_stride, cache.table_stride, cache.n_pages, cache.page_shift, place);
    fill_table(tables[wave], rot, positions ? positions[t] : place);
    const int of_q = (n_q + 3) >> 2, of_kv = (cache.n_kv + 3) >> 2;
    int g0 = part * per, g1 = min(of_q + 2 * of_kv, g0 + per);
    const long long at = row_of(max(page, 0), 0, cache.n_kv, cache.page_shift, place) * kHeadDim;
    auto normed = [&](const Rows& r, const HeadNorm& norm) {
        if (!norm.weight) plain_rows<kOnce, true>(r, rot, tables[wave]);
        else if (norm.stride) normed_rows<kOnce, true, false>(r, norm, rot, tables[wave], nullptr);
        else normed_rows<kOnce, false, false>(r, norm, rot, tables[wave], nullptr);
    };
    if (g0 < of_q) normed(Rows{q + t * q_stride, q_out + (long long)t * n_q * kHeadDim, kHeadDim, nullptr, 4 * g0, min(n_q, 4 * g1)}, q_norm);
    if (page < 0) return;
    g0 = max(g0 - of_q, 0);
    g1 -= of_q;
    const long long step = (long long)kHeadDim << cache.page_shift;
    if (g0 < min(g1, of_kv)) normed(Rows{k + t * k_stride, cache.K + at, step, nullptr, 4 * g0, min(cache.n_kv, 4 * g1)}, k_norm);
    g0 = max(g0 - of_kv, 0);
    g1 -= of_kv;
    if (g0 < g1) plain_rows<kOnce, false>(Rows{v + t * v_stride, cache.V + at, step, nullptr, 4 * g0, min(cache.n_kv, 4 * g1)}, rot, tables[wave]);
}

}  // namespace

hipError_t launch_norm_rotary(const Rotation& rot, const HeadNorm& norm, const TokenRows& x, const int32_t* positions, int n_tokens, uint16_t* out,
                              long long out_stride, uint16_t* out_lookup, int lookup_position, hipStream_t s)
{
    if (n_tokens <= 0) return hipSuccess;
    const int rows = rows_of_a_wave(n_tokens, x.n_heads), parts = (x.n_heads + rows - 1) / rows;
    const long long blocks = ((long long)n_tokens * parts + kWaves - 1) / kWaves;
    const bool once = past_caches((long long)n_tokens * x.n_heads * ((out != nullptr) + (out_lookup != nullptr)));
    const auto on = norm.stride ? (once ? Launch<norm_rotary_kernel<true, true>>::on : Launch<norm_rotary_kernel<false, true>>::on)
                                : (once ? Launch<norm_rotary_kernel<true, false>>::on : Launch<norm_rotary_kernel<false, false>>::on);
    return on(dim3((unsigned)blocks), dim3(64 * kWaves), s, rot, norm, x.p, x.stride, positions, out, out_stride, out_lookup, lookup_position, n_tokens, x.n_heads, rows,
              parts);
}

hipError_t launch_paged_append_norm(const PagedKv& c, const Rotation& rot, const HeadNorm& q_norm, const HeadNorm& k_norm, const int32_t* positions,
                                    const TokenRows& q, uint16_t* q_out, const TokenRows& k, const TokenRows& v, int n_tokens, hipStream_t s)
{
    if (n_tokens <= 0 || c.n_seqs <= 0) return hipSuccess;
    const int groups = (q.n_heads + 3) / 4 + 2 * ((c.n_kv + 3) / 4);
    const int per = rows_of_a_wave(n_tokens, 4 * groups) / 4, parts = (groups + per - 1) / per;
    const long long blocks = ((long long)n_tokens * parts + kWaves - 1) / kWaves;
    const auto on = past_caches((long long)n_tokens * (q.n_heads + 2 * c.n_kv)) ? Launch<paged_append_norm_kernel<true>>::on : Launch<paged_append_norm_kernel<false>>::on;
    return on(dim3((unsigned)blocks), dim3(64 * kWaves), s, c, rot, q_norm, k_norm, positions, q.p, q.stride, q_out, k.p, k.stride, v.p, v.stride, n_tokens, q.n_heads, per,
              parts);
}

}  // namespace mp
