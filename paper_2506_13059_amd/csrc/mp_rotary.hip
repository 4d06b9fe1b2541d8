// Rotary positions, the paged cache's append and its rows in order, for gfx950.
//
// A pair (x0, x1) of a row at position p becomes A (x0 cos - x1 sin, x1 cos + x0 sin) with the angle p theta of its frequency.  The angle
// is worked out in fp64, in turns (p theta / 2 pi; what is left of it after whole turns goes to fp32), so far positions lose nothing;
// sine and cosine, the products and their sum are fp32, and the result is rounded to bf16 once.
//
// All three are copies that rotate on the way: bound by memory, or by a launch and two trips to memory where there are few tokens.  A
// row is 16 lanes of 16 bytes.  Sines and cosines of a position are worked out once a wave (one pair a lane) or workgroup and serve all of its
// heads from LDS; a lane's partner elements of the half layout come from another lane's registers.  A decode step's calls take 4.4 to 4.8 us on the device; 8191 tokens' 40
// query heads 34 us (4.9 TB/s read and written), five prompts' append 94 us (5.2 TB/s), the gather of four sequences of 64K with lookup keys 509 us (5.3 TB/s).
#include "mp_turn.h"

namespace mp {

namespace {

// One wave: `rows` rows (a multiple of four) of one token.
template <bool kOnce>
__global__ __launch_bounds__(64 * kWaves) void rotary_kernel(Rotation rot, const uint16_t* x, long long x_stride, const int32_t* positions,
                                                             uint16_t* out, long long out_stride, uint16_t* lookup, int lookup_position,
                                                             int n_tokens, int n_heads, int rows, int parts)
{
    __shared__ float2 tables[kWaves][2][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15;
    const long long w = (long long)blockIdx.x * kWaves + wave;
    const int t = (int)(w / parts), part = (int)(w - (long long)t * parts);
    if (t >= n_tokens) return;
    Turn own{}, fixed{};
    if (out) {
        fill_table(tables[wave][0], rot, positions[t]);
        own = load_turn(tables[wave][0], rot);
    }
    if (lookup) {
        fill_table(tables[wave][1], rot, lookup_position);
        fixed = load_turn(tables[wave][1], rot);
    }
    const int end = min(n_heads, (part + 1) * rows);
    for (int h0 = part * rows; h0 < end; h0 += 4 * kDeep) {
        uint4 v[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {                   // (rows past the end repeat the last one: all lanes take part in the exchange)
            const int h = min(h0 + 4 * i + (lane >> 4), end - 1);
            v[i] = reinterpret_cast<const uint4*>(x + t * x_stride + (long long)h * kHeadDim)[c];
        }
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int h = h0 + 4 * i + (lane >> 4);
            if (h0 + 4 * i >= end) break;
            float y[8];
            partners(v[i], out ? own : fixed, rot, y);
            if (out && h < end) store16<kOnce>(reinterpret_cast<uint4*>(out + t * out_stride + (long long)h * kHeadDim) + c, turned(v[i], y, own));
            if (lookup && h < end) store16<kOnce>(reinterpret_cast<uint4*>(lookup + ((long long)t * n_heads + h) * kHeadDim) + c, turned(v[i], y, fixed));
        }
    }
}

// One wave: `rows` rows of one token, which are its query heads, then its key heads, then its value heads.
template <bool kOnce>
__global__ __launch_bounds__(64 * kWaves) void paged_append_kernel(PagedKv cache, Rotation rot, const uint16_t* q, long long q_stride,
                                                                   uint16_t* q_out, const uint16_t* k, long long k_stride, const uint16_t* v,
                                                                   long long v_stride, int n_tokens, int n_q, int rows, int parts)
{
    __shared__ float2 tables[kWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15;
    const long long w = (long long)blockIdx.x * kWaves + wave;
    const int t = (int)(w / parts), part = (int)(w - (long long)t * parts);
    if (t >= n_tokens) return;
    const int b = sequence_of(cache.q_start, cache.n_seqs, t);
    if (b < 0) return;
    const int position = cache.kv_len[b] - (cache.q_start[b + 1] - t);
    const int page = page_of(cache.table + (long long)b * cache.table_stride, cache.table_stride, cache.n_pages, cache.page_shift, position);
    const bool stored = page >= 0;
    fill_table(tables[wave], rot, position);
    const Turn turn = load_turn(tables[wave], rot);
    const int total = n_q + 2 * cache.n_kv, end = min(total, (part + 1) * rows);
    for (int r0 = part * rows; r0 < end; r0 += 4 * kDeep) {
        uint4 x[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int r = min(r0 + 4 * i + (lane >> 4), end - 1), kv = r - n_q, h = kv < cache.n_kv ? kv : kv - cache.n_kv;
            const uint16_t* from = kv < 0 ? q + t * q_stride + (long long)r * kHeadDim
                                   : kv < cache.n_kv ? k + t * k_stride + (long long)h * kHeadDim : v + t * v_stride + (long long)h * kHeadDim;
            x[i] = reinterpret_cast<const uint4*>(from)[c];
        }
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int r = r0 + 4 * i + (lane >> 4), kv = r - n_q, h = kv < cache.n_kv ? kv : kv - cache.n_kv;
            if (r0 + 4 * i >= end) break;
            float y[8];
            partners(x[i], turn, rot, y);
            if (kv < cache.n_kv) x[i] = turned(x[i], y, turn);
            uint16_t* to;
            if (kv < 0) to = q_out + ((long long)t * n_q + r) * kHeadDim;
            else to = (kv < cache.n_kv ? cache.K : cache.V) + row_of(stored ? page : 0, h, cache.n_kv, cache.page_shift, position) * kHeadDim;
            if (r < end && (kv < 0 || stored)) store16<kOnce>(reinterpret_cast<uint4*>(to) + c, x[i]);
        }
    }
}

constexpr int kGatherTokens = 16;

// One workgroup: 16 positions of a sequence, all heads.
template <bool kOnce>
__global__ __launch_bounds__(64 * kWaves) void paged_gather_kernel(PagedKv cache, Rotation rot, int first, int n, int lookup_position, uint16_t* k,
                                                                   uint16_t* k_lookup, uint16_t* v, int blocks_per_seq)
{
    __shared__ float2 tables[kGatherTokens][64];
    const int b = blockIdx.x / blocks_per_seq, i0 = (blockIdx.x - b * blocks_per_seq) * kGatherTokens;
    const int i = i0 + (threadIdx.x >> 4), c = threadIdx.x & 15;
    const int position = first + i;
    int page = -1;
    if (i < n && position < cache.kv_len[b])
        page = page_of(cache.table + (long long)b * cache.table_stride, cache.table_stride, cache.n_pages, cache.page_shift, position);
    const bool held = page >= 0;
    if (k_lookup) {
        for (int e = threadIdx.x; e < kGatherTokens * 64; e += 64 * kWaves) {
            const int pair = e & 63;
            if (pair < (rot.rot_dim >> 1)) tables[e >> 6][pair] = cos_sin((double)lookup_position - (double)(first + i0 + (e >> 6)), rot.freqs[pair], 1.f);
        }
        __syncthreads();
    }
    Turn turn{};
    if (k_lookup) turn = load_turn(tables[threadIdx.x >> 4], rot);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int h0 = 0; h0 < cache.n_kv; h0 += 2) {
        uint4 x[2], z[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const long long from = row_of(held ? page : 0, min(h0 + e, cache.n_kv - 1), cache.n_kv, cache.page_shift, position) * kHeadDim;
            x[e] = z[e] = zero;
            if (held && (k || k_lookup)) x[e] = reinterpret_cast<const uint4*>(cache.K + from)[c];
            if (held && v) z[e] = reinterpret_cast<const uint4*>(cache.V + from)[c];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (h0 + e >= cache.n_kv) break;
            const long long to = (((long long)b * cache.n_kv + h0 + e) * n + i) * kHeadDim;
            if (k && i < n) store16<kOnce>(reinterpret_cast<uint4*>(k + to) + c, x[e]);
            if (k_lookup) {
                float y[8];
                partners(x[e], turn, rot, y);
                if (i < n) store16<kOnce>(reinterpret_cast<uint4*>(k_lookup + to) + c, turned(x[e], y, turn));
            }
            if (v && i < n) store16<kOnce>(reinterpret_cast<uint4*>(v + to) + c, z[e]);
        }
    }
}

}  // namespace

hipError_t launch_rotary(const Rotation& rot, const TokenRows& x, const int32_t* positions, int n_tokens, uint16_t* out, long long out_stride,
                         uint16_t* out_lookup, int lookup_position, hipStream_t s)
{
    if (n_tokens <= 0) return hipSuccess;
    const int rows = rows_of_a_wave(n_tokens, x.n_heads), parts = (x.n_heads + rows - 1) / rows;
    const long long blocks = ((long long)n_tokens * parts + kWaves - 1) / kWaves;
    const auto kernel = past_caches((long long)n_tokens * x.n_heads * ((out != nullptr) + (out_lookup != nullptr))) ? rotary_kernel<true> : rotary_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kWaves), 0, s, rot, x.p, x.stride, positions, out, out_stride, out_lookup,
                       lookup_position, n_tokens, x.n_heads, rows, parts);
    return hipGetLastError();
}

hipError_t launch_paged_append(const PagedKv& c, const Rotation& rot, const TokenRows& q, uint16_t* q_out, const TokenRows& k, const TokenRows& v,
                               int n_tokens, hipStream_t s)
{
    if (n_tokens <= 0 || c.n_seqs <= 0) return hipSuccess;
    const int total = q.n_heads + 2 * c.n_kv;
    const int rows = rows_of_a_wave(n_tokens, total), parts = (total + rows - 1) / rows;
    const long long blocks = ((long long)n_tokens * parts + kWaves - 1) / kWaves;
    const auto kernel = past_caches((long long)n_tokens * total) ? paged_append_kernel<true> : paged_append_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kWaves), 0, s, c, rot, q.p, q.stride, q_out, k.p, k.stride, v.p, v.stride,
                       n_tokens, q.n_heads, rows, parts);
    return hipGetLastError();
}

hipError_t launch_paged_gather(const PagedKv& c, const Rotation& rot, int first, int n, int lookup_position, uint16_t* k, uint16_t* k_lookup,
                               uint16_t* v, hipStream_t s)
{
    if (n <= 0 || c.n_seqs <= 0) return hipSuccess;
    const int per = (n + kGatherTokens - 1) / kGatherTokens;
    const auto kernel = past_caches((long long)c.n_seqs * c.n_kv * n * ((k != nullptr) + (k_lookup != nullptr) + (v != nullptr))) ? paged_gather_kernel<true> : paged_gather_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((long long)per * c.n_seqs)), dim3(64 * kWaves), 0, s, c, rot, first, n, lookup_position, k,
                       k_lookup, v, per);
    return hipGetLastError();
}

}  // namespace mp
