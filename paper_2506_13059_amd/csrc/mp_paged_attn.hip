// Attention of new tokens over a paged cache, for gfx950.
//
// Query row i of a sequence with n new tokens and len keys (the new ones among them) stands at position p = len - n + i and attends the
// keys j with p - window < j <= p (window 0: all up to p) whose page is there:
//     o = sum_j e^(s q.k_j - m) v_j / l,   l = sum_j e^(s q.k_j - m),   lse = m + ln l,
// a row without such a key gives zeros and -inf.
#include "mp_device.h"
#include "mp_paged.h"

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

// One wave a query row and head: four keys at a time, 16 lanes of eight dims each.
__global__ __launch_bounds__(256) void paged_row_kernel(PagedAttention a)
{
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(w / a.n_q_heads), hq = (int)(w - (long long)t * a.n_q_heads);
    if (t >= a.n_tokens) return;
    const int b = sequence_of(a.c.q_start, a.c.n_seqs, t);
    if (b < 0 || t - a.c.q_start[b] >= a.max_new) return;
    const int len = a.c.kv_len[b], p = len - (a.c.q_start[b + 1] - t);
    const int h = hq / (a.n_q_heads / a.c.n_kv);
    float q[8], acc[8], m = -INFINITY, l = 0.f;
    const uint4 qw = reinterpret_cast<const uint4*>(a.q + t * a.q_stride + (long long)hq * kHeadDim)[c];
    const uint32_t qu[4] = {qw.x, qw.y, qw.z, qw.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = i & 1 ? bf16hi_to_f32(qu[i >> 1]) : bf16lo_to_f32(qu[i >> 1]);
        acc[i] = 0.f;
    }
    const long long room = (long long)a.c.table_stride << a.c.page_shift;
    const int end = (int)min((long long)p + 1, room), begin = a.window ? max(0, p - a.window + 1) : 0;
    for (int j0 = begin; j0 < end; j0 += 4) {
        const int j = j0 + g;
        int page = -1;
        if (j < end) page = page_of(a.c.table + (long long)b * a.c.table_stride, a.c.table_stride, a.c.n_pages, a.c.page_shift, j);
        const bool there = page >= 0;
        float s = 0.f, vv[8] = {};
        if (there) {
            const long long at = row_of(page, h, a.c.n_kv, a.c.page_shift, j) * kHeadDim;
            const uint4 kw = reinterpret_cast<const uint4*>(a.c.K + at)[c], vw = reinterpret_cast<const uint4*>(a.c.V + at)[c];
            const uint32_t ku[4] = {kw.x, kw.y, kw.z, kw.w}, vu[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s = fmaf(q[2 * i], bf16lo_to_f32(ku[i]), s);
                s = fmaf(q[2 * i + 1], bf16hi_to_f32(ku[i]), s);
                vv[2 * i] = bf16lo_to_f32(vu[i]);
                vv[2 * i + 1] = bf16hi_to_f32(vu[i]);
            }
        }
        s = row_sum_f32(s) * a.scale_log2e;
        if (there) {
            const float mn = fmaxf(m, s), f = __builtin_amdgcn_exp2f(m - mn), e = __builtin_amdgcn_exp2f(s - mn);
            m = mn;
            l = fmaf(l, f, e);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = fmaf(acc[i], f, e * vv[i]);
        }
    }
    float M = fmaxf(m, __shfl_xor(m, 16, 64));
    M = fmaxf(M, __shfl_xor(M, 32, 64));
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
    l *= f;
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    uint32_t o[4];
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float x = f == 0.f ? 0.f : acc[i] * f;
        x += __shfl_xor(x, 16, 64);
        x += __shfl_xor(x, 32, 64);
        r[i] = l > 0.f ? x / l : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (uint32_t)f32_to_bf16_rne(r[2 * i]) | ((uint32_t)f32_to_bf16_rne(r[2 * i + 1]) << 16);
    if (g == 0) reinterpret_cast<uint4*>(a.out + ((long long)t * a.n_q_heads + hq) * kHeadDim)[c] = make_uint4(o[0], o[1], o[2], o[3]);
    if (a.lse && lane == 0) a.lse[(long long)t * a.n_q_heads + hq] = l > 0.f ? (M + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -INFINITY;
}

}  // namespace

size_t paged_partial_floats(int, int, int, int, int) { return 0; }

hipError_t launch_paged_attention(const PagedAttention& a, hipStream_t s)
{
    if (a.n_tokens <= 0 || a.c.n_seqs <= 0) return hipSuccess;
    const long long blocks = ((long long)a.n_tokens * a.n_q_heads + 3) / 4;
    hipLaunchKernelGGL(paged_row_kernel, dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace mp
