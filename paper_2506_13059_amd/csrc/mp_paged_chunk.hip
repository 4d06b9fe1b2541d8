// Attention of many new tokens over a paged cache, on the matrix cores, for gfx950.  (mp_paged_attn.hip says what is computed.)
//
// Eight waves of 32 query rows each work on one item (mp_paged_plan.h): 64 keys and values at a time are brought to LDS by all of them, through registers, a block
// ahead.  S^T = K Q^T and O^T += V^T P^T are v_mfma_f32_32x32x16_bf16, so a lane holds one query row in both (its column): its softmax
// needs no more of other lanes than one exchange of maxima, and the rows of S^T that it holds are, converted to bf16, what the second product takes from it,
// with the values' rows read (transposed by LDS) in the same order.
#include "mp_paged_plan.h"

namespace mp {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

constexpr int kWaves = 8, kKeys = 64, kRows = 32 * kWaves;
constexpr int kBlockBytes = kKeys * 256;
constexpr int kWorkgroups = 256;
constexpr int kPartFloats = kRows * kHeadDim + 2 * kRows;       // a part: weighted values as the lanes hold them, then maxima, then sums

template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_at(uint32_t at)
{
    return reinterpret_cast<__attribute__((address_space(3))) T*>((uintptr_t)at);
}
__device__ __forceinline__ uint32_t lds_offset(const void* p) { return (uint32_t)(uintptr_t)(lds_byte*)p; }

struct Softmax {
    f32x16 o[4];             // rows of block d: dims 32 d + 8 (i / 4) + 4 (lane / 32) + i % 4
    float m, l;              // of this lane's query row, m in powers of two; l of the keys that the lane has seen
};

__device__ __forceinline__ float over_halves_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float over_halves_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ void workgroup_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The lowest n of 64 bits.
__device__ __forceinline__ unsigned long long below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }

// The rows of a finished item.
__device__ __forceinline__ void store_rows(const PagedAttention& a, const Softmax& st, float l, int token, int head, bool there)
{
    const int half = (threadIdx.x & 63) >> 5;
    if (!there) return;
    const float f = l > 0.f ? 1.f / l : 0.f;
    const long long row = (long long)token * a.n_q_heads + head;
    unsigned char* out = reinterpret_cast<unsigned char*>(a.out) + row * 256 + half * 8;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (__bf16)(l > 0.f ? st.o[d][4 * j + e] * f : 0.f);
            *reinterpret_cast<bf16x4*>(out + d * 64 + j * 16) = w;
        }
    if (a.lse && half == 0) a.lse[row] = l > 0.f ? (st.m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -INFINITY;
}

__device__ __forceinline__ void store_part(float* part, const Softmax& st, float l)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    f32x4* o = reinterpret_cast<f32x4*>(part) + wave * 16 * 64 + lane;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[(4 * d + j) * 64] = f32x4{st.o[d][4 * j], st.o[d][4 * j + 1], st.o[d][4 * j + 2], st.o[d][4 * j + 3]};
    if (lane < 32) {
        part[kRows * kHeadDim + wave * 32 + lane] = st.m;
        part[kRows * kHeadDim + kRows + wave * 32 + lane] = l;
    }
}

__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_chunk_kernel(PagedAttention a, Tiling tl, float* parts, Cut* cuts)
{
    __shared__ __align__(256) unsigned char lds_k[2][kBlockBytes];
    __shared__ __align__(256) unsigned char lds_v[2][kBlockBytes];
    __shared__ __align__(8) unsigned char lds_valid[2][kWaves];      // keys that are there, a bit each
    __shared__ __align__(8) unsigned char lds_odd[2][kWaves];        // ... of an edge's block, whose values are not all finite
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
    const Line line = line_of(a, tl);
    const int share = share_of(line, blockIdx.x);
    if (share >= line.used) {
        if (threadIdx.x == 0) cuts[share].parts = 0;
        return;
    }
    const float scale = a.scale_log2e;
    const int G = tl.group;

    // LDS addresses: of the lane's row in the first 32 keys, chunk 2 ks + half; of its place in the first 16 values, dims 32 d; and of what it loads
    uint32_t k_at[8], v_at[4], k_to, v_to;
    {
        const int g = lane >> 4, c = lane & 15;
        k_to = lds_offset(lds_k) + (8 * wave + g) * 256 + ((c ^ (8 * (wave & 1) + g)) << 4);
        v_to = lds_offset(lds_v) + (8 * wave + g) * 256 + ((c ^ (g << 2)) << 4);
        const int row = lane & 31, v_row = 4 * half + ((lane & 15) >> 2);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) k_at[ks] = lds_offset(lds_k) + row * 256 + (((2 * ks + half) ^ (row & 15)) << 4);
#pragma unroll
        for (int d = 0; d < 4; ++d)
            v_at[d] = lds_offset(lds_v) + v_row * 256 + (((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ ((v_row & 3) << 2)) << 4) + (lane & 1) * 8;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) asm volatile("" : "+v"(k_at[ks]));
#pragma unroll
        for (int d = 0; d < 4; ++d) asm volatile("" : "+v"(v_at[d]));
    }

#ifdef PRIO
    if (wave < 4) __builtin_amdgcn_s_setprio(PRIO);
#endif
    long long x = share * line.share;
    const long long x_end = min(x + line.share, line.all);
    Cut cut{};
    while (x < x_end) {
        const int h = (int)(x / line.of_head);
        Item it;
        walk<true>(a, tl, (uint32_t)(x - (long long)h * line.of_head), &it);
        const int first = it.b0 + (int)((uint32_t)(x - (long long)h * line.of_head) - it.before);
        const int last = (int)min((long long)it.b1, first + (x_end - x));
        const bool whole = first == it.b0 && last == it.b1;

        // this lane's query row
        const int tile_rows = min(it.rows.n - it.tile * tl.tokens, tl.tokens) * G;
        const int r = min(wave * 32 + (lane & 31), tile_rows - 1);
        const int i = it.tile * tl.tokens + r / G, head = h * G + r % G;
        const int position = it.rows.base + i;
        const bool active = wave * 32 < tile_rows;
        const int pos_min = lane_value(position, 0), pos_max = lane_value(position, 31);
        bf16x8 q[8];
        {
            const uint4* from = reinterpret_cast<const uint4*>(a.q + (long long)(it.rows.q0 + i) * a.q_stride + (long long)head * kHeadDim);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) q[ks] = __builtin_bit_cast(bf16x8, from[2 * ks + half]);
        }

        // Loading: rows 8 wave + 4 e + lane / 16 of a block, chunk lane % 16 of 16 bytes.  In LDS chunk j of row k lies at j ^ k % 16 (keys) or j ^ 4 (k % 4)
        // (values): what the lanes of a read touch together lies in different banks.  Pages of eight rows or more hold all that a wave loads of a
        // block, so its address is a scalar.
        const int32_t* entries = a.c.table + (long long)it.b * a.c.table_stride;
        const int chunk = lane & 15;
        const int end = min(it.rows.base + it.rows.n, room_of(a));       // keys of the sequence
        const bool one_page = a.c.page_shift >= 3;
        // (entries are looked at a block after they were asked for: looked at at once, they made a wave wait for all loads before them)
        auto entry_at = [&](int block, int (&entry)[2]) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (e == 1 && one_page) break;
                const int key = block * kKeys + 8 * wave + (one_page ? 0 : 4 * e + (lane >> 4));
                entry[e] = entries[min(key, end - 1) >> a.c.page_shift];
            }
        };
        auto held = [&](int entry, int key) { return key < end && (uint32_t)entry < (uint32_t)a.c.n_pages; };
        const uint4 zero = make_uint4(0, 0, 0, 0);
        // One block's rows of this wave; what is not there keeps what the registers held.
        auto load = [&](int block, const int (&entry)[2], uint4 (&kw)[2], uint4 (&vw)[2]) {
            const int key = block * kKeys + 8 * wave;
            if (one_page) {
                const int page = __builtin_amdgcn_readfirstlane(entry[0]);
                if (held(page, key)) {
                    const long long at = row_of(page, h, a.c.n_kv, a.c.page_shift, key) * 16;
                    const uint4 *k = reinterpret_cast<const uint4*>(a.c.K) + at, *v = reinterpret_cast<const uint4*>(a.c.V) + at;
                    kw[0] = k[(uint32_t)lane];
                    kw[1] = k[(uint32_t)lane + 64];
                    vw[0] = v[(uint32_t)lane];
                    vw[1] = v[(uint32_t)lane + 64];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row_key = key + 4 * e + (lane >> 4);
                    if (held(entry[e], row_key)) {
                        const long long at = row_of(entry[e], h, a.c.n_kv, a.c.page_shift, row_key) * 16 + chunk;
                        kw[e] = reinterpret_cast<const uint4*>(a.c.K)[at];
                        vw[e] = reinterpret_cast<const uint4*>(a.c.V)[at];
                    }
                }
            }
        };
        // a block in which some row of the item sees a key that another one does not
        auto edge = [&](int block) {
            return block * kKeys + kKeys - 1 > it.rows.base + it.tile * tl.tokens ||
                   (a.window && block * kKeys <= it.rows.base + min(it.rows.n, (it.tile + 1) * tl.tokens) - 1 - a.window);
        };
        auto store = [&](int block, const int (&entry)[2], uint4 (&kw)[2], uint4 (&vw)[2]) {
            uint32_t bits = 0, odd = 0;
            if (one_page) {
                const int n = end - (block * kKeys + 8 * wave);
                if ((uint32_t)__builtin_amdgcn_readfirstlane(entry[0]) < (uint32_t)a.c.n_pages) bits = n >= 8 ? 255u : n > 0 ? (1u << n) - 1u : 0u;
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const unsigned long long in = __ballot(held(entry[e], block * kKeys + 8 * wave + 4 * e + (lane >> 4)));
#pragma unroll
                    for (int k = 0; k < 4; ++k) bits |= (uint32_t)(in >> (16 * k) & 1) << (4 * e + k);
                }
            }
            if (bits != 255u) {              // (rows without a key are zero: a probability of zero meets them)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (!(bits >> (4 * e + (lane >> 4)) & 1)) vw[e] = zero;
            }
            if (edge(block)) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t u[4] = {vw[e].x, vw[e].y, vw[e].z, vw[e].w};
                    bool off_range = false;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const bool lo = (u[k] & 0x7f80u) == 0x7f80u, hi = (u[k] & 0x7f800000u) == 0x7f800000u;
                        off_range |= lo | hi;
                        u[k] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
                    }
                    vw[e] = make_uint4(u[0], u[1], u[2], u[3]);
                    const unsigned long long in = __ballot(off_range);
#pragma unroll
                    for (int k = 0; k < 4; ++k) odd |= (uint32_t)((in >> (16 * k) & 0xffff) != 0) << (4 * e + k);
                }
            }
            if (lane == 0) {
                lds_valid[block & 1][wave] = (unsigned char)bits;
                lds_odd[block & 1][wave] = (unsigned char)odd;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                *lds_at<u32x4>((e ? k_to ^ 64u : k_to) + (block & 1) * kBlockBytes + e * 1024) = u32x4{kw[e].x, kw[e].y, kw[e].z, kw[e].w};
                *lds_at<u32x4>(v_to + (block & 1) * kBlockBytes + e * 1024) = u32x4{vw[e].x, vw[e].y, vw[e].z, vw[e].w};
            }
        };

        // (reads kAhead ahead of the products that take them: left alone, the compiler has each product wait for a read of its own)
        auto scores = [&](int block, f32x16 (&s)[2]) {
#ifndef KA
#define KA 4
#endif
            constexpr int kAhead = KA;
            bf16x8 k[kAhead];
            auto read = [&](int i) { k[i % kAhead] = *lds_at<bf16x8>(k_at[i >> 1] + (block & 1) * kBlockBytes + (i & 1) * 32 * 256); };
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[t][j] = 0.f;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) read(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[i % kAhead], q[i >> 1], s[i & 1], 0, 0, 0);
                if (i + kAhead < 16) read(i + kAhead);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // 16 keys from 16 s and 32 dims from 32 d of the values, transposed: keys 4 half .. + 3, then 8 + 4 half .. + 3, of the lane's dim
        auto values = [&](int block, int s, int d) {
            auto* p = lds_at<s16x4>(v_at[d] + (block & 1) * kBlockBytes + s * 16 * 256);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(v_at[d] + (block & 1) * kBlockBytes + s * 16 * 256 + 8 * 256));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };

        Softmax st;
        st.m = -INFINITY;
        st.l = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int j = 0; j < 16; ++j) st.o[d][j] = 0.f;

        uint4 kw[2] = {zero, zero}, vw[2] = {zero, zero};
        if (end > 0) {
            int now[2], next[2];
            entry_at(first, now);
            entry_at(first + 1, next);
            load(first, now, kw, vw);
            workgroup_sync();                              // (the item before is done with LDS)
            store(first, now, kw, vw);
            load(first + 1, next, kw, vw);
            workgroup_sync();
            for (int t = first; t < last; ++t) {
            int far[2];
            entry_at(t + 2, far);
            if (active && t * kKeys <= pos_max) {
                f32x16 s[2];
                scores(t, s);
                const unsigned long long valid = *reinterpret_cast<const unsigned long long*>(lds_valid[t & 1]);
                const uint32_t valid_lo = __builtin_amdgcn_readfirstlane((uint32_t)valid), valid_hi = __builtin_amdgcn_readfirstlane((uint32_t)(valid >> 32));
                const bool masked = (valid_lo & valid_hi) != 0xffffffffu || t * kKeys + kKeys - 1 > pos_min || (a.window && t * kKeys <= pos_max - a.window);
                if (masked) {
                    // keys (from, upto] of the block, those that are there; bit k of `see` for key 4 half + k
                    const int upto = position - t * kKeys, from = a.window ? upto - a.window : -1;
                    const unsigned long long see = (valid & below(upto + 1) & ~below(from + 1)) >> (4 * half);
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt) {
                        const uint32_t in = (uint32_t)(see >> (32 * tt));
#pragma unroll
                        for (int j = 0; j < 16; ++j) s[tt][j] = in & (1u << (8 * (j >> 2) + (j & 3))) ? s[tt][j] : -INFINITY;
                    }
                }
                float mx = s[0][0];
#pragma unroll
                for (int j = 1; j < 16; ++j) mx = fmaxf(mx, s[0][j]);
#pragma unroll
                for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[1][j]);
                mx = over_halves_max(mx) * scale;
                // The maximum in use may be up to 2^8 behind: sums in fp32 and products of bf16 have room for it, and it is soon never moved.
                if (__any(mx > st.m + 8.f)) {
                    const float m = fmaxf(st.m, mx), f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - m);
                    st.m = m;
                    st.l *= f;
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int j = 0; j < 16; ++j) st.o[d][j] *= f;
                }
                const float m = st.m == -INFINITY ? 0.f : st.m;
                // Probabilities of 16 keys at a time, two elements behind each product of the 16 keys before; values are read two products ahead.
                bf16x8 p[4];
                auto probabilities = [&](int k, int e) {
#pragma unroll
                    for (int j = e; j < e + 2; ++j) {
                        const float x = __builtin_amdgcn_exp2f(fmaf(s[k >> 1][8 * (k & 1) + j], scale, -m));
                        st.l += x;
                        p[k][j] = (__bf16)x;
                    }
                };
#ifndef VA
#define VA 2
#endif
                constexpr int kAhead = VA;
                s16x8 v[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) v[i] = values(t, 0, i);
#pragma unroll
                for (int e = 0; e < 8; e += 2) probabilities(0, e);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    st.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[i % kAhead]), p[i >> 2], st.o[i & 3], 0, 0, 0);
                    if (i + kAhead < 16) v[i % kAhead] = values(t, (i + kAhead) >> 2, (i + kAhead) & 3);
                    if (i < 12) probabilities((i >> 2) + 1, 2 * (i & 3));
#ifndef NOSB
                    __builtin_amdgcn_sched_barrier(0);
#endif
                }
                // Values that are not finite have been taken out of an edge's block, lest they meet the zero of a row that does not see them: they are
                // added to the rows that do.
                if (edge(t)) {
                    const unsigned long long flags = *reinterpret_cast<const unsigned long long*>(lds_odd[t & 1]);
                    unsigned long long odd = (unsigned long long)__builtin_amdgcn_readfirstlane((uint32_t)(flags >> 32)) << 32 | __builtin_amdgcn_readfirstlane((uint32_t)flags);
                    for (; odd; odd &= odd - 1) {
                        const int key = t * kKeys + __ffsll((long long)odd) - 1;
                        const int page = __builtin_amdgcn_readfirstlane(page_of(entries, a.c.table_stride, a.c.n_pages, a.c.page_shift, key));
                        const bool sees = key <= position && !(a.window && key <= position - a.window);
                        const uint2* from = reinterpret_cast<const uint2*>(a.c.V + row_of(page, h, a.c.n_kv, a.c.page_shift, key) * kHeadDim);
#pragma unroll
                        for (int d = 0; d < 4; ++d)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint2 w = from[8 * d + 2 * j + half];
                                const uint32_t u[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (sees && (u[e] & 0x7f800000u) == 0x7f800000u) st.o[d][4 * j + e] += __uint_as_float(u[e]);
                            }
                    }
                }
            }
            store(t + 1, next, kw, vw);
            next[0] = far[0];
            next[1] = far[1];
            load(t + 2, next, kw, vw);
            workgroup_sync();
            }
        }

        const float l = over_halves_sum(st.l);
        if (whole) store_rows(a, st, l, it.rows.q0 + i, head, wave * 32 + (lane & 31) < tile_rows);
        else {
            store_part(parts + (2ll * share + (x > share * line.share ? 1 : 0)) * kPartFloats, st, l);
            if (last < it.b1) cut = cut_of(it, tl, line, share, h);
        }
        x += last - first;
    }
    if (threadIdx.x == 0) cuts[share] = cut;
}

// One wave a cut and 32 rows.
__global__ __launch_bounds__(64) void paged_chunk_merge_kernel(PagedAttention a, int group, const float* parts, const Cut* cuts)
{
    const int share = blockIdx.x >> 3, wave = blockIdx.x & 7, lane = threadIdx.x;
    const Cut c = cuts[share];
    if (c.parts == 0 || wave * 32 >= c.rows) return;
    auto part = [&](int g) { return parts + (2ll * (share + g) + (g == 0 ? c.slot : 0)) * kPartFloats; };
    const int at_m = kRows * kHeadDim + wave * 32 + (lane & 31);
    Softmax st;
    st.m = -INFINITY;
    for (int g = 0; g < c.parts; ++g) st.m = fmaxf(st.m, part(g)[at_m]);
    float l = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int j = 0; j < 16; ++j) st.o[d][j] = 0.f;
    for (int g = 0; g < c.parts; ++g) {
        const float* p = part(g);
        const float m = p[at_m];
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - st.m);
        l = fmaf(p[at_m + kRows], f, l);
        const f32x4* o = reinterpret_cast<const f32x4*>(p) + wave * 16 * 64 + lane;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 w = o[(4 * d + j) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) st.o[d][4 * j + e] = fmaf(w[e], f, st.o[d][4 * j + e]);
            }
    }
    const int r = min(wave * 32 + (lane & 31), c.rows - 1);
    store_rows(a, st, l, c.q0 + r / group, c.head * group + r % group, wave * 32 + (lane & 31) < c.rows);
}

Tiling chunk_tiling(int group, int over)
{
    Tiling t;
    t.group = group;
    t.tokens = kRows / group;
    t.over = over;
    t.most = 0x7fffffff;
    t.unit = kKeys;
    t.least = 4;
    t.workgroups = kWorkgroups;
    return t;
}

constexpr size_t kCutFloats = sizeof(Cut) / sizeof(float) * kWorkgroups;

}  // namespace

size_t paged_chunk_floats() { return (size_t)2 * kWorkgroups * kPartFloats + kCutFloats; }

hipError_t launch_paged_chunks(const PagedAttention& a, int over, float* room, hipStream_t s)
{
    const Tiling tl = chunk_tiling(a.n_q_heads / a.c.n_kv, over);
    Cut* cuts = reinterpret_cast<Cut*>(room);
    float* parts = room + kCutFloats;
    hipLaunchKernelGGL(paged_chunk_kernel, dim3(kWorkgroups), dim3(64 * kWaves), 0, s, a, tl, parts, cuts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_chunk_merge_kernel, dim3(8 * kWorkgroups), dim3(64), 0, s, a, tl.group, (const float*)parts, (const Cut*)cuts);
    return hipGetLastError();
}

}  // namespace mp
