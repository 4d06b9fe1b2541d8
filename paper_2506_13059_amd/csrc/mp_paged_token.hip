// Attention of one or a few new tokens over a paged cache, on the matrix cores, for gfx950.  (mp_paged_attn.hip says what is computed.)
//
// Up to 16 query rows (new tokens times the heads of a group) meet every key of their sequence once: bound by memory.  A wave streams tiles of
// 32 keys and values straight to LDS (global_load_lds, 16 bytes a lane, four rows an instruction) into a ring of two tiles, three of four
// 8 KiB pieces on their way while one is used.  S^T = K Q^T is eight v_mfma_f32_16x16x32_bf16 and O^T += V^T P^T as many: a lane holds one
// query row (its column) in both, and what it holds of S^T is what the second product takes of it.  Four waves with runs of tiles of their own make a workgroup,
// whose sums meet in LDS; workgroups have equal shares of all sequences' keys (mp_paged_plan.h).
#include <type_traits>

#include "mp_paged_plan.h"

namespace mp {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

constexpr int kWaves = 4, kTile = 32, kRows = 16;
constexpr int kPiece = kTile * 256, kSlot = 2 * kPiece, kRing = 2 * kSlot;
constexpr int kWorkgroups = 256;
constexpr int kPartFloats = kRows * kHeadDim + 2 * kRows;       // a part: weighted values as the lanes hold them, then maxima, then sums
constexpr size_t kCutFloats = sizeof(Cut) / sizeof(float) * kWorkgroups;

__device__ __forceinline__ void load_to_lds(const void* src, uint32_t lds_off)
{
    // (the LDS address is the same in all lanes; lane i's bytes go to it + 16 i)
    auto* dst = reinterpret_cast<__attribute__((address_space(3))) uint32_t*>((uintptr_t)lds_off);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src, dst, 16, 0, 2);      // (2: non-temporal)
}
template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

struct State {
    f32x4 o[8];              // of this lane's query row: dims 16 d + 4 (lane / 16) + i
    float m, l;              // m in powers of two; l of the keys that the lane has seen
};

struct Source {
    const unsigned char *K, *V;      // of head 0 of page 0
    const int32_t* entries;
    int stride, n_pages, shift, n_kv, h, end;
};

// Tiles [t0, t1) of 32 keys through one wave; `ring`: LDS offset of its ring.
__device__ __forceinline__ void stream(State& st, const Source& c, const bf16x8 (&q)[4], int t0, int t1, uint32_t ring, int position, int pos_min, int pos_max,
                                       int window, float scale)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    // LDS: chunk j (16 bytes) of key r lies at j ^ r % 16, of value r at j ^ 2 (r % 8): the lanes of a read touch different banks
    const uint32_t k_at = ring + (uint32_t)(col * 256 + ((g ^ col) << 4));                                  // ^ 64 ks
    const int vr = 4 * g + (col >> 2);
    const uint32_t v_at = ring + kPiece + (uint32_t)(vr * 256 + ((((col & 3) >> 1) ^ ((vr & 7) << 1)) << 4) + (col & 1) * 8);      // ^ 32 d

    // (entries are looked at two tiles after they were asked for: looked at at once, they made the wave wait for all loads before them)
    auto entry_at = [&](int t) { return c.entries[min(t * kTile + (lane & 31), c.end - 1) >> c.shift]; };      // of key 32 t + lane % 32
    auto held = [&](int t, int entry) { return (uint32_t)__ballot(t * kTile + (lane & 31) < c.end && (uint32_t)entry < (uint32_t)c.n_pages); };
    long long off[8];
    auto offsets = [&](int t, int entry, uint32_t valid) {    // bytes, of rows 4 i + g; those that are not there: somewhere in page 0
        if (c.shift >= 5) {                  // (the tile lies in one page)
            const int page = valid ? __builtin_amdgcn_readfirstlane(entry) : 0;
            const long long at = row_of(page, c.h, c.n_kv, c.shift, t * kTile) * 256 + g * 256;
#pragma unroll
            for (int i = 0; i < 8; ++i) off[i] = at + i * 1024;
        } else {
            const int mine = (valid >> (lane & 31) & 1) ? entry : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) off[i] = row_of(__shfl(mine, 4 * i + g, 64), c.h, c.n_kv, c.shift, t * kTile + 4 * i + g) * 256;
        }
    };
    auto load_keys = [&](int t) {
#pragma unroll
        for (int i = 0; i < 8; ++i) load_to_lds(c.K + off[i] + ((col ^ ((4 * i + g) & 15)) << 4), ring + (uint32_t)((t & 1) * kSlot + i * 1024));
    };
    auto load_values = [&](int t) {
#pragma unroll
        for (int i = 0; i < 8; ++i) load_to_lds(c.V + off[i] + ((col ^ (((4 * i + g) & 7) << 1)) << 4), ring + (uint32_t)((t & 1) * kSlot + kPiece + i * 1024));
    };

    // Loads come back in order: K V K V ..., eight instructions a piece, and one for the pages of a tile four ahead now and then; "at most as many on their
    // way as the pieces behind it have" means that a piece is there.  Nothing is asked for past the end.
    int entries[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) entries[i] = entry_at(t0 + i);
    uint32_t valid0 = held(t0, entries[0]), valid1 = 0;
    offsets(t0, entries[0], valid0);
    load_keys(t0);
    load_values(t0);
    if (t0 + 1 < t1) {
        valid1 = held(t0 + 1, entries[1]);
        offsets(t0 + 1, entries[1], valid1);
        load_keys(t0 + 1);
        load_values(t0 + 1);
    }
    auto tile = [&](int t, auto ahead) {
        constexpr int kAhead = decltype(ahead)::value;               // tiles behind this one (2: two or more)
        const uint32_t slot = (uint32_t)((t & 1) * kSlot);
        const uint32_t valid = valid0;
        valid0 = valid1;
        wait_vm<kAhead == 0 ? 8 : 24>();
        bf16x8 k[8];
        const uint32_t a0 = k_at + slot, a1 = (k_at ^ 64u) + slot, a2 = (k_at ^ 128u) + slot, a3 = (k_at ^ 192u) + slot;
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
                     "ds_read_b128 %4, %8 offset:4096\n\tds_read_b128 %5, %9 offset:4096\n\tds_read_b128 %6, %10 offset:4096\n\t"
                     "ds_read_b128 %7, %11 offset:4096\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3]), "=&v"(k[4]), "=&v"(k[5]), "=&v"(k[6]), "=&v"(k[7])
                     : "v"(a0), "v"(a1), "v"(a2), "v"(a3)
                     : "memory");
        if constexpr (kAhead == 2) {
            valid1 = held(t + 2, entries[2]);
            offsets(t + 2, entries[2], valid1);
            load_keys(t + 2);
            entries[2] = entries[3];
            entries[3] = entry_at(t + 4);
        }
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[ks], q[ks], s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[4 + ks], q[ks], s1, 0, 0, 0);
        }
        float s[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[i] = s0[i];
            s[4 + i] = s1[i];
        }
        // a tile in which some row sees a key that another one does not
        const bool edge = t * kTile + kTile - 1 > pos_min || (window && t * kTile <= pos_max - window);
        if (valid != 0xffffffffu || edge) {
            const int upto = position - t * kTile, from = window ? upto - window : -1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = 16 * (i >> 2) + 4 * g + (i & 3);
                s[i] = (valid >> key & 1) && key <= upto && key > from ? s[i] : -INFINITY;
            }
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7]))) * scale;
        if (__any(mx > st.m)) {              // (the running maximum settles after a few tiles)
            mx = fmaxf(mx, st.m);
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - mx);
            st.m = mx;
            st.l *= f;
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.o[d][i] *= f;
        }
        const float m = st.m == -INFINITY ? 0.f : st.m;
        bf16x8 p;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = __builtin_amdgcn_exp2f(fmaf(s[i], scale, -m));
            st.l += e;
            p[i] = (__bf16)e;
        }
        wait_vm<kAhead == 2 ? 24 : 16 * kAhead>();
        uint32_t odd = 0;
        if (valid != 0xffffffffu || edge) {
            // Rows without a key are zeroed, and so are values of an edge's tile that are not finite, lest they meet the zero of a row that does not see them.
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                auto* at = reinterpret_cast<__attribute__((address_space(3))) u32x4*>((uintptr_t)(ring + slot + kPiece + (uint32_t)(i * 1024 + lane * 16)));
                u32x4 w = *at;
                bool off_range = false;
                if (!(valid >> (4 * i + g) & 1)) {
                    w = u32x4{0u, 0u, 0u, 0u};
                } else if (edge) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool lo = (w[e] & 0x7f80u) == 0x7f80u, hi = (w[e] & 0x7f800000u) == 0x7f800000u;
                        off_range |= lo | hi;
                        w[e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
                    }
                }
                *at = w;
                const unsigned long long in = __ballot(off_range);
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= (uint32_t)((in >> (16 * e) & 0xffff) != 0) << (4 * i + e);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
#pragma unroll
        for (int d4 = 0; d4 < 2; ++d4) {
            s16x4 v[8];
            const uint32_t b0 = (v_at ^ (128u * d4)) + slot, b1 = (v_at ^ (128u * d4 + 32u)) + slot, b2 = (v_at ^ (128u * d4 + 64u)) + slot,
                           b3 = (v_at ^ (128u * d4 + 96u)) + slot;
            asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:4096\n\tds_read_b64_tr_b16 %2, %9\n\t"
                         "ds_read_b64_tr_b16 %3, %9 offset:4096\n\tds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:4096\n\t"
                         "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:4096\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
                         : "v"(b0), "v"(b1), "v"(b2), "v"(b3)
                         : "memory");
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const auto a = __builtin_shufflevector(v[2 * d], v[2 * d + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                st.o[4 * d4 + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), p, st.o[4 * d4 + d], 0, 0, 0);
            }
        }
        if constexpr (kAhead == 2) load_values(t + 2);
        // the values taken out are added to the rows that see them
        for (; odd; odd &= odd - 1) {
            const int key = t * kTile + __builtin_ctz(odd);
            const int page = page_of(c.entries, c.stride, c.n_pages, c.shift, key);
            const bool sees = key <= position && !(window && key <= position - window);
            const uint2* from = reinterpret_cast<const uint2*>(c.V + row_of(max(page, 0), c.h, c.n_kv, c.shift, key) * 256);
#pragma unroll
            for (int d = 0; d < 8; ++d) {
                const uint2 w = from[4 * d + g];
                const uint32_t u[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (sees && (u[e] & 0x7f800000u) == 0x7f800000u) st.o[d][e] += __uint_as_float(u[e]);
            }
        }
    };
    int t = t0;
    for (; t + 2 < t1; ++t) tile(t, std::integral_constant<int, 2>{});
    if (t + 1 < t1) tile(t++, std::integral_constant<int, 1>{});
    tile(t, std::integral_constant<int, 0>{});
}

__device__ __forceinline__ void store_row(const PagedAttention& a, int token, int head, const f32x4& o, float m, float l, int d, int g)
{
    const float f = l > 0.f ? 1.f / l : 0.f;
    const long long row = (long long)token * a.n_q_heads + head;
    bf16x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (__bf16)(l > 0.f ? o[e] * f : 0.f);
    *reinterpret_cast<bf16x4*>(a.out + row * kHeadDim + 16 * d + 4 * g) = w;
    if (a.lse && d == 0 && g == 0) a.lse[row] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -INFINITY;
}

__global__ __launch_bounds__(64 * kWaves, 1) void paged_token_kernel(PagedAttention a, Tiling tl, float* parts, Cut* cuts)
{
    __shared__ __align__(256) unsigned char lds[kWaves * kRing];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const Line line = line_of(a, tl);
    const int share = share_of(line, blockIdx.x);
    if (share >= line.used) {
        if (threadIdx.x == 0) cuts[share].parts = 0;
        return;
    }
    const uint32_t ring = (uint32_t)(uintptr_t)(lds_byte*)lds + (uint32_t)(wave * kRing);
    const int G = tl.group;
    long long x = share * line.share;
    const long long x_end = min(x + line.share, line.all);
    Cut cut{};
    Segment seg;
    for (bool known = false; x < x_end; known = true, x = seg.next) {
        segment_at(a, tl, line, x, x_end, known, &seg);
        const Item& it = seg.it;
        const int h = seg.h, first = seg.first, last = seg.last;
        if (first == last) continue;                       // (the share ends among the places in front)
        const bool whole = first == it.b0 && last == it.b1;
        const int tile_rows = min(it.rows.n - it.tile * tl.tokens, tl.tokens) * G;
        const int r = min(col, tile_rows - 1);
        const int i = it.tile * tl.tokens + r / G, head = h * G + r % G, position = it.rows.base + i;
        const int pos_min = lane_value(position, 0), pos_max = lane_value(position, 15);
        bf16x8 q[4];
        {
            const uint4* from = reinterpret_cast<const uint4*>(a.q + (long long)(it.rows.q0 + i) * a.q_stride + (long long)head * kHeadDim);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) q[ks] = __builtin_bit_cast(bf16x8, from[4 * ks + g]);
        }
        Source c;
        c.K = reinterpret_cast<const unsigned char*>(a.c.K);
        c.V = reinterpret_cast<const unsigned char*>(a.c.V);
        c.entries = a.c.table + (long long)it.b * a.c.table_stride;
        c.stride = a.c.table_stride;
        c.n_pages = a.c.n_pages;
        c.shift = a.c.page_shift;
        c.n_kv = a.c.n_kv;
        c.h = h;
        c.end = min(pos_max + 1, room_of(a));
        // the wave's tiles: a quarter of the share's
        const int t0 = first * kWaves + wave * (last - first), t1 = min(t0 + (last - first), c.end > 0 ? (c.end - 1) / kTile + 1 : 0);
        State st;
        st.m = -INFINITY;
        st.l = 0.f;
#pragma unroll
        for (int d = 0; d < 8; ++d) st.o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (t0 < t1) stream(st, c, q, t0, t1, ring, position, pos_min, pos_max, a.window, a.scale_log2e);

        // The waves' sums meet.
        float l = st.l;
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        __syncthreads();
        f32x4* sm_o = reinterpret_cast<f32x4*>(lds);                            // [kWaves][8][64]
        float* sm_m = reinterpret_cast<float*>(lds + kWaves * 8 * 64 * 16);     // [kWaves][16], then sums
        float* sm_l = sm_m + kWaves * 16;
#pragma unroll
        for (int d = 0; d < 8; ++d) sm_o[(wave * 8 + d) * 64 + lane] = st.o[d];
        if (lane < 16) {
            sm_m[wave * 16 + lane] = st.m;
            sm_l[wave * 16 + lane] = l;
        }
        __syncthreads();
        float M = -INFINITY, L = 0.f, f[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm_m[w * 16 + col]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            f[w] = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm_m[w * 16 + col] - M);
            L = fmaf(sm_l[w * 16 + col], f[w], L);
        }
        float* part = parts + (2ll * share + slot_of(blocks_from(it, tl, line, h), share, line.share)) * kPartFloats;
#pragma unroll
        for (int dd = 0; dd < 2; ++dd) {
            const int d = wave + 4 * dd;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const f32x4 y = sm_o[(w * 8 + d) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], f[w], o[e]);
            }
            if (whole) {
                if (col < tile_rows) store_row(a, it.rows.q0 + i, head, o, M, L, d, g);
            } else {
                reinterpret_cast<f32x4*>(part)[d * 64 + lane] = o;
            }
        }
        if (!whole) {
            if (threadIdx.x < 16) {
                part[kRows * kHeadDim + lane] = M;
                part[kRows * kHeadDim + kRows + lane] = L;
            }
            if (last < it.b1) cut = cut_of(it, tl, line, share, h);
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) cuts[share] = cut;
}

// One workgroup a cut and 16 dims: its waves take parts in turn.
__global__ __launch_bounds__(256) void paged_token_merge_kernel(PagedAttention a, int group, const float* parts, const Cut* cuts)
{
    __shared__ float sm[2][16][16];
    __shared__ f32x4 sm_o[4][64];
    const int share = blockIdx.x >> 3, d = blockIdx.x & 7, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const Cut c = cuts[share];
    if (c.parts == 0) return;
    auto part = [&](int i) { return parts + (2ll * (share + i) + (i == 0 ? c.slot : 0)) * kPartFloats; };
    float m = -INFINITY;
    for (int i = threadIdx.x >> 4; i < c.parts; i += 16) m = fmaxf(m, part(i)[kRows * kHeadDim + col]);
    sm[0][threadIdx.x >> 4][col] = m;
    __syncthreads();
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) M = fmaxf(M, sm[0][i][col]);
    const float Ms = M == -INFINITY ? 0.f : M;
    float l = 0.f;
    for (int i = threadIdx.x >> 4; i < c.parts; i += 16)
        l = fmaf(part(i)[kRows * kHeadDim + kRows + col], __builtin_amdgcn_exp2f(part(i)[kRows * kHeadDim + col] - Ms), l);
    sm[1][threadIdx.x >> 4][col] = l;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = wave; i < c.parts; i += 4) {
        const float* p = part(i);
        const float f = __builtin_amdgcn_exp2f(p[kRows * kHeadDim + col] - Ms);
        const f32x4 y = reinterpret_cast<const f32x4*>(p)[d * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], f, o[e]);
    }
    sm_o[wave][lane] = o;
    __syncthreads();
    if (wave != 0) return;
    float L = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) L += sm[1][i][col];
#pragma unroll
    for (int w = 1; w < 4; ++w) o += sm_o[w][lane];
    if (col < c.rows) store_row(a, c.q0 + col / group, c.head * group + col % group, o, M, L, d, g);
}

}  // namespace

size_t paged_token_floats() { return (size_t)2 * kWorkgroups * kPartFloats + kCutFloats; }

hipError_t launch_paged_tokens(const PagedAttention& a, float* room, hipStream_t s)
{
    Tiling tl;
    tl.group = a.n_q_heads / a.c.n_kv;
    tl.tokens = kRows / tl.group;
    tl.over = 0;
    tl.most = kPagedTokenRows;
    tl.unit = kWaves * kTile;
    tl.ahead = 2;
    tl.least = 1 + tl.ahead;
    tl.workgroups = kWorkgroups;
    Cut* cuts = reinterpret_cast<Cut*>(room);
    float* parts = room + kCutFloats;
    hipLaunchKernelGGL(paged_token_kernel, dim3(kWorkgroups), dim3(64 * kWaves), 0, s, a, tl, parts, cuts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_token_merge_kernel, dim3(8 * kWorkgroups), dim3(256), 0, s, a, tl.group, (const float*)parts, (const Cut*)cuts);
    return hipGetLastError();
}

}  // namespace mp
