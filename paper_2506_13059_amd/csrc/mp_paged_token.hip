// Attention of one or a few new tokens over a paged cache, on the matrix cores, for gfx950.  (mp_paged_attn.hip says what is computed.)
//
// Up to 64 query rows (new tokens times the heads of a group; kGroups times 16) meet every key of their sequence once: bound by memory.  A wave streams tiles of
// 32 keys and values straight to LDS (global_load_lds, 16 bytes a lane, four rows an instruction) into a ring of two tiles, three of four
// 8 KiB pieces on their way while one is used.  For 16 rows, S^T = K Q^T is eight v_mfma_f32_16x16x32_bf16 and O^T += V^T P^T as many: a lane holds one
// query row of each 16 (its column) in both, and what it holds of S^T is what the second product takes of it.  Four waves with runs of tiles of their own make a workgroup,
// whose sums meet in LDS; workgroups have equal shares of all sequences' keys (mp_paged_plan.h), one a compute unit.
//
// One token each of 16 sequences of up to 128K keys, 8 KV heads of four: 585 to 593 us, 6.6 to 6.7 TB/s; 40 rows each of 8 sequences of up to 30K: 95 us, 5.1 TB/s; one
// token over 4096 keys: 8.0 us and 4.9 for the merge, trips to memory one behind the other (lengths, page, keys, parts) and two launches.
#include <type_traits>

#include "mp_paged_tile.h"

namespace mp {

namespace {

constexpr int kWaves = 4, kTile = 32;
constexpr int kPiece = kTile * 256, kSlot = 2 * kPiece, kRing = 2 * kSlot;
constexpr size_t kCutFloats = sizeof(Cut) / sizeof(float) * kWorkgroups;

template <int kGroups>
struct State {
    f32x4 o[kGroups][8];     // of this lane's query rows (one of each 16): dims 16 d + 4 (lane / 16) + i
    float m[kGroups], l[kGroups];      // m in powers of two; l of the keys that the lane has seen
};

struct Source {
    const unsigned char *K, *V;      // of head 0 of page 0
    const int32_t* entries;
    int stride, n_pages, shift, n_kv, h, end;
};

// Which keys the lane's query rows attend.  edge: some row of the tile sees one of its keys that another one does not.
template <int kGroups, class A>
struct Seen;
template <int kGroups>
struct Seen<kGroups, PagedAttention> {       // those up to their own position, the last `window` of them
    int position[kGroups], pos_min, pos_max, window;
    __device__ __forceinline__ void item(const PagedAttention& a, const Item& it, int first, int tokens)
    {
        pos_min = it.rows.base + first;
        pos_max = pos_min + tokens - 1;
        window = a.window;
    }
    __device__ __forceinline__ void row(const PagedAttention&, const Item& it, int r, int i) { position[r] = it.rows.base + i; }
    __device__ __forceinline__ int end() const { return pos_max + 1; }
    __device__ __forceinline__ bool edge(int t) const { return t * kTile + kTile - 1 > pos_min || (window && t * kTile <= pos_max - window); }
    struct Tile {
        int upto, from;
        __device__ __forceinline__ bool operator()(int key) const { return key <= upto && key > from; }
    };
    __device__ __forceinline__ Tile in(int t, int r) const
    {
        const int upto = position[r] - t * kTile;
        return Tile{upto, window ? upto - window : -1};
    }
    __device__ __forceinline__ bool sees(int key, int r) const { return key <= position[r] && !(window && key <= position[r] - window); }
};
template <int kGroups>
struct Seen<kGroups, PagedTreeAttention> {       // see TreeRow; the tokens of a tile are 64 at most, one word
    unsigned long long marks[kGroups];
    int low[kGroups], base, last;
    TreeEdges edges;
    __device__ __forceinline__ void item(const PagedTreeAttention& a, const Item& it, int, int)
    {
        base = it.rows.base;
        last = base + it.rows.n;
        edges = tree_edges(a, it.rows);
    }
    __device__ __forceinline__ void row(const PagedTreeAttention& a, const Item& it, int r, int i)
    {
        const TreeRow t = tree_row(a, it.rows, i);
        marks[r] = t.mask[0];
        low[r] = t.low;
    }
    __device__ __forceinline__ int end() const { return last; }
    __device__ __forceinline__ bool edge(int t) const { return t * kTile + kTile - 1 >= edges.from || t * kTile < edges.upto; }
    struct Tile {
        uint32_t bits;
        __device__ __forceinline__ bool operator()(int key) const { return bits >> key & 1; }
    };
    __device__ __forceinline__ Tile in(int t, int r) const
    {
        const int at = t * kTile - base;                      // of the tile's first key among the new ones
        const uint32_t marked = at >= 64 || at <= -kTile ? 0u : (uint32_t)(at >= 0 ? marks[r] >> at : marks[r] << -at);
        return Tile{((uint32_t)below(-at) | marked) & ~(uint32_t)below(low[r] - t * kTile)};
    }
    __device__ __forceinline__ bool sees(int key, int r) const { return in(key / kTile, r)(key & (kTile - 1)); }
};

// Tiles [t0, t1) of 32 keys through one wave; `ring`: LDS offset of its ring.
// kOnePage: pages of 16 rows or more, which hold halves of tiles, so that their addresses are scalars.
template <int kGroups, bool kOnePage, class A>
__device__ __forceinline__ void stream(State<kGroups>& st, const Source& c, const bf16x8 (&q)[kGroups][4], int t0, int t1, uint32_t ring,
                                       const Seen<kGroups, A>& seen, float scale)
{
    const float top = hidden_infinity();
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    // LDS: chunk j (16 bytes) of key r lies at j ^ r % 16, of value r at j ^ 2 (r % 8): the lanes of a read touch different banks
    const uint32_t k_at = ring + (uint32_t)(col * 256 + ((g ^ col) << 4));                                  // ^ 64 ks
    const int vr = 4 * g + (col >> 2);
    const uint32_t v_at = ring + kPiece + (uint32_t)(vr * 256 + ((((col & 3) >> 1) ^ ((vr & 7) << 1)) << 4) + (col & 1) * 8);      // ^ 32 d

    // (entries are looked at two tiles after they were asked for: looked at at once, they made the wave wait for all loads before them)
    auto entry_at = [&](int t) { return c.entries[entry_of(t, kTile, kOnePage ? lane & 16 : lane & 31, c.end, c.shift)]; };      // of key 32 t + lane % 32, or of its half
    auto held = [&](int t, int entry) {
        if constexpr (kOnePage) {
            const int n = c.end - t * kTile;
            const uint32_t in = ((uint32_t)lane_value(entry, 0) < (uint32_t)c.n_pages ? 0xffffu : 0u) | ((uint32_t)lane_value(entry, 16) < (uint32_t)c.n_pages ? 0xffff0000u : 0u);
            return n >= 32 ? in : in & ((1u << n) - 1u);
        } else {
            return (uint32_t)__ballot(t * kTile + (lane & 31) < c.end && (uint32_t)entry < (uint32_t)c.n_pages);
        }
    };
    // What a lane loads, in bytes: rows 4 i + g of a half tile, i = 0 .. 3 (keys) or 0, 1 (values; 2 and 3 are 2048 on).
    uint32_t k_from[4], v_from[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) k_from[i] = (uint32_t)((4 * i + g) * 256 + ((col ^ (4 * i + g)) << 4));
#pragma unroll
    for (int i = 0; i < 2; ++i) v_from[i] = (uint32_t)((4 * i + g) * 256 + ((col ^ ((4 * i + g) << 1)) << 4));
    long long off[kOnePage ? 2 : 8];
    auto offsets = [&](int t, int entry, uint32_t valid) {    // bytes, of the tile's halves or of rows 4 i + g; those that are not there: somewhere in page 0
        if constexpr (kOnePage) {
            off[0] = row_of(valid & 0xffffu ? lane_value(entry, 0) : 0, c.h, c.n_kv, c.shift, t * kTile) * 256;
            off[1] = row_of(valid >> 16 ? lane_value(entry, 16) : 0, c.h, c.n_kv, c.shift, t * kTile + 16) * 256;
        } else {
            const int mine = (valid >> (lane & 31) & 1) ? entry : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) off[i] = row_of(__shfl(mine, 4 * i + g, 64), c.h, c.n_kv, c.shift, t * kTile + 4 * i + g) * 256;
        }
    };
    auto load_keys = [&](int t) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t to = ring + (uint32_t)((t & 1) * kSlot + i * 1024);
            if constexpr (kOnePage) load_to_lds(c.K + off[i >> 2] + k_from[i & 3], to);
            else load_to_lds(c.K + off[i] + (k_from[i & 3] & 255u), to);
        }
    };
    auto load_values = [&](int t) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t to = ring + (uint32_t)((t & 1) * kSlot + kPiece + i * 1024);
            if constexpr (kOnePage) load_to_lds(c.V + off[i >> 2] + ((i >> 1) & 1) * 2048 + v_from[i & 1], to);
            else load_to_lds(c.V + off[i] + (v_from[i & 1] & 255u), to);
        }
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
        const bool edge = seen.edge(t);
        f32x4 s[kGroups][2];
#pragma unroll
        for (int r = 0; r < kGroups; ++r) s[r][0] = s[r][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int r = 0; r < kGroups; ++r) {
                s[r][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[ks], q[r][ks], s[r][0], 0, 0, 0);
                s[r][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[4 + ks], q[r][ks], s[r][1], 0, 0, 0);
            }
        if (valid != 0xffffffffu || edge) {
#pragma unroll
            for (int r = 0; r < kGroups; ++r) {
                const auto sees = seen.in(t, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = 16 * (i >> 2) + 4 * g + (i & 3);
                    s[r][i >> 2][i & 3] = (valid >> key & 1) && sees(key) ? s[r][i >> 2][i & 3] : -INFINITY;
                }
            }
        }
        float mx[kGroups];
        bool grown = false;
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            mx[r] = larger(s[r][0][0], s[r][1][0], top);
#pragma unroll
            for (int i = 1; i < 4; ++i) mx[r] = fmaxf(mx[r], larger(s[r][0][i], s[r][1][i], top));
            mx[r] *= scale;
            grown |= mx[r] > st.m[r] + 8.f;
        }
        // The maximum in use may be up to 2^8 behind: sums in fp32 and products of bf16 have room for it, and it is soon never moved.
        if (__any(grown)) {
#pragma unroll
            for (int r = 0; r < kGroups; ++r) {
                float n = fmaxf(mx[r], st.m[r]);
                n = fmaxf(n, __shfl_xor(n, 16, 64));
                n = fmaxf(n, __shfl_xor(n, 32, 64));
                const float f = n == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m[r] - n);
                st.m[r] = n;
                st.l[r] *= f;
#pragma unroll
                for (int d = 0; d < 8; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) st.o[r][d][i] *= f;
            }
        }
        // Probabilities are two bf16 values each where the products for that cost nothing (up to 32 rows): what truncation leaves of one (2^-7) is the second, rounded (2^-8): an error of 2^-15.
        // Four groups take them rounded to bf16 (2^-8): 40 rows over 30K keys, eight sequences, 95 us, with two values 104.
        constexpr bool kTwo = kGroups <= 2;
        bf16x8 p[kGroups], p2[kTwo ? kGroups : 1];
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            const float m = st.m[r] == -INFINITY ? 0.f : st.m[r];
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(fmaf(s[r][i >> 2][i & 3], scale, -m));
                st.l[r] += e[i];
                if constexpr (!kTwo) p[r][i] = (__bf16)e[i];
                else p2[r][i] = (__bf16)(e[i] - __uint_as_float(__float_as_uint(e[i]) & 0xffff0000u));
            }
            if constexpr (kTwo) {
                u32x4 top_halves;
#pragma unroll
                for (int i = 0; i < 4; ++i) top_halves[i] = __builtin_amdgcn_perm(__float_as_uint(e[2 * i + 1]), __float_as_uint(e[2 * i]), 0x07060302u);
                p[r] = __builtin_bit_cast(bf16x8, top_halves);
                // (a second part of zero would make an infinite value NaN: it is 2^-126 at least, or the probability if that is less)
                const u16x8 tiny = {0x0080, 0x0080, 0x0080, 0x0080, 0x0080, 0x0080, 0x0080, 0x0080};
                const u16x8 floor = __builtin_elementwise_min(__builtin_bit_cast(u16x8, top_halves), tiny);
                p2[r] = __builtin_bit_cast(bf16x8, __builtin_elementwise_max(__builtin_bit_cast(u16x8, p2[r]), floor));
            }
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
#pragma unroll
                for (int r = 0; r < kGroups; ++r) {
                    st.o[r][4 * d4 + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), p[r], st.o[r][4 * d4 + d], 0, 0, 0);
                    if constexpr (kTwo)
                        st.o[r][4 * d4 + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), p2[r], st.o[r][4 * d4 + d], 0, 0, 0);
                }
            }
        }
        if constexpr (kAhead == 2) load_values(t + 2);
        // the values taken out are added to the rows that see them
        for (; odd; odd &= odd - 1) {
            const int key = t * kTile + __builtin_ctz(odd);
            const int page = page_of(c.entries, c.stride, c.n_pages, c.shift, key);
            const uint2* from = reinterpret_cast<const uint2*>(c.V + row_of(max(page, 0), c.h, c.n_kv, c.shift, key) * 256);
#pragma unroll
            for (int d = 0; d < 8; ++d) {
                const uint2 w = from[4 * d + g];
                const uint32_t u[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
                for (int r = 0; r < kGroups; ++r) {
                    const bool sees = seen.sees(key, r);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (sees && (u[e] & 0x7f800000u) == 0x7f800000u) st.o[r][d][e] += __uint_as_float(u[e]);
                }
            }
        }
    };
    int t = t0;
    for (; t + 2 < t1; ++t) tile(t, std::integral_constant<int, 2>{});
    if (t + 1 < t1) tile(t++, std::integral_constant<int, 1>{});
    tile(t, std::integral_constant<int, 0>{});
}

template <int kGroups, bool kOnePage, class A>
__device__ __forceinline__ void attend(const A& a, const Tiling& tl, float* parts, Cut* cuts)
{
    constexpr int kRows = 16 * kGroups;
    __shared__ __align__(256) unsigned char lds[kWaves * kRing + 2 * kWaves * kRows * 4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    Line line = line_of<true>(a, tl);
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
        segment_at<true>(a, tl, line, x, x_end, known, &seg);
        const Item& it = seg.it;
        const int h = seg.h, first = seg.first, last = seg.last;
        if (first == last) continue;                       // (the share ends among the places in front)
        const bool whole = first == it.b0 && last == it.b1;
        const int tokens = min(it.rows.n - it.tile * tl.tokens, tl.tokens), tile_rows = tokens * G;
        Seen<kGroups, A> seen;
        seen.item(a, it, it.tile * tl.tokens, tokens);
        int token[kGroups], head[kGroups];
        bf16x8 q[kGroups][4];
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            const int row = min(16 * r + col, tile_rows - 1), in_tile = token_of_row(tl, row), i = it.tile * tl.tokens + in_tile;
            token[r] = it.rows.q0 + i;
            head[r] = h * G + row - in_tile * G;
            seen.row(a, it, r, i);
            const uint4* from = reinterpret_cast<const uint4*>(a.q + (long long)token[r] * a.q_stride + (long long)head[r] * kHeadDim);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) q[r][ks] = __builtin_bit_cast(bf16x8, from[4 * ks + g]);
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
        c.end = min(seen.end(), room_of(a));
        // the wave's tiles: a quarter of the share's
        const int t0 = first * kWaves + wave * (last - first), t1 = min(t0 + (last - first), c.end > 0 ? (c.end - 1) / kTile + 1 : 0);
        State<kGroups> st;
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            st.m[r] = -INFINITY;
            st.l[r] = 0.f;
#pragma unroll
            for (int d = 0; d < 8; ++d) st.o[r][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if (t0 < t1) stream<kGroups, kOnePage, A>(st, c, q, t0, t1, ring, seen, a.scale_log2e);

        // The waves' sums meet.
        __syncthreads();
        f32x4* sm_o = reinterpret_cast<f32x4*>(lds);                            // [kWaves][kGroups][8][64]
        float* sm_m = reinterpret_cast<float*>(lds + kWaves * kRing);           // [kWaves][kRows], then sums
        float* sm_l = sm_m + kWaves * kRows;
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            float l = st.l[r];
            l += __shfl_xor(l, 16, 64);
            l += __shfl_xor(l, 32, 64);
#pragma unroll
            for (int d = 0; d < 8; ++d) sm_o[((wave * kGroups + r) * 8 + d) * 64 + lane] = st.o[r][d];
            if (lane < 16) {
                sm_m[wave * kRows + 16 * r + lane] = st.m[r];
                sm_l[wave * kRows + 16 * r + lane] = l;
            }
        }
        __syncthreads();
        float* part = parts + (2ll * share + slot_of(blocks_from(it, line, h), share, line.share)) * part_floats(kGroups);
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            float M = -INFINITY, L = 0.f, f[kWaves];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm_m[w * kRows + 16 * r + col]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                f[w] = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm_m[w * kRows + 16 * r + col] - M);
                L = fmaf(sm_l[w * kRows + 16 * r + col], f[w], L);
            }
#pragma unroll
            for (int dd = 0; dd < 2; ++dd) {
                const int d = wave + 4 * dd;
                f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const f32x4 y = sm_o[((w * kGroups + r) * 8 + d) * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], f[w], o[e]);
                }
                if (whole) {
                    if (16 * r + col < tile_rows) store_row(a, token[r], head[r], o, M, L, d, g);
                } else {
                    reinterpret_cast<f32x4*>(part)[(8 * r + d) * 64 + lane] = o;
                }
            }
            if (!whole && wave == 0 && lane < 16) {
                part[kRows * kHeadDim + 16 * r + lane] = M;
                part[kRows * kHeadDim + kRows + 16 * r + lane] = L;
            }
        }
        if (last < it.b1) cut = cut_of(it, tl, line, share, h);
        __syncthreads();
    }
    if (threadIdx.x == 0) cuts[share] = cut;
}

template <int kGroups, bool kOnePage>
__global__ __launch_bounds__(64 * kWaves, 1) void paged_token_kernel(PagedAttention a, Tiling tl, float* parts, Cut* cuts)
{
    attend<kGroups, kOnePage>(a, tl, parts, cuts);
}
template <int kGroups, bool kOnePage>
__global__ __launch_bounds__(64 * kWaves, 1) void paged_tree_token_kernel(PagedTreeAttention a, Tiling tl, float* parts, Cut* cuts)
{
    attend<kGroups, kOnePage>(a, tl, parts, cuts);
}

// One workgroup a cut, 16 rows and 16 dims: its waves take parts in turn, eight at a time, so that a cut of up to 32 parts costs one trip to memory.
template <int kGroups>
__global__ __launch_bounds__(256) void paged_token_merge_kernel(PagedAttention a, int group, const float* parts, const Cut* cuts)
{
    constexpr int kRows = 16 * kGroups;
    __shared__ f32x4 sm_o[4][64];
    __shared__ float sm_m[4][16], sm_l[4][16];
    const int share = blockIdx.x / (8 * kGroups), r = blockIdx.x / 8 % kGroups, d = blockIdx.x & 7;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const Cut c = cuts[share];
    if (c.parts == 0 || 16 * r >= c.rows) return;
    float M = -INFINITY, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = wave; i0 < c.parts; i0 += 32) {
        float m[8], l[8];
        f32x4 y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = min(i0 + 4 * k, c.parts - 1);
            const float* p = parts + (2ll * (share + i) + (i == 0 ? c.slot : 0)) * part_floats(kGroups);
            m[k] = p[kRows * kHeadDim + 16 * r + col];
            l[k] = p[kRows * kHeadDim + kRows + 16 * r + col];
            y[k] = reinterpret_cast<const f32x4*>(p)[(8 * r + d) * 64 + lane];
        }
        float n = M;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (i0 + 4 * k >= c.parts) m[k] = -INFINITY;
            n = fmaxf(n, m[k]);
        }
        const float base = n == -INFINITY ? 0.f : n, before = __builtin_amdgcn_exp2f(M - base);
        M = n;
        L *= before;
        o *= before;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float f = __builtin_amdgcn_exp2f(m[k] - base);
            if (i0 + 4 * k < c.parts) {
                L = fmaf(l[k], f, L);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(y[k][e], f, o[e]);
            }
        }
    }
    sm_o[wave][lane] = o;
    if (lane < 16) {
        sm_m[wave][lane] = M;
        sm_l[wave][lane] = L;
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) M = fmaxf(M, sm_m[w][col]);
    const float base = M == -INFINITY ? 0.f : M;
    L = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm_m[w][col] - base);
        L = fmaf(sm_l[w][col], f, L);
        const f32x4 y = sm_o[w][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], f, o[e]);
    }
    const int row = 16 * r + col;
    if (row < c.rows) store_row(a, c.q0 + row / group, c.head * group + row % group, o, M, L, d, g);
}

// The same where most cuts have two or three parts, of which eight loads a wave bring most several times: parts of 64 rows or more of many items, us: 24 tokens each of 32 sequences of up to 2K,
// 8 KV heads of four, 15.0 -> 9.2; 12 each 9.7 -> 6.1.  (For everything, this costs single tokens over 4096 keys 5.5 us for 4.8.)  Both give the same bits.
template <int kGroups>
__global__ __launch_bounds__(256) void paged_token_merge_few_kernel(PagedAttention a, int group, const float* parts, const Cut* cuts)
{
    constexpr int kRows = 16 * kGroups;
    __shared__ f32x4 sm_o[4][64];
    __shared__ float sm_m[4][16], sm_l[4][16];
    const int share = blockIdx.x / (8 * kGroups), r = blockIdx.x / 8 % kGroups, d = blockIdx.x & 7;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const Cut c = cuts[share];
    if (c.parts == 0 || 16 * r >= c.rows) return;
    float M = -INFINITY, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    // The wave's parts from i0 on, every fourth, up to kAtOnce of them on their way together.
    auto take = [&](int i0, auto at_once) {
        constexpr int kAtOnce = decltype(at_once)::value;
        float m[kAtOnce], l[kAtOnce];
        f32x4 y[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int i = min(i0 + 4 * k, c.parts - 1);
            const float* p = parts + (2ll * (share + i) + (i == 0 ? c.slot : 0)) * part_floats(kGroups);
            m[k] = p[kRows * kHeadDim + 16 * r + col];
            l[k] = p[kRows * kHeadDim + kRows + 16 * r + col];
            y[k] = reinterpret_cast<const f32x4*>(p)[(8 * r + d) * 64 + lane];
        }
        float n = M;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            if (i0 + 4 * k >= c.parts) m[k] = -INFINITY;
            n = fmaxf(n, m[k]);
        }
        const float base = n == -INFINITY ? 0.f : n, before = __builtin_amdgcn_exp2f(M - base);
        M = n;
        L *= before;
        o *= before;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const float f = __builtin_amdgcn_exp2f(m[k] - base);
            if (i0 + 4 * k < c.parts) {
                L = fmaf(l[k], f, L);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(y[k][e], f, o[e]);
            }
        }
    };
    if (c.parts <= 4) {
        if (wave < c.parts) take(wave, std::integral_constant<int, 1>{});
    } else {
        for (int i0 = wave; i0 < c.parts; i0 += 32) take(i0, std::integral_constant<int, 8>{});
    }
    sm_o[wave][lane] = o;
    if (lane < 16) {
        sm_m[wave][lane] = M;
        sm_l[wave][lane] = L;
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) M = fmaxf(M, sm_m[w][col]);
    const float base = M == -INFINITY ? 0.f : M;
    L = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm_m[w][col] - base);
        L = fmaf(sm_l[w][col], f, L);
        const f32x4 y = sm_o[w][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], f, o[e]);
    }
    const int row = 16 * r + col;
    if (row < c.rows) store_row(a, c.q0 + row / group, c.head * group + row % group, o, M, L, d, g);
}

template <int kGroups, bool kOnePage>
auto kernel_of(const PagedAttention&) { return paged_token_kernel<kGroups, kOnePage>; }
template <int kGroups, bool kOnePage>
auto kernel_of(const PagedTreeAttention&) { return paged_tree_token_kernel<kGroups, kOnePage>; }

template <int kGroups, class A>
hipError_t launch(const A& a, float* room, hipStream_t s)
{
    const Tiling tl = tiling(a.n_q_heads / a.c.n_kv, 16 * kGroups, 0, 16 * kGroups, kWaves * kTile, 2, 1);
    Cut* cuts = reinterpret_cast<Cut*>(room);
    float* parts = room + kCutFloats;
    const auto kernel = a.c.page_shift >= 4 ? kernel_of<kGroups, true>(a) : kernel_of<kGroups, false>(a);
    hipLaunchKernelGGL(kernel, dim3(kWorkgroups), dim3(64 * kWaves), 0, s, a, tl, parts, cuts);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_paged_token_merge(a, kGroups, parts, cuts, s);
}

}  // namespace

// Sequences times KV heads from which on the merge for few parts runs.  Whole calls by that for many parts and by that for few, us, sequences of up to 2K, 12 and 24 tokens each, 8 KV heads of four: 16
// items 14.1 and 14.0, 19.2 and 17.9; 64 items 23.4 and 22.2, 32.5 and 29.8; 128 items 32.6 and 30.1, 42.4 and 37.4; 256 items 40.1 and 36.7, 53.1 and 46.6.  The line lies where it is safe rather
// than where they meet: one sequence over 4096 keys, 8 items, is the case above that loses.
constexpr int kManyItems = 128;

template <int kGroups>
static hipError_t merge(const PagedAttention& a, const float* parts, const Cut* cuts, hipStream_t s)
{
    auto kernel = paged_token_merge_kernel<kGroups>;
    if constexpr (kGroups >= 4)
        if ((long long)a.c.n_seqs * a.c.n_kv >= kManyItems) kernel = paged_token_merge_few_kernel<kGroups>;
    hipLaunchKernelGGL(kernel, dim3(8 * kGroups * kWorkgroups), dim3(256), 0, s, a, a.n_q_heads / a.c.n_kv, parts, cuts);
    return hipGetLastError();
}
hipError_t launch_paged_token_merge(const PagedAttention& a, int groups, const float* parts, const void* cuts, hipStream_t s)
{
    const Cut* c = (const Cut*)cuts;
    return groups == 1 ? merge<1>(a, parts, c, s) : groups == 2 ? merge<2>(a, parts, c, s) : groups == 4 ? merge<4>(a, parts, c, s) : merge<8>(a, parts, c, s);
}

size_t paged_token_floats(int rows) { return (size_t)2 * kWorkgroups * part_floats(rows / 16) + kCutFloats; }

hipError_t launch_paged_tokens(const PagedAttention& a, int rows, float* room, hipStream_t s)
{
    return rows == 16 ? launch<1>(a, room, s) : rows == 32 ? launch<2>(a, room, s) : rows == 64 ? launch<4>(a, room, s) : hipErrorInvalidValue;
}
// (more rows of a tree: mp_paged_rows.hip)
hipError_t launch_paged_tokens(const PagedTreeAttention& a, int rows, float* room, hipStream_t s)
{
    return rows == 16 ? launch<1>(a, room, s) : rows == 32 ? launch<2>(a, room, s) : hipErrorInvalidValue;
}

}  // namespace mp
