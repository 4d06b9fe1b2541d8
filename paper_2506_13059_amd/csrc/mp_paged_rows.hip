// Attention of a tree's tokens over a paged cache, up to 128 query rows a KV head, on the matrix cores, for gfx950.  (mp_paged_attn.hip says what is computed.)
//
// Four or eight waves of 16 query rows each meet the same keys: 64 of them and their values at a time go straight to LDS (global_load_lds, 16 bytes a lane) into a ring of four
// blocks, one in use and three on their way, and the waves meet behind each.  S^T = K Q^T and O^T += V^T P^T are v_mfma_f32_16x16x32_bf16 as in mp_paged_token.hip; a wave's rows are
// its own, so nothing is put together in the workgroup.  Bound by memory, or by trips to it and to instructions: a third of the code of mp_paged_token.hip for 64 rows, where each wave has all rows and keys of its own.
//
// By this and by what ran before (that one up to 64 rows, mp_paged_chunk.hip), 8 KV heads of four, us: 12 tokens over 4096 keys 16.8 and 22.4, 24 over as many 20 and 23.6; 12 each of 8 sequences of up to 30K 81 and
// 87 (5.4 TB/s), 24 each 106 and 124, 32 each 91 and 102; 12 each of 32 of up to 2K 38 and 62, 24 each 46.8 and 46.9 (lengths
// are drawn anew for each number of tokens, so that those of 32 each hold less than those of 24).  Two groups of rows a wave, for up to 256, took 8 to 10 % longer than chunks.
#include "mp_paged_tile.h"

namespace mp {

namespace {

constexpr int kKeys = 64, kRing = 4;
constexpr int kHalf = 2 * 32 * 256, kBlockBytes = 2 * kHalf, kValues = 32 * 256;      // LDS: 32 keys and their values, and 32 more

// 16 bytes at `at` and each 1024 behind.
__device__ __forceinline__ void lds_read(u32x4 (&w)[2], uint32_t at)
{
    asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:1024\n\ts_waitcnt lgkmcnt(0)" : "=&v"(w[0]), "=&v"(w[1]) : "v"(at) : "memory");
}
__device__ __forceinline__ void lds_read(u32x4 (&w)[4], uint32_t at)
{
    asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:0x400\n\tds_read_b128 %2, %4 offset:0x800\n\tds_read_b128 %3, %4 offset:0xc00\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3])
                 : "v"(at)
                 : "memory");
}
// (this and the next: waited for where the waves meet)
__device__ __forceinline__ void lds_write16(uint32_t at, u32x4 w) { asm volatile("ds_write_b128 %0, %1" ::"v"(at), "v"(w) : "memory"); }
__device__ __forceinline__ unsigned long long lds_read8(uint32_t at)        // the same in all lanes
{
    unsigned long long w;
    asm volatile("ds_read_b64 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(w) : "v"(at) : "memory");
    return (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(w >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)w);
}
template <int kBytes>
__device__ __forceinline__ void lds_write_bits(uint32_t at, uint32_t v)
{
    if constexpr (kBytes == 1) asm volatile("ds_write_b8 %0, %1" ::"v"(at), "v"(v) : "memory");
    else asm volatile("ds_write_b16 %0, %1" ::"v"(at), "v"(v) : "memory");
}
__device__ __forceinline__ void workgroup_sync()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Four bytes a lane, lane i's to lds_off + 4 i.
__device__ __forceinline__ void load4_to_lds(const void* src, uint32_t lds_off)
{
    auto* dst = reinterpret_cast<__attribute__((address_space(3))) uint32_t*>((uintptr_t)lds_off);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src, dst, 4, 0, 0);
}
__device__ __forceinline__ int lds_read4(uint32_t at)
{
    int w;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(w) : "v"(at) : "memory");
    return w;
}

// kOnePage: a page holds the rows that a wave brings of a block, so that their address is a scalar.  Entries of smaller pages go to LDS as the rows do, two blocks before they are used: a load to
// a register is waited for with all that was asked for before it, which were the three blocks on their way.  12 tokens each of 8 sequences of up to 30K, 8 KV heads of four, pages of 8: 97.2 us
// and, so, 90.9 (pages of 16 rows 87.9); pages of one 102.7 and 93.3; 24 each, pages of 4, where it is eight waves' instructions that take the time, 107.0 and 108.4.
template <int kWaves, bool kOnePage>
__global__ __launch_bounds__(64 * kWaves, kWaves / 4) void paged_tree_rows_kernel(PagedTreeAttention a, Tiling tl, float* parts, Cut* cuts)
{
    constexpr int kBring = kKeys / kWaves, kLoads = kBring / 4;          // rows that a wave brings of a block, and instructions for its keys
    constexpr int kBitBytes = kBring / 8;
    __shared__ __align__(256) unsigned char lds[kRing * kBlockBytes + 2 * kRing * 8 + (kOnePage ? 0 : kWaves * kRing * 256)];
    const uint32_t ring = (uint32_t)(uintptr_t)(lds_byte*)lds, valid_at = ring + kRing * kBlockBytes, odd_at = valid_at + kRing * 8;      // (a bit a key: there; its values not all finite)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const float top = hidden_infinity();
    Line line = line_of<true>(a, tl);
    const int share = share_of(line, blockIdx.x);
    if (share >= line.used) {
        if (threadIdx.x == 0) cuts[share].parts = 0;
        return;
    }
    const int G = tl.group;
    const float scale = a.scale_log2e;

    // LDS: chunk j (16 bytes) of key r lies at j ^ r % 16, of value r at j ^ 2 (r % 8): the lanes of a read touch different banks
    const uint32_t k_at = ring + (uint32_t)(col * 256 + ((g ^ col) << 4));                                  // ^ 64 ks
    const int vr = 4 * g + (col >> 2);
    const uint32_t v_at = ring + kValues + (uint32_t)(vr * 256 + ((((col & 3) >> 1) ^ ((vr & 7) << 1)) << 4) + (col & 1) * 8);      // ^ 32 d
    const int row0 = kBring * wave;
    const uint32_t wave_at = ring + (uint32_t)((row0 >> 5) * kHalf + (row0 & 31) * 256), entries_at = odd_at + kRing * 8 + (uint32_t)(wave * kRing * 256);
    uint32_t k_from[kLoads], v_from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = row0 + 4 * i + g;
        k_from[i] = (uint32_t)((4 * i + g) * 256 + ((col ^ (r & 15)) << 4));
        v_from[i] = (uint32_t)((4 * i + g) * 256 + ((col ^ ((r & 7) << 1)) << 4));
    }

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
        const int base = it.rows.base, end = min(base + it.rows.n, room_of(a));      // keys of the sequence

        // Loading: the wave's rows of a block.
        const int32_t* entries = a.c.table + (long long)it.b * a.c.table_stride;
        typedef const __attribute__((address_space(4))) int32_t constant_int;
        // What a wave needs to know of them: the entry (or, for small pages, one of each row in lanes 64 / kBring r ..).
        auto place_at = [&](int block) { return max(min(block * kKeys + row0 + (kOnePage ? 0 : lane / (64 / kBring)), end - 1), 0) >> a.c.page_shift; };
        auto entry_at = [&](int block) {
            if constexpr (kOnePage) return (int)((constant_int*)entries)[place_at(block)];
            else return (int)entries[place_at(block)];
        };
        // (small pages: asked for, and read by the same wave when blocks behind have come)
        auto ask = [&](int block) { load4_to_lds(entries + place_at(block), entries_at + (uint32_t)((block & (kRing - 1)) * 256)); };
        auto asked = [&](int block) { return lds_read4(entries_at + (uint32_t)((block & (kRing - 1)) * 256 + lane * 4)); };
        // A bit for each of them that is there.
        auto bits_of = [&](int block, int entry) {
            const int n = end - (block * kKeys + row0);
            const uint32_t in = n >= kBring ? (1u << kBring) - 1u : n > 0 ? (1u << n) - 1u : 0u;
            if constexpr (kOnePage) return (uint32_t)__builtin_amdgcn_readfirstlane(entry) < (uint32_t)a.c.n_pages ? in : 0u;
            const unsigned long long ok = __ballot((uint32_t)entry < (uint32_t)a.c.n_pages);
            uint32_t held = 0;
#pragma unroll
            for (int r = 0; r < kBring; ++r) held |= (uint32_t)(ok >> (64 / kBring * r) & 1) << r;
            return in & held;
        };
        // (rows that are not there: those of page 0)
        auto load = [&](int block, int entry, uint32_t bits) {
            const int key = block * kKeys + row0, place = block & (kRing - 1);
            const uint32_t to = wave_at + (uint32_t)(place * kBlockBytes);
            lds_write_bits<kBitBytes>(valid_at + (uint32_t)(place * 8 + wave * kBitBytes), bits);
            const unsigned char *K = reinterpret_cast<const unsigned char*>(a.c.K), *V = reinterpret_cast<const unsigned char*>(a.c.V);
            if constexpr (kOnePage) {
                const long long at = row_of(bits ? __builtin_amdgcn_readfirstlane(entry) : 0, h, a.c.n_kv, a.c.page_shift, key) * 256;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) load_to_lds(K + at + k_from[i], to + i * 1024);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) load_to_lds(V + at + v_from[i], to + kValues + i * 1024);
            } else {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int n = 4 * i + g, page = __shfl(entry, 64 / kBring * n, 64);
                    const long long at = row_of((bits >> n & 1) ? page : 0, h, a.c.n_kv, a.c.page_shift, key + n) * 256;
                    load_to_lds(K + at + (k_from[i] & 255u), to + i * 1024);
                    load_to_lds(V + at + (v_from[i] & 255u), to + kValues + i * 1024);
                }
            }
        };
        constexpr int kEntries = kOnePage ? 4 : 3;
        int entry[kEntries];
        uint32_t bits[4];                                  // of blocks t .. t + 3
#pragma unroll
        for (int i = 0; i < kEntries; ++i) entry[i] = entry_at(min(first + i, last - 1));

        // this lane's query row
        const int tile_rows = min(it.rows.n - it.tile * tl.tokens, tl.tokens) * G;
        const bool active = wave * 16 < tile_rows;
        const int r = min(wave * 16 + col, tile_rows - 1), in_tile = token_of_row(tl, r), i = it.tile * tl.tokens + in_tile;
        const int token = it.rows.q0 + i, head = h * G + r - in_tile * G;
        bf16x8 q[4];
        {
            const uint4* from = reinterpret_cast<const uint4*>(a.q + (long long)token * a.q_stride + (long long)head * kHeadDim);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) q[ks] = __builtin_bit_cast(bf16x8, from[4 * ks + g]);
        }
        const TreeRow row = tree_row(a, it.rows, i);
        unsigned long long marks0 = row.mask[0], marks1 = row.mask[a.words > 1 ? 1 : 0];      // (128 rows: 128 tokens at most)
        if (a.words == 1) marks1 = 0;
        // (here, for otherwise the wait for them is put into the loop, and there it is one for all loads to LDS)
        asm volatile("" : "+v"(q[0]), "+v"(q[1]), "+v"(q[2]), "+v"(q[3]), "+v"(marks0), "+v"(marks1));
        const TreeEdges edges = tree_edges(a, it.rows);
        auto edge = [&](int block) { return block * kKeys + kKeys - 1 >= edges.from || block * kKeys < edges.upto; };
        // a bit for each key of a block
        auto attended = [&](int block) {
            const int at = block * kKeys - base, by = at & 63;
            const unsigned long long lo = at >= 128 || at <= -64 ? 0ull : at >= 64 ? marks1 : at >= 0 ? marks0 : 0ull;
            const unsigned long long hi = at >= 64 || at <= -64 ? 0ull : at >= 0 ? marks1 : marks0;
            const unsigned long long marked = by ? lo >> by | hi << (64 - by) : lo;
            return (below(-at) | marked) & ~below(row.low - block * kKeys);
        };
        // When the wave's rows of a block have come: values of rows that are not there are zeroed (a probability of zero meets them), and so are those of an edge's block that
        // are not finite, lest they meet the zero of a row that does not see them.
        auto arrived = [&](int block, uint32_t there) {
            uint32_t odd = 0;
            const bool at_edge = edge(block);
            const int place = block & (kRing - 1);
            if (there != (1u << kBring) - 1u || at_edge) {
                const uint32_t at = wave_at + (uint32_t)(place * kBlockBytes) + kValues + lane * 16;
                u32x4 w[kLoads];
                lds_read(w, at);
#pragma unroll
                for (int e = 0; e < kLoads; ++e) {
                    bool off_range = false;
                    if (!(there >> (4 * e + g) & 1)) {
                        w[e] = u32x4{0u, 0u, 0u, 0u};
                    } else if (at_edge) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const bool lo = (w[e][k] & 0x7f80u) == 0x7f80u, hi = (w[e][k] & 0x7f800000u) == 0x7f800000u;
                            off_range |= lo | hi;
                            w[e][k] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
                        }
                    }
                    lds_write16(at + e * 1024, w[e]);
                    const unsigned long long in = __ballot(off_range);
#pragma unroll
                    for (int k = 0; k < 4; ++k) odd |= (uint32_t)((in >> (16 * k) & 0xffff) != 0) << (4 * e + k);
                }
            }
            if (at_edge) lds_write_bits<kBitBytes>(odd_at + (uint32_t)(place * 8 + wave * kBitBytes), odd);
        };
        // Blocks up to `block` have come; of those behind, up to two are on their way.
        auto wait_for = [&](int block) {
            const int behind = last - 1 - block;
            if (behind >= 2) wait_vm<4 * kLoads>();
            else if (behind == 1) wait_vm<2 * kLoads>();
            else wait_vm<0>();
        };

        f32x4 o[8];                                        // dims 16 d + 4 g + i
        float m = -INFINITY, l = 0.f;                      // m in powers of two; l of the keys that the lane has seen
#pragma unroll
        for (int d = 0; d < 8; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (end > 0) {
            workgroup_sync();                              // (the item before is done with LDS)
            if constexpr (!kOnePage) {
                ask(min(first + 3, last - 1));
                ask(min(first + 4, last - 1));
            }
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                bits[i] = bits_of(min(first + i, last - 1), entry[i]);
                if (first + i < last) load(first + i, entry[i], bits[i]);
            }
            int next = entry[kEntries - 1];
            wait_for(first);
            arrived(first, bits[0]);
            workgroup_sync();
            for (int t = first; t < last; ++t) {
                const int place = t & (kRing - 1);
                const uint32_t slot = (uint32_t)(place * kBlockBytes);
                if (t + 3 < last) {                        // (its place was that of t - 1, which all waves are done with)
                    if constexpr (!kOnePage) {
                        ask(min(t + 5, last - 1));
                        next = asked(t + 3);
                    }
                    bits[3] = bits_of(t + 3, next);
                    load(t + 3, next, bits[3]);
                    if constexpr (kOnePage) next = entry_at(min(t + 4, last - 1));
                }
                if (active) {
                    f32x4 s[4];
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        bf16x8 k[8];
                        const uint32_t at = slot + half * kHalf, a0 = k_at + at, a1 = (k_at ^ 64u) + at, a2 = (k_at ^ 128u) + at, a3 = (k_at ^ 192u) + at;
                        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
                                     "ds_read_b128 %4, %8 offset:4096\n\tds_read_b128 %5, %9 offset:4096\n\tds_read_b128 %6, %10 offset:4096\n\t"
                                     "ds_read_b128 %7, %11 offset:4096\n\ts_waitcnt lgkmcnt(0)"
                                     : "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3]), "=&v"(k[4]), "=&v"(k[5]), "=&v"(k[6]), "=&v"(k[7])
                                     : "v"(a0), "v"(a1), "v"(a2), "v"(a3)
                                     : "memory");
                        s[2 * half] = s[2 * half + 1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks) {
                            s[2 * half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[ks], q[ks], s[2 * half], 0, 0, 0);
                            s[2 * half + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[4 + ks], q[ks], s[2 * half + 1], 0, 0, 0);
                        }
                    }
                    const unsigned long long valid = lds_read8(valid_at + (uint32_t)(place * 8));
                    const bool at_edge = edge(t);
                    if (valid != ~0ull || at_edge) {
                        const unsigned long long see = (at_edge ? valid & attended(t) : valid) >> (4 * g);
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[e >> 2][e & 3] = see >> (16 * (e >> 2) + (e & 3)) & 1 ? s[e >> 2][e & 3] : -INFINITY;
                    }
                    float mx = larger(s[0][0], s[1][0], top);
                    mx = fmaxf(mx, larger(s[2][0], s[3][0], top));
#pragma unroll
                    for (int e = 1; e < 4; ++e) mx = fmaxf(mx, fmaxf(larger(s[0][e], s[1][e], top), larger(s[2][e], s[3][e], top)));
                    mx *= scale;
                    // The maximum in use may be up to 2^8 behind: sums in fp32 and products of bf16 have room for it, and it is soon never moved.
                    if (__any(mx > m + 8.f)) {
                        float n = fmaxf(mx, m);
                        n = fmaxf(n, __shfl_xor(n, 16, 64));
                        n = fmaxf(n, __shfl_xor(n, 32, 64));
                        const float f = n == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - n);
                        m = n;
                        l *= f;
#pragma unroll
                        for (int d = 0; d < 8; ++d)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[d][e] *= f;
                    }
                    const float shift = m == -INFINITY ? 0.f : m;
                    // Probabilities are rounded to bf16 once (2^-8, as much as the results are), as of the causal form for more than 32 rows; their sum is that of the unrounded ones.  Error against 64
                    // bits 0.0021 (0.0016 where they have two parts, up to 32 rows).  Two parts here: 12 tokens over 4096 keys 16.3 -> 16.6 us, 12 each of 8 sequences of up to 30K 87.7 -> 93.8, 24
                    // each 105 -> 124.
                    bf16x8 p[2];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float y = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], scale, -shift));
                        l += y;
                        p[e >> 3][e & 7] = (__bf16)y;
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int d4 = 0; d4 < 2; ++d4) {
                            s16x4 v[8];
                            const uint32_t at = slot + half * kHalf, b0 = (v_at ^ (128u * d4)) + at, b1 = (v_at ^ (128u * d4 + 32u)) + at, b2 = (v_at ^ (128u * d4 + 64u)) + at,
                                           b3 = (v_at ^ (128u * d4 + 96u)) + at;
                            asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:4096\n\tds_read_b64_tr_b16 %2, %9\n\t"
                                         "ds_read_b64_tr_b16 %3, %9 offset:4096\n\tds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:4096\n\t"
                                         "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:4096\n\ts_waitcnt lgkmcnt(0)"
                                         : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
                                         : "v"(b0), "v"(b1), "v"(b2), "v"(b3)
                                         : "memory");
#pragma unroll
                            for (int d = 0; d < 4; ++d) {
                                const auto w = __builtin_shufflevector(v[2 * d], v[2 * d + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                                o[4 * d4 + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), p[half], o[4 * d4 + d], 0, 0, 0);
                            }
                        }
                    // Values that are not finite have been taken out of an edge's block: they are added to the rows that see them.
                    if (at_edge) {
                        for (unsigned long long odd = lds_read8(odd_at + (uint32_t)(place * 8)); odd; odd &= odd - 1) {
                            const int in = __ffsll((long long)odd) - 1, key = t * kKeys + in;
                            const int page = __builtin_amdgcn_readfirstlane(page_of(entries, a.c.table_stride, a.c.n_pages, a.c.page_shift, key));
                            const bool sees = attended(t) >> in & 1;
                            const uint2* from = reinterpret_cast<const uint2*>(a.c.V + row_of(max(page, 0), h, a.c.n_kv, a.c.page_shift, key) * kHeadDim);
#pragma unroll
                            for (int d = 0; d < 8; ++d) {
                                const uint2 w = from[4 * d + g];
                                const uint32_t u[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (sees && (u[e] & 0x7f800000u) == 0x7f800000u) o[d][e] += __uint_as_float(u[e]);
                            }
                        }
                    }
                }
                if (t + 1 < last) {
                    wait_for(t + 1);
                    arrived(t + 1, bits[1]);
                    bits[1] = bits[2];
                    bits[2] = bits[3];
                    workgroup_sync();
                }
            }
        }

        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (whole) {
            if (wave * 16 + col < tile_rows)
#pragma unroll
                for (int d = 0; d < 8; ++d) store_row(a, token, head, o[d], m, l, d, g);
        } else {
            float* part = parts + (2ll * share + slot_of(blocks_from(it, line, h), share, line.share)) * part_floats(kWaves);
            if (active) {
#pragma unroll
                for (int d = 0; d < 8; ++d) reinterpret_cast<f32x4*>(part)[(8 * wave + d) * 64 + lane] = o[d];
                if (lane < 16) {
                    part[16 * kWaves * kHeadDim + 16 * wave + lane] = m;
                    part[16 * kWaves * kHeadDim + 16 * kWaves + 16 * wave + lane] = l;
                }
            }
            if (last < it.b1) cut = cut_of(it, tl, line, share, h);
        }
    }
    if (threadIdx.x == 0) cuts[share] = cut;
}

template <int kWaves>
hipError_t launch(const PagedTreeAttention& a, float* room, hipStream_t s)
{
    const Tiling tl = tiling(a.n_q_heads / a.c.n_kv, 16 * kWaves, 0, 16 * kWaves, kKeys, 2, 1);
    Cut* cuts = reinterpret_cast<Cut*>(room);
    float* parts = room + sizeof(Cut) / sizeof(float) * kWorkgroups;
    const auto kernel = 1 << a.c.page_shift >= kKeys / kWaves ? paged_tree_rows_kernel<kWaves, true> : paged_tree_rows_kernel<kWaves, false>;
    hipLaunchKernelGGL(kernel, dim3(kWorkgroups), dim3(64 * kWaves), 0, s, a, tl, parts, cuts);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_paged_token_merge(a, kWaves, parts, cuts, s);
}

}  // namespace

hipError_t launch_paged_tree_rows(const PagedTreeAttention& a, int rows, float* room, hipStream_t s)
{
    return rows == 64 ? launch<4>(a, room, s) : rows == 128 ? launch<8>(a, room, s) : hipErrorInvalidValue;
}

}  // namespace mp
