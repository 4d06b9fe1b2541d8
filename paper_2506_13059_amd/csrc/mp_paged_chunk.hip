// Attention of many new tokens over a paged cache, on the matrix cores, for gfx950.  (mp_paged_attn.hip says what is computed.)
//
// Eight waves of 32 query rows each work on one item (mp_paged_plan.h): 64 keys and values at a time go straight to LDS (global_load_lds, 16 bytes a lane), into
// a ring of four blocks, two in use and two on their way.  S^T = K Q^T and O^T += V^T P^T are v_mfma_f32_32x32x16_bf16, so a lane holds one query row in both (its column): its softmax
// needs no more of other lanes than one exchange of maxima, and the rows of S^T that it holds are, converted to bf16, what the second product takes from it,
// with the values' rows read (transposed by LDS) in the same order.
//
// Bound by the matrix cores, at the clock that the power limit leaves (1370 of 1400 W read while it ran): 2048 tokens at 128K, 32 heads, 4.1 to 4.6 ms = 0.95 to 1.06 PFLOP/s at 2.0 to
// 2.1 GHz, from card to card (a large library product: 1.35 to 1.39 PFLOP/s at 1.8 GHz); the cores are busy 49 % of the cycles, the vector ALU with exponentials, sums, maxima and conversions (about
// 175 instructions a block and wave) 46 %, both as counted.  Eight waves, so that each SIMD has two: one computes where the other waits.  What brought it there, the same call: rows
// through registers, one block ahead 5.03 ms; straight to LDS 4.73; loads among the products 4.46; cheaper shares and page entries 4.35; waves that meet every second block 4.31; maxima 4.20 -> 4.12.
// Did nothing: waves of a SIMD half a block apart, priorities, more reads ahead.
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
constexpr int kRing = 4, kPiece = kKeys * 256, kBlockBytes = 2 * kPiece;      // LDS: blocks, keys and then values of one
constexpr int kPartFloats = kRows * kHeadDim + 2 * kRows;       // a part: weighted values as the lanes hold them, then maxima, then sums

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

// (what a wave has asked of LDS it has waited for by then)
__device__ __forceinline__ void workgroup_sync()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ void load_to_lds(const void* src, uint32_t lds_off)
{
    // (the LDS address is the same in all lanes; lane i's bytes go to it + 16 i)
    auto* dst = reinterpret_cast<__attribute__((address_space(3))) uint32_t*>((uintptr_t)lds_off);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src, dst, 16, 0, 0);
}
// At most N loads on their way, and nothing asked of LDS.
template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// LDS is read and written by hand: the compiler would have each access wait for every load to LDS that is on its way.
// Keys: the 16 bytes at a ^ 32 ks (ks = 0 .. 3), and 32 rows on: k[2 ks], k[2 ks + 1].
__device__ __forceinline__ void read_keys(bf16x8 (&k)[8], uint32_t a, uint32_t slot)
{
    const uint32_t a0 = a + slot, a1 = (a ^ 32u) + slot, a2 = (a ^ 64u) + slot, a3 = (a ^ 96u) + slot;
    asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:8192\n\tds_read_b128 %2, %9\n\tds_read_b128 %3, %9 offset:8192\n\t"
                 "ds_read_b128 %4, %10\n\tds_read_b128 %5, %10 offset:8192\n\tds_read_b128 %6, %11\n\tds_read_b128 %7, %11 offset:8192\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3]), "=&v"(k[4]), "=&v"(k[5]), "=&v"(k[6]), "=&v"(k[7])
                 : "v"(a0), "v"(a1), "v"(a2), "v"(a3)
                 : "memory");
}
// Values of 32 keys, transposed: v[2 (4 s + d)], v[2 (4 s + d) + 1] have dims 32 d .. of 16 keys from 16 s.
__device__ __forceinline__ void read_values(s16x4 (&v)[16], uint32_t a, uint32_t slot)
{
    const uint32_t a0 = a + slot, a1 = (a ^ 64u) + slot, a2 = (a ^ 128u) + slot, a3 = (a ^ 192u) + slot;
    asm volatile("ds_read_b64_tr_b16 %0, %16\n\tds_read_b64_tr_b16 %1, %16 offset:2048\n\tds_read_b64_tr_b16 %2, %17\n\t"
                 "ds_read_b64_tr_b16 %3, %17 offset:2048\n\tds_read_b64_tr_b16 %4, %18\n\tds_read_b64_tr_b16 %5, %18 offset:2048\n\t"
                 "ds_read_b64_tr_b16 %6, %19\n\tds_read_b64_tr_b16 %7, %19 offset:2048\n\t"
                 "ds_read_b64_tr_b16 %8, %16 offset:4096\n\tds_read_b64_tr_b16 %9, %16 offset:6144\n\tds_read_b64_tr_b16 %10, %17 offset:4096\n\t"
                 "ds_read_b64_tr_b16 %11, %17 offset:6144\n\tds_read_b64_tr_b16 %12, %18 offset:4096\n\tds_read_b64_tr_b16 %13, %18 offset:6144\n\t"
                 "ds_read_b64_tr_b16 %14, %19 offset:4096\n\tds_read_b64_tr_b16 %15, %19 offset:6144\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7]), "=&v"(v[8]), "=&v"(v[9]),
                   "=&v"(v[10]), "=&v"(v[11]), "=&v"(v[12]), "=&v"(v[13]), "=&v"(v[14]), "=&v"(v[15])
                 : "v"(a0), "v"(a1), "v"(a2), "v"(a3)
                 : "memory");
}
__device__ __forceinline__ u32x4 lds_read16(uint32_t at)
{
    u32x4 w;
    asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(w) : "v"(at) : "memory");
    return w;
}
__device__ __forceinline__ void lds_write16(uint32_t at, u32x4 w) { asm volatile("ds_write_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" ::"v"(at), "v"(w) : "memory"); }
__device__ __forceinline__ unsigned long long lds_read8(uint32_t at)        // the same in all lanes
{
    unsigned long long w;
    asm volatile("ds_read_b64 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(w) : "v"(at) : "memory");
    return (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(w >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)w);
}
// (not waited for: the wave's next read is)
__device__ __forceinline__ void lds_write1(uint32_t at, uint32_t v) { asm volatile("ds_write_b8 %0, %1" ::"v"(at), "v"(v) : "memory"); }

// The lowest n of 64 bits.
__device__ __forceinline__ unsigned long long below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }

// (a denominator of 0: no key, or none of any weight; NaN, of a logit that is NaN or +inf, stays)
__device__ __forceinline__ float lse_of(float m, float l) { return l != 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -INFINITY; }

// A lane's dims 32 d + 8 j + 4 half .. of a finished row, o[j] over l.
__device__ __forceinline__ void store_dims(const PagedAttention& a, long long row, int d, int half, const f32x4 (&o)[4], float l)
{
    const float f = l != 0.f ? 1.f / l : 0.f;
    unsigned char* out = reinterpret_cast<unsigned char*>(a.out) + row * 256 + half * 8 + d * 64;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (__bf16)(l != 0.f ? o[j][e] * f : 0.f);
        *reinterpret_cast<bf16x4*>(out + j * 16) = w;
    }
}

// The rows of a finished item.
__device__ __forceinline__ void store_rows(const PagedAttention& a, const Softmax& st, float l, int token, int head, bool there)
{
    const int half = (threadIdx.x & 63) >> 5;
    if (!there) return;
    const long long row = (long long)token * a.n_q_heads + head;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        f32x4 o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][e] = st.o[d][4 * j + e];
        store_dims(a, row, d, half, o, l);
    }
    if (a.lse && half == 0) a.lse[row] = lse_of(st.m, l);
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

// kOnePage: pages of eight rows or more.  (Smaller ones take addresses a lane, and eight registers more than there are: 2048 tokens at 32K 1.06 ms for 1.02.)
template <bool kOnePage>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_chunk_kernel(PagedAttention a, Tiling tl, float* parts, Cut* cuts)
{
    __shared__ __align__(256) unsigned char lds[kRing * kBlockBytes + 2 * kRing * kWaves];
    const uint32_t ring = lds_offset(lds), valid_at = ring + kRing * kBlockBytes, odd_at = valid_at + kRing * kWaves;      // (a byte a wave: keys that are there; whose values are not all finite)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
    const float top = hidden_infinity();
    Line line = line_of<false>(a, tl);
    const int share = share_of(line, blockIdx.x);
    if (share >= line.used) {
        if (threadIdx.x == 0) cuts[share].parts = 0;
        return;
    }
    const float scale = a.scale_log2e;
    const int G = tl.group;

    // LDS addresses in the first block: of the lane's row among 32 keys, chunk 2 ks + half (of ks = 0); of its place among 16 values (of dims 32 d, d = 0); where the
    // wave's loads go; and what a lane loads, in bytes from the wave's first row.  Chunk j (16 bytes) of row k lies at j ^ k % 16 (keys) or j ^ 4 (k % 4)
    // (values): what the lanes of a read touch together lies in different banks.
    uint32_t k_at, v_at, k_from, v_from;
    {
        const int g = lane >> 4, c = lane & 15, v_row = 4 * half + (c >> 2);
        k_at = ring + (lane & 31) * 256 + ((half ^ c) << 4);
        v_at = ring + kPiece + v_row * 256 + (((2 * (g & 1) + ((c & 3) >> 1)) ^ ((v_row & 3) << 2)) << 4) + (c & 1) * 8;
        k_from = g * 256 + ((c ^ (8 * (wave & 1) + g)) << 4);
        v_from = g * 256 + ((c ^ (g << 2)) << 4);
    }
    const uint32_t wave_at = ring + 8 * wave * 256;

    long long x = share * line.share;
    const long long x_end = min(x + line.share, line.all);
    Cut cut{};
    Segment seg;
    for (bool known = false; x < x_end; known = true, x = seg.next) {
        segment_at<false>(a, tl, line, x, x_end, known, &seg);
        const Item& it = seg.it;
        const int h = seg.h, first = seg.first, last = seg.last;
        if (first == last) continue;                       // (the share ends among the places in front)
        const bool whole = first == it.b0 && last == it.b1;

        // this lane's query row
        const int tile_rows = min(it.rows.n - it.tile * tl.tokens, tl.tokens) * G;
        const int r = min(wave * 32 + (lane & 31), tile_rows - 1);
        const int in_tile = token_of_row(tl, r), i = it.tile * tl.tokens + in_tile, head = h * G + r - in_tile * G;
        const int position = it.rows.base + i;
        const bool active = wave * 32 < tile_rows;
        const int pos_min = lane_value(position, 0), pos_max = lane_value(position, 31);
        bf16x8 q[8];
        {
            const uint4* from = reinterpret_cast<const uint4*>(a.q + (long long)(it.rows.q0 + i) * a.q_stride + (long long)head * kHeadDim);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) q[ks] = __builtin_bit_cast(bf16x8, from[2 * ks + half]);
        }

        // Loading: a wave brings rows 8 wave .. + 7 of a block, two times two instructions of four rows.  Pages of eight rows or more hold all of them, so their
        // address is a scalar.
        const int32_t* entries = a.c.table + (long long)it.b * a.c.table_stride;
        typedef const __attribute__((address_space(4))) int32_t constant_int;
        const int end = min(it.rows.base + it.rows.n, room_of(a));       // keys of the sequence
        // What a wave needs to know of the rows that it loads: the entry (or, for small pages, one of each row in lanes 8 r ..).
        auto entry_at = [&](int block) {
            const int key = block * kKeys + 8 * wave;
            if constexpr (kOnePage) return (int)((constant_int*)entries)[min(key, end - 1) >> a.c.page_shift];
            else return (int)entries[min(key + (lane >> 3), end - 1) >> a.c.page_shift];
        };
        // A bit for each of them that is there.
        auto bits_of = [&](int block, int entry) {
            const int n = end - (block * kKeys + 8 * wave);
            const uint32_t in = n >= 8 ? 255u : n > 0 ? (1u << n) - 1u : 0u;
            if constexpr (kOnePage) return (uint32_t)__builtin_amdgcn_readfirstlane(entry) < (uint32_t)a.c.n_pages ? in : 0u;
            const unsigned long long ok = __ballot((uint32_t)entry < (uint32_t)a.c.n_pages);
            uint32_t held = 0;
#pragma unroll
            for (int r = 0; r < 8; ++r) held |= (uint32_t)(ok >> (8 * r) & 1) << r;
            return in & held;
        };
        // Four instructions, two of keys and two of values; rows that are not there: those of page 0.
        struct Rows {
            const unsigned char *k[2], *v[2];      // from here, a lane each
            uint32_t to;
        };
        auto rows_at = [&](int block, int place, int entry, uint32_t bits) {
            const int key = block * kKeys + 8 * wave;
            Rows r;
            r.to = wave_at + (uint32_t)((place & (kRing - 1)) * kBlockBytes);
            lds_write1(valid_at + (uint32_t)((place & (kRing - 1)) * kWaves + wave), bits);
            if constexpr (kOnePage) {
                const int page = bits ? __builtin_amdgcn_readfirstlane(entry) : 0;
                const long long at = row_of(page, h, a.c.n_kv, a.c.page_shift, key) * 256;
                r.k[0] = r.k[1] = reinterpret_cast<const unsigned char*>(a.c.K) + at;
                r.v[0] = r.v[1] = reinterpret_cast<const unsigned char*>(a.c.V) + at;
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int n = 4 * e + (lane >> 4), page = __shfl(entry, 8 * n, 64);
                    const long long at = row_of((bits >> n & 1) ? page : 0, h, a.c.n_kv, a.c.page_shift, key + n) * 256 - n * 256;
                    r.k[e] = reinterpret_cast<const unsigned char*>(a.c.K) + at;
                    r.v[e] = reinterpret_cast<const unsigned char*>(a.c.V) + at;
                }
            }
            return r;
        };
        auto load = [&](const Rows& r, int i) {
            if (i == 0) load_to_lds(r.k[0] + k_from, r.to);
            if (i == 1) load_to_lds(r.k[1] + ((k_from ^ 64u) + 1024u), r.to + 1024);
            if (i == 2) load_to_lds(r.v[0] + v_from, r.to + kPiece);
            if (i == 3) load_to_lds(r.v[1] + (v_from + 1024u), r.to + kPiece + 1024);
        };
        auto load_all = [&](const Rows& r) {
#pragma unroll
            for (int i = 0; i < 4; ++i) load(r, i);
        };
        // Blocks in which some row of the item sees a key that another one does not: those from edge_from on, and with a window those up to edge_upto.
        const int low = it.rows.base + it.tile * tl.tokens, high = it.rows.base + min(it.rows.n, (it.tile + 1) * tl.tokens) - 1;
        const int edge_from = low < 0 ? -1 : (low + 1) / kKeys, edge_upto = a.window && high >= a.window ? (high - a.window) / kKeys : -1;
        auto edge = [&](int block) { return block >= edge_from || block <= edge_upto; };
        // When the wave's rows of a block have come: values of rows that are not there are zeroed (a probability of zero meets them), and so are those of an
        // edge's block that are not finite, lest they meet the zero of a row that does not see them.
        auto arrived = [&](int block, uint32_t bits) {
            uint32_t odd = 0;
            const bool at_edge = edge(block);
            if (bits != 255u || at_edge) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t at = wave_at + (uint32_t)((block & (kRing - 1)) * kBlockBytes) + kPiece + e * 1024 + lane * 16;
                    u32x4 w = lds_read16(at);
                    bool off_range = false;
                    if (!(bits >> (4 * e + (lane >> 4)) & 1)) {
                        w = u32x4{0u, 0u, 0u, 0u};
                    } else if (at_edge) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const bool lo = (w[k] & 0x7f80u) == 0x7f80u, hi = (w[k] & 0x7f800000u) == 0x7f800000u;
                            off_range |= lo | hi;
                            w[k] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
                        }
                    }
                    lds_write16(at, w);
                    const unsigned long long in = __ballot(off_range);
#pragma unroll
                    for (int k = 0; k < 4; ++k) odd |= (uint32_t)((in >> (16 * k) & 0xffff) != 0) << (4 * e + k);
                }
            }
            if (at_edge) {
                lds_write1(odd_at + (uint32_t)((block & (kRing - 1)) * kWaves + wave), odd);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
        };

        Softmax st;
        st.m = -INFINITY;
        st.l = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int j = 0; j < 16; ++j) st.o[d][j] = 0.f;

        if (end > 0) {
            // what the wave knows of the rows on their way, a block ahead and more
            uint32_t bits1, bits2, bits3 = 0;
            int entry = entry_at(first);
            const int entry1 = entry_at(min(first + 1, last - 1)), entry2 = entry_at(min(first + 2, last - 1));
            workgroup_sync();                              // (the item before is done with LDS)
            bits1 = bits_of(first, entry);
            load_all(rows_at(first, first, entry, bits1));
            int block = min(first + 1, last - 1);
            bits2 = bits_of(block, entry1);
            load_all(rows_at(block, first + 1, entry1, bits2));
            block = min(first + 2, last - 1);
            entry = entry2;
            wait_vm<0>();
            arrived(first, bits1);
            if (first + 1 < last) arrived(first + 1, bits2);
            workgroup_sync();
            for (int t = first; t < last; ++t) {
                const uint32_t slot = (uint32_t)((t & (kRing - 1)) * kBlockBytes);
                // Waves meet behind every second block (behind each: 4.34 ms for 2048 tokens at 128K, now 4.27); block t + 2 takes the place of one that all of them were done with then.
                // A wave's four loads are spread over its products: eight waves' loads take the memory path some 500 cycles, in which a wave that asks for more has to stand.
                bits2 = bits3;
                // (Past the share's end the last block is loaded again: a branch for that would cut the products' code into pieces.)
                bits3 = bits_of(block, entry);
                const Rows coming = rows_at(block, t + 2, entry, bits3);
                block = min(t + 3, last - 1);
                entry = entry_at(block);
                // (with this as the `else` of what follows, its state was copied at the end of both, and registers ran out)
                const bool sees_some = active && t * kKeys <= pos_max;
                if (!sees_some) load_all(coming);
                if (sees_some) {
                // (keys and values are read a half at a time: with all of a block's keys at once, registers run out)
                bf16x8 k[8];
                read_keys(k, k_at, slot);
                f32x16 s[2];
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int j = 0; j < 16; ++j) s[tt][j] = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (i == 8) read_keys(k, k_at ^ 128u, slot);
                    s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[i & 7], q[i >> 1], s[i & 1], 0, 0, 0);
                    if ((i & 3) == 1) {
                        __builtin_amdgcn_sched_barrier(0);
                        load(coming, i >> 2);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                s16x4 v[16];
                read_values(v, v_at, slot);
                const unsigned long long valid = lds_read8(valid_at + (uint32_t)((t & (kRing - 1)) * kWaves));
                const bool masked = valid != ~0ull || t * kKeys + kKeys - 1 > pos_min || (a.window && t * kKeys <= pos_max - a.window);
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
                float part[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) part[j] = larger(s[0][j], s[1][j], top);
#pragma unroll
                for (int j = 4; j < 16; ++j) part[j & 3] = fmaxf(part[j & 3], larger(s[0][j], s[1][j], top));
                float mx = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
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
                // Probabilities of 16 keys at a time, two elements behind each product of the 16 keys before.  Each is rounded to bf16 once (2^-8, as much as the results are). In two
                // parts (2^-15, as for single tokens) they take half as many products again: 2048 tokens at 128K 5.64 ms for 4.24, a prompt of 8192 in groups of five 0.93 for 0.74,
                // fifteen tokens beside 333 of a prompt 116 us for 98.
                bf16x8 p[4];
                auto probabilities = [&](int k, int e) {
#pragma unroll
                    for (int j = e; j < e + 2; ++j) {
                        const float x = __builtin_amdgcn_exp2f(fmaf(s[k >> 1][8 * (k & 1) + j], scale, -m));
                        st.l += x;
                        p[k][j] = (__bf16)x;
                    }
                };
#pragma unroll
                for (int e = 0; e < 8; e += 2) probabilities(0, e);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (i == 8) read_values(v, v_at, slot + 8192u);
                    const auto w = __builtin_shufflevector(v[2 * (i & 7)], v[2 * (i & 7) + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                    st.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), p[i >> 2], st.o[i & 3], 0, 0, 0);
                    if (i < 12) probabilities((i >> 2) + 1, 2 * (i & 3));
                    __builtin_amdgcn_sched_barrier(0);
                }
                // Values that are not finite have been taken out of an edge's block, lest they meet the zero of a row that does not see them: they are
                // added to the rows that do.
                if (edge(t)) {
                    for (unsigned long long odd = lds_read8(odd_at + (t & (kRing - 1)) * kWaves); odd; odd &= odd - 1) {
                        const int key = t * kKeys + __ffsll((long long)odd) - 1;
                        const int page = __builtin_amdgcn_readfirstlane(page_of(entries, a.c.table_stride, a.c.n_pages, a.c.page_shift, key));
                        const bool sees = key <= position && !(a.window && key <= position - a.window);
                        const uint2* from = reinterpret_cast<const uint2*>(a.c.V + row_of(max(page, 0), h, a.c.n_kv, a.c.page_shift, key) * kHeadDim);
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
                if ((t - first) & 1) {
                    wait_vm<0>();
                    if (t + 1 < last) arrived(t + 1, bits2);
                    if (t + 2 < last) arrived(t + 2, bits3);
                    workgroup_sync();
                }
            }
            wait_vm<0>();
        }

        const float l = over_halves_sum(st.l);
        if (whole) store_rows(a, st, l, it.rows.q0 + i, head, wave * 32 + (lane & 31) < tile_rows);
        else {
            if (active) store_part(parts + (2ll * share + slot_of(blocks_from(it, line, h), share, line.share)) * kPartFloats, st, l);
            if (last < it.b1) cut = cut_of(it, tl, line, share, h);
        }
    }
    if (threadIdx.x == 0) cuts[share] = cut;
}

// One wave a cut, 32 rows and 32 dims.
__global__ __launch_bounds__(64) void paged_chunk_merge_kernel(PagedAttention a, int group, const float* parts, const Cut* cuts)
{
    const int share = blockIdx.x >> 5, wave = (blockIdx.x >> 2) & 7, d = blockIdx.x & 3, lane = threadIdx.x, half = lane >> 5;
    const Cut c = cuts[share];
    if (c.parts == 0 || wave * 32 >= c.rows) return;
    auto part = [&](int g) { return parts + (2ll * (share + g) + (g == 0 ? c.slot : 0)) * kPartFloats; };
    const int at_m = kRows * kHeadDim + wave * 32 + (lane & 31);
    float m = -INFINITY;
#pragma unroll 4
    for (int g = 0; g < c.parts; ++g) m = fmaxf(m, part(g)[at_m]);
    const float ms = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int g = 0; g < c.parts; ++g) {
        const float* p = part(g);
        const float f = __builtin_amdgcn_exp2f(p[at_m] - ms);
        l = fmaf(p[at_m + kRows], f, l);
        const f32x4* from = reinterpret_cast<const f32x4*>(p) + (wave * 16 + 4 * d) * 64 + lane;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4 w = from[j * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][e] = fmaf(w[e], f, o[j][e]);
        }
    }
    const int r = wave * 32 + (lane & 31);
    if (r >= c.rows) return;
    const long long row = (long long)(c.q0 + r / group) * a.n_q_heads + c.head * group + r % group;
    store_dims(a, row, d, half, o, l);
    if (a.lse && d == 0 && half == 0) a.lse[row] = lse_of(m, l);
}

constexpr size_t kCutFloats = sizeof(Cut) / sizeof(float) * kWorkgroups;

}  // namespace

size_t paged_chunk_floats() { return (size_t)2 * kWorkgroups * kPartFloats + kCutFloats; }

hipError_t launch_paged_chunks(const PagedAttention& a, int over, float* room, hipStream_t s)
{
    const Tiling tl = tiling(a.n_q_heads / a.c.n_kv, kRows, over, 0x7fffffff, kKeys, 3, 4);
    Cut* cuts = reinterpret_cast<Cut*>(room);
    float* parts = room + kCutFloats;
    const auto kernel = a.c.page_shift >= 3 ? paged_chunk_kernel<true> : paged_chunk_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3(kWorkgroups), dim3(64 * kWaves), 0, s, a, tl, parts, cuts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_chunk_merge_kernel, dim3(32 * kWorkgroups), dim3(64), 0, s, a, tl.group, (const float*)parts, (const Cut*)cuts);
    return hipGetLastError();
}

}  // namespace mp
