// How attention over a paged cache is shared out: device code of mp_paged_chunk.hip and mp_paged_token.hip.
//
// A sequence's query rows of one KV head are its new tokens times the G heads of the group, token after token.  An item is a tile of such rows
// with the blocks of keys that some of them attend.  All items' blocks, head after head, sequence after sequence, are one line that is cut into equal
// shares, a workgroup each: lengths are known on the device only, and one long sequence among short ones, or few rows over many keys,
// come out even.  In front of its blocks an item has some places that stand for its beginning and end (the first loads, the results), so that shares of
// many short items do not take longer (a prompt of 8192 in groups of five: 813 us with one place, 751 with three).  An item within a share is finished there; one that is cut leaves its parts (maximum, sum and weighted values, in fp32) in the
// workspace for the launch behind.
#pragma once
#include "mp_device.h"
#include "mp_paged.h"

namespace mp {

namespace {

// The larger of two numbers, `top` being infinity as a value that the compiler does not know.  (Of products of the matrix cores, fmaxf first takes each through an
// instruction of its own, lest it be a signalling NaN.)
__device__ __forceinline__ float larger(float a, float b, float top) { return __builtin_amdgcn_fmed3f(a, b, top); }
__device__ __forceinline__ float hidden_infinity()
{
    float top = INFINITY;
    asm volatile("" : "+s"(top));
    return top;
}

// A sequence is an item's if it has more than `over` and at most `most` rows.
struct Tiling {
    int group;                // G
    int tokens;               // of a tile
    int over, most;
    int unit;                 // keys of a block
    int ahead;                // places in front of an item's blocks
    int least;                // places of a share, at least
    int inverse;              // row / group = row * inverse >> 16 for the rows of a tile
};
constexpr int kWorkgroups = 256;
inline Tiling tiling(int group, int rows, int over, int most, int unit, int ahead, int least)
{
    return Tiling{group, rows / group, over, most, unit, ahead, least, 65536 / group + 1};
}
__device__ __forceinline__ int token_of_row(const Tiling& tl, int row) { return row * tl.inverse >> 16; }

struct SequenceRows {
    int q0, n, base;          // first token, tokens, position of the first
};

__device__ __forceinline__ SequenceRows rows_of_sequence(const PagedAttention& a, int b)
{
    const int s0 = a.c.q_start[b], s1 = a.c.q_start[b + 1];
    SequenceRows r;
    r.q0 = min(max(s0, 0), a.n_tokens);
    r.n = min(min(max(s1, r.q0), a.n_tokens) - r.q0, a.max_new);
    r.base = a.c.kv_len[b] - (s1 - s0);
    return r;
}

// Of sequence s0 + lane.
__device__ __forceinline__ SequenceRows rows_of_lane(const PagedAttention& a, int s0)
{
    const int b = s0 + (threadIdx.x & 63);
    return b < a.c.n_seqs ? rows_of_sequence(a, b) : SequenceRows{0, 0, 0};
}

struct Item {
    int b, tile;
    SequenceRows rows;
    int b0, b1;               // its blocks
    uint32_t before;          // places of the items before it (of one head)
};

__device__ __forceinline__ int room_of(const PagedAttention& a) { return a.c.table_stride << a.c.page_shift; }

__device__ __forceinline__ void blocks_of_tile(const PagedAttention& a, const Tiling& tl, const SequenceRows& r, int tile, int* b0, int* b1)
{
    const int i0 = tile * tl.tokens;
    blocks_of(r.base, i0, min(r.n, i0 + tl.tokens) - 1, a.window, room_of(a), tl.unit, b0, b1);
}
// (of a tree: from the older keys that a window leaves a token without marks, to the last new one, whichever the tile)
__device__ __forceinline__ void blocks_of_tile(const PagedTreeAttention& a, const Tiling& tl, const SequenceRows& r, int, int* b0, int* b1)
{
    blocks_of(r.base - 1, 0, r.n, a.window, room_of(a), tl.unit, b0, b1);
}

// What a query row of a tree attends, see tree_keys.
struct TreeRow {
    const unsigned long long* mask;
    int low;
};
__device__ __forceinline__ TreeRow tree_row(const PagedTreeAttention& a, const SequenceRows& r, int i)
{
    const unsigned long long* mask = a.mask + (long long)(r.q0 + i) * a.words;
    return TreeRow{mask, tree_low(mask, a.words, r.base, r.n, a.window)};
}
// Keys of a sequence before `upto` are not seen by some of its rows (a window's), those from `from` on may be new ones; all rows see what lies between.
struct TreeEdges {
    int upto, from;
};
__device__ __forceinline__ TreeEdges tree_edges(const PagedTreeAttention& a, const SequenceRows& r)
{
    return TreeEdges{a.window > 0 ? r.base - max(a.window - r.n, 0) : 0, max(r.base, 0)};
}


__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ int tiles_of(const Tiling& tl, const SequenceRows& r)
{
    const long long rows = (long long)r.n * tl.group;
    return rows > tl.over && rows <= tl.most ? (r.n + tl.tokens - 1) / tl.tokens : 0;
}
// The item of lane `at`, whose places end at incl.
__device__ __forceinline__ void take_item(Item* it, int at, int b, int tile, const SequenceRows& r, int b0, int b1, uint32_t incl, int ahead)
{
    it->b = lane_value(b, at);
    it->tile = lane_value(tile, at);
    it->rows.q0 = lane_value(r.q0, at);
    it->rows.n = lane_value(r.n, at);
    it->rows.base = lane_value(r.base, at);
    it->b0 = lane_value(b0, at);
    it->b1 = lane_value(b1, at);
    it->before = (uint32_t)lane_value((int)incl, at) - (uint32_t)(ahead + it->b1 - it->b0);
}

// Returns the places of one head's items in all, `ahead` of them in front of each one's blocks (*items: how many there are); kFind: goes up to the item that
// place x of the line lies in, puts it into *found and returns x (anything else: there is none).  One wave, 64 sequences (or, where some have several tiles, 64 tiles) at a time.  `head`: rows_of_lane(a, 0).
template <bool kFind, class A>
__device__ __forceinline__ uint32_t walk(const A& a, const Tiling& tl, const SequenceRows& head, int ahead, uint32_t x, Item* found, uint32_t* items)
{
    const int lane = threadIdx.x & 63;
    uint32_t sum = 0;
    for (int s0 = 0; s0 < a.c.n_seqs; s0 += 64) {
        const SequenceRows r = s0 == 0 ? head : rows_of_lane(a, s0);
        const int tiles = tiles_of(tl, r);
        const bool several = __any(tiles > 1);
        const int upto = several ? (int)wave_incl_scan_u32((uint32_t)tiles) : 0;
        const int all = several ? lane_value(upto, 63) : 64;
        for (int c = 0; c < all; c += 64) {
            int k = lane, tile = 0;
            SequenceRows m = r;
            bool there = tiles > 0;
            if (several) {
                k = 0;
#pragma unroll
                for (int step = 32; step; step >>= 1)
                    if (__shfl(upto, k + step - 1, 64) <= c + lane) k += step;
                tile = c + lane - (__shfl(upto, k, 64) - __shfl(tiles, k, 64));
                m.q0 = __shfl(r.q0, k, 64);
                m.n = __shfl(r.n, k, 64);
                m.base = __shfl(r.base, k, 64);
                there = c + lane < all;
            }
            int b0 = 0, b1 = 0;
            if (there) blocks_of_tile(a, tl, m, tile, &b0, &b1);
            const uint32_t incl = wave_incl_scan_u32(there ? (uint32_t)(ahead + b1 - b0) : 0u);
            if constexpr (!kFind) *items += (uint32_t)__popcll(__ballot(there));
            if constexpr (kFind) {
                const unsigned long long past = __ballot(sum + incl > x);
                if (past) {
                    take_item(found, __ffsll((long long)past) - 1, s0 + k, tile, m, b0, b1, sum + incl, ahead);
                    return x;
                }
            }
            sum += (uint32_t)lane_value((int)incl, 63);
        }
    }
    return kFind ? x + 1 : sum;
}

// The line and its shares.  Neighbouring shares go to workgroups of one XCD: they mostly work on one head, whose keys its L2 then holds once.
struct Line {
    SequenceRows head;        // the lane's among the first 64 sequences: walks begin with them, and need not ask for them again
    uint32_t of_head;
    int ahead;
    long long all, share;
    int used;                 // workgroups with a share
    // The 64 sequences looked at, if none has more than one tile: the lane's blocks, and where its places end in the `total` of them behind the `before` of those
    // before s0.
    bool look;
    int s0, b0, b1;
    uint32_t before, total, incl;
};
// x / d (a head has fewer than 2^32 places, all of them together mostly)
__device__ __forceinline__ long long quotient(long long x, long long d)
{
    return ((x | d) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)d) : x / d;
}
// Looks at sequences s0 .., whose rows are in l->head.
template <class A>
__device__ __forceinline__ void look_at(const A& a, const Tiling& tl, Line* l, int s0, uint32_t before)
{
    const bool there = tiles_of(tl, l->head) > 0;
    l->s0 = s0;
    l->before = before;
    l->b0 = l->b1 = 0;
    if (there) blocks_of_tile(a, tl, l->head, 0, &l->b0, &l->b1);
    l->incl = wave_incl_scan_u32(there ? (uint32_t)(l->ahead + l->b1 - l->b0) : 0u);
    l->total = (uint32_t)lane_value((int)l->incl, 63);
}
// kSingle: no sequence of the tiling has more than one tile.
template <bool kSingle, class A>
__device__ __forceinline__ Line line_of(const A& a, const Tiling& tl)
{
    Line l;
    l.head = rows_of_lane(a, 0);
    l.ahead = 0;
    l.look = kSingle || (a.c.n_seqs <= 64 && !__any(tiles_of(tl, l.head) > 1));
    uint32_t items = 0;
    if (l.look) {
        l.of_head = 0;
        for (int s0 = 0;;) {
            look_at(a, tl, &l, s0, l.of_head);
            l.of_head += l.total;
            items += (uint32_t)__popcll(__ballot(l.b1 > l.b0));
            s0 += 64;
            if (s0 >= a.c.n_seqs) break;
            l.head = rows_of_lane(a, s0);
        }
    } else {
        l.of_head = walk<false>(a, tl, l.head, 0, 0, nullptr, &items);
    }
    // (where shares are a few blocks anyway, every workgroup is worth more than evenness)
    l.ahead = (long long)l.of_head * a.c.n_kv >= 8 * kWorkgroups ? tl.ahead : 0;
    l.of_head += (uint32_t)l.ahead * items;
    if (l.look && (l.ahead || l.s0)) {
        if (l.s0) l.head = rows_of_lane(a, 0);
        look_at(a, tl, &l, 0, 0);
    }
    l.all = (long long)l.of_head * a.c.n_kv;
    l.share = max((l.all + kWorkgroups - 1) / kWorkgroups, (long long)(tl.least + l.ahead));
    l.used = (int)quotient(l.all + l.share - 1, l.share);
    return l;
}
// The share of a workgroup; those from l.used on are empty.
__device__ __forceinline__ int share_of(const Line& l, int block)
{
    const int of_xcd = (l.used + 7) >> 3, xcd = block & 7, i = block >> 3;
    if (i < of_xcd) return xcd * of_xcd + i;
    return 8 * of_xcd + (i - of_xcd) * 8 + xcd;
}

// Where the line is at a place of it: the item, and the blocks of it that lie between that place and `end`.
struct Segment {
    Item it;
    int h, first, last;
    long long next;           // place behind it
};
__device__ __forceinline__ long long blocks_from(const Item& it, const Line& line, int h)
{
    return (long long)h * line.of_head + it.before + line.ahead;
}
// `known`: s->it is the item before, which ended at x.
template <bool kSingle, class A>
__device__ __forceinline__ void segment_at(const A& a, const Tiling& tl, Line& line, long long x, long long end, bool known, Segment* s)
{
    Item& it = s->it;
    bool found = true;
    if (!kSingle && known && (it.tile + 1) * tl.tokens < it.rows.n) {
        it.before += (uint32_t)(line.ahead + it.b1 - it.b0);
        blocks_of_tile(a, tl, it.rows, ++it.tile, &it.b0, &it.b1);
    } else {
        s->h = (int)quotient(x, line.of_head);
        const uint32_t of_this = (uint32_t)(x - (long long)s->h * line.of_head);
        if (line.look) {
            if constexpr (kSingle) {         // (from the sequences looked at last, or from the first)
                while (of_this < line.before || of_this - line.before >= line.total) {
                    const bool again = of_this < line.before;
                    const int s0 = again ? 0 : line.s0 + 64;
                    const uint32_t before = again ? 0 : line.before + line.total;
                    if (s0 >= a.c.n_seqs) break;
                    line.head = rows_of_lane(a, s0);
                    look_at(a, tl, &line, s0, before);
                }
            }
            found = of_this - line.before < line.total;
            const int at = found ? __ffsll((long long)__ballot(line.incl > of_this - line.before)) - 1 : 0;
            take_item(&it, at, line.s0 + (threadIdx.x & 63), 0, line.head, line.b0, line.b1, line.before + line.incl, line.ahead);
        } else {
            found = walk<true>(a, tl, line.head, line.ahead, of_this, &it, nullptr) == of_this;
        }
    }
    if (!found) {                            // (lengths that change under the launch: nothing is done for them, but it ends)
        s->first = s->last = 0;
        s->next = end;
        return;
    }
    const long long x0 = blocks_from(it, line, s->h), x1 = x0 + (it.b1 - it.b0);
    s->next = min(x1, end);
    s->first = it.b0 + (int)max(x - x0, 0ll);
    s->last = it.b0 + (int)max(s->next - x0, 0ll);
}

// An item that begins in a workgroup's share and ends in another one's, for the launch that puts its parts together: a line for each
// workgroup, written by it (parts == 0: none).
struct Cut {
    int parts;                // workgroups with a part of it, this one first
    int slot;                 // of this workgroup's part; the others' are their first
    int q0, rows, head;       // first token, query rows, KV head
    int unused[3];
};
__device__ __forceinline__ Cut cut_of(const Item& it, const Tiling& tl, const Line& line, int share, int h)
{
    const long long x0 = blocks_from(it, line, h);
    const Parts p = parts_of(x0, x0 + (it.b1 - it.b0), line.share);
    Cut c{};
    c.parts = p.first == share ? (int)(p.last - p.first) + 1 : 0;
    c.slot = slot_of(x0, share, line.share);
    c.q0 = it.rows.q0 + it.tile * tl.tokens;
    c.rows = min(it.rows.n - it.tile * tl.tokens, tl.tokens) * tl.group;
    c.head = h;
    return c;
}

}  // namespace
}  // namespace mp
