// Where the keys of a paged cache are and which of them a tile of rows sees: the integer arithmetic of the paged attention kernels, for host and device.
#pragma once
#include <cstdint>

#include "opmap.h"

namespace nt {

// n / d for 0 <= n < 2^31 as a product and a shift: with s = ceil(log2 d), m = ceil(2^(31 + s) / d) fits 32 bits and m d - 2^(31 + s) < d <= 2^s,
// so that n m / 2^(31 + s) is above n / d by less than 1 / d.
struct Divider {
    uint32_t m;
    int32_t shift;
    uint32_t d;
};
inline Divider divider_of(uint32_t d)
{
    int s = 0;
    while ((1ull << s) < d) ++s;
    return Divider{(uint32_t)(((1ull << (31 + s)) + d - 1) / d), 31 + s, d};
}
NT_HD uint32_t divide(uint32_t n, const Divider &d) { return (uint32_t)(((uint64_t)n * d.m) >> d.shift); }

NT_HD int32_t clamp_i32(int32_t v, int32_t lo, int32_t hi) { return v < lo ? lo : v > hi ? hi : v; }

// Positions end here: the ends of blocks, and keys that are looked up ahead of their block, are below 2^31 too.
constexpr int32_t kMostKeys = 0x7fffffff - 4095;

// Entries of a table row, `width` long, that name positions below kMostKeys
inline int32_t entries_in_reach(int64_t width, uint32_t page_size)
{
    const int64_t most = kMostKeys / page_size;
    return (int32_t)(width < most ? width : most);
}

// A sequence: its first row of the queries, its new tokens, its tokens in the cache (with the new ones)
struct Sequence {
    int32_t first, count, length;
};
// ... number b.  Whatever the arrays hold, [first, first + count) lies inside [0, T], and the length is at most what no table reaches.
NT_HD Sequence sequence_at(const int32_t *starts, const int32_t *lengths, int b, int32_t T)
{
    const int32_t s0 = clamp_i32(starts[b], 0, T), s1 = clamp_i32(starts[b + 1], s0, T), n = lengths[b];
    return Sequence{s0, s1 - s0, clamp_i32(n, 0, kMostKeys + 1)};
}

// The keys that token i of the sequence sees, [lo, hi) (none if hi <= lo).  Its position is length - count + i; negative where the length is too small
// for the new tokens.
struct KeyRange {
    int32_t lo, hi;
};
NT_HD KeyRange keys_seen(const Sequence &q, int32_t i, int32_t causal, int32_t window)
{
    const int32_t pos = q.length - q.count + i;
    return KeyRange{window && pos >= window ? pos - window + 1 : 0, causal && pos + 1 < q.length ? pos + 1 : q.length};
}

// The keys [lo, hi) inside the sequence that some of tokens i0 .. i1 sees, and of them share number `split` of `splits`: share_keys each (the last: what is
// left), from the first key on, rounded down to a multiple of `block`.  Of the positions from `capacity` on, which the table has no entry for, a token that sees any
// needs one to show it: the first that it sees.  The range ends behind those, however long the sequence is said to be.
NT_HD KeyRange key_range(const Sequence &q, int32_t i0, int32_t i1, int32_t causal, int32_t window, int split, int splits, int32_t share_keys, int32_t block,
                         int32_t capacity = kMostKeys)
{
    int32_t lo = keys_seen(q, i0, causal, window).lo, hi = keys_seen(q, i1, causal, window).hi;
    const int32_t last = keys_seen(q, i1, causal, window).lo, enough = last > capacity ? last : capacity;
    hi = hi > enough ? enough + 1 : hi;
    lo = lo > 0 ? lo : 0;
    hi = hi > 0 ? hi : 0;
    if (splits > 1) {
        const int64_t base = lo / block * block, from = base + (int64_t)split * share_keys, to = from + share_keys;
        if (split > 0 && from > lo) lo = from > hi ? hi : (int32_t)from;
        if (split + 1 < splits && to < hi) hi = (int32_t)to;
    }
    return KeyRange{lo, hi < lo ? lo : hi};
}

// ---- trees of drafted tokens: token i sees the positions before the new ones, `past` = length - count of them (a window: the last ones, counted from past + its
// depth), and of position past + k it sees what bit k of its mask says.

// bits [from, to) of 64
NT_HD uint64_t bits_between(int32_t from, int32_t to)
{
    const uint64_t below = from <= 0 ? 0ull : from >= 64 ? ~0ull : (1ull << from) - 1, under = to <= 0 ? 0ull : to >= 64 ? ~0ull : (1ull << to) - 1;
    return under & ~below;
}

// 64 bits of a mask of `words` words, from bit `at` on (before the first bit and behind the last there are zeros)
NT_HD uint64_t bits_from(const uint64_t *mask, int32_t words, int32_t at)
{
    const int32_t w = at >> 6, s = at & 63;
    const uint64_t lo = (uint32_t)w < (uint32_t)words ? mask[w] : 0, hi = s && (uint32_t)(w + 1) < (uint32_t)words ? mask[w + 1] : 0;
    return s ? lo >> s | hi << (64 - s) : lo;
}

// The first position that a token of this depth (0 to count - 1) sees of the past
NT_HD int32_t tree_row_lo(int32_t past, int32_t count, int32_t depth, int32_t window)
{
    const int64_t lo = (int64_t)past + clamp_i32(depth, 0, count - 1) - window + 1;
    return window && lo > 0 ? (int32_t)(lo < past ? lo : past) : 0;
}

// Which of the 64 positions from `base` (0 <= base < length) on the token sees; row_lo: as above
NT_HD uint64_t tree_keys(const uint64_t *mask, int32_t words, int32_t base, int32_t row_lo, int32_t past, int32_t length)
{
    const uint64_t before = past > 0 ? bits_between(row_lo > base ? (row_lo - base < 64 ? row_lo - base : 64) : 0, past > base ? (past - base < 64 ? past - base : 64) : 0) : 0;
    if (past >= 64 && base <= past - 64) return before;
    const int32_t first = past - base, end = length - base < 64 ? length - base : 64;             // (base < length <= past + new tokens: both fit)
    return before | (bits_from(mask, words, -first) & bits_between(first, end));
}

// The keys that some token of a tree may see.  Where the past passes what the table reaches, whoever sees anything sees a position without a page among the last of the past and
// the new ones: no others are needed to show it.
NT_HD KeyRange tree_range(const Sequence &q, int32_t window, int32_t capacity)
{
    const int32_t past = q.length - q.count;
    return KeyRange{past > capacity ? past - 1 : window && past >= window ? past - window + 1 : 0, q.length};
}

// ... in blocks of `block` keys; tokens that see nothing have a block too
NT_HD int32_t tree_blocks(const Sequence &q, int32_t window, int32_t block, int32_t capacity)
{
    if (q.count == 0) return 0;
    const KeyRange k = tree_range(q, window, capacity);
    const int32_t n = k.lo < k.hi ? (k.hi - 1) / block + 1 - k.lo / block : 0;
    return n > 0 ? n : 1;
}

// Blocks [from, to) of it
NT_HD KeyRange tree_part(const KeyRange &k, int32_t block, int32_t blocks, int32_t from, int32_t to)
{
    const int32_t first = k.lo / block;
    return KeyRange{from ? (first + from) * block : k.lo, to < blocks ? (first + to) * block : k.hi};
}

// The page of a position, in two steps: its entry of the table row is on its way long before the page is needed.
// Which entry is read for number `index`: past the row's end its last, which is not used then (of a row without entries the first: the launcher puts something
// to read in its place)
NT_HD uint32_t entry_read(uint32_t index, int32_t width) { return index < (uint32_t)width ? index : width > 0 ? (uint32_t)width - 1 : 0; }
// Whether `id`, read so, names a page of the cache for entry `index`
NT_HD bool names_page(uint32_t index, int32_t id, int32_t width, int32_t pages) { return index < (uint32_t)width && (uint32_t)id < (uint32_t)pages; }
// Both steps: the page, -1 if none is named (the kernels take them apart; host checks call this)
NT_HD int32_t page_at(const int32_t *row, uint32_t index, int32_t width, int32_t pages)
{
    if (width <= 0) return -1;
    const int32_t id = row[entry_read(index, width)];
    return names_page(index, id, width, pages) ? id : -1;
}

// Tiles of `rows` (token, query head) rows, `group` heads to a token: sequence b's are numbered from here on.  Rounding the rows before it down and adding b
// leaves room for each sequence's last, unfilled one: ceil(x) <= floor(a + x) - floor(a) + 1.
NT_HD int32_t first_tile(const int32_t *starts, int b, int32_t T, int32_t group, int32_t rows)
{
    return (int32_t)(((int64_t)clamp_i32(starts[b], 0, T) * group) / rows) + b;
}

}  // namespace nt
