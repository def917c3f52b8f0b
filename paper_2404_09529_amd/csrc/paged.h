// Where the tokens of a paged cache lie, and how the attention over them is split: index arithmetic
// that the kernels, the entry points and a test on the CPU share.
#pragma once
#include <stdint.h>

namespace ppk {

// Row of the pool that page `page` (an entry of a page table) holds for position `pos`; -1: none, the page
// is not one of the pool's.  n_pages << shift fits 31 bits.
constexpr int32_t paged_row(int32_t page, int32_t n_pages, int32_t pos, int shift) {
    return page >= 0 && page < n_pages ? (page << shift) | (pos & ((1 << shift) - 1)) : -1;
}

// Positions that a table of max_pages entries reaches, at most INT32_MAX.
constexpr int32_t paged_span(int32_t max_pages, int shift) {
    return (int64_t(max_pages) << shift) > INT32_MAX ? INT32_MAX : max_pages << shift;
}

// Keys that a sequence of stated length has in reach of its table.
constexpr int32_t paged_len(int32_t len, int32_t span) { return len < 0 ? 0 : len < span ? len : span; }

// The split of the attention.  A tile is kPagedTile keys, a step of a workgroup.  With T tiles in all sequences,
// every sequence is cut into units of `unit` = ceil(T / target) tiles (`least` at least), the last one shorter; a
// sequence without keys has one unit, which writes its zeros.  All sequences together have at most target + k units.
constexpr int kPagedTile = 128;
constexpr int32_t paged_tiles(int32_t len) { return len / kPagedTile + (len % kPagedTile != 0); }
constexpr int32_t paged_unit(int64_t tiles, int32_t target, int32_t least) {
    const int64_t unit = (tiles + target - 1) / target;
    return unit < least ? least : static_cast<int32_t>(unit);
}
constexpr int32_t paged_units(int32_t tiles, int32_t unit) { return tiles <= unit ? 1 : (tiles + unit - 1) / unit; }

// Workgroups are dealt to the 8 XCDs in turn.  All heads of a unit go to one XCD: the keys of neighbouring heads
// lie side by side in a row, and an XCD's L2 then fetches whole rows.  Unit and head of workgroup b:
struct PagedPlace {
    int32_t unit, head;
};
constexpr PagedPlace paged_place(uint32_t b, int32_t heads) {
    return {static_cast<int32_t>(b / 8 / heads * 8 + b % 8), static_cast<int32_t>(b / 8 % heads)};
}

}  // namespace ppk
