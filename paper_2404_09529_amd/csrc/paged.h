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

// The split of the attention.  A step is kPagedStep keys of one sequence for one key/value head, the work of one
// wavefront; all S steps of all sequences, one sequence after the other, are dealt to W ranges of equal length, range w
// starting with step w S / W, and a wavefront has one range of one head.
constexpr int kPagedStep = 32, kPagedWaves = 8;   // keys; wavefronts of a workgroup
constexpr int32_t paged_steps(int32_t len) { return len / kPagedStep + (len % kPagedStep != 0); }
// (Operands fit 63 bits: a sequence has at most 2^26 steps, there are at most 2^22 sequences and 2^14 ranges.)
constexpr int64_t paged_quotient(int64_t a, int64_t b) {
    return (uint64_t(a) | uint64_t(b)) >> 32 ? int64_t(uint64_t(a) / uint64_t(b)) : int64_t(uint32_t(a) / uint32_t(b));
}
constexpr int64_t paged_start(int32_t w, int64_t S, int32_t W) { return paged_quotient(w * S, W); }
// The range that holds step s.
constexpr int32_t paged_range(int64_t s, int64_t S, int32_t W) {
    return static_cast<int32_t>(paged_quotient((s + 1) * W - 1, S));
}

// Workgroups and ranges for `heads` key/value heads (each counted once per 16 query heads): about 256 workgroups.
constexpr int32_t paged_groups(int32_t heads) {
    return heads <= 256 * kPagedWaves ? 256 : (heads + kPagedWaves * 8 - 1) / (kPagedWaves * 8) * 8;
}
constexpr int32_t paged_ranges(int32_t heads) { return paged_groups(heads) * kPagedWaves / heads; }

// Workgroups are dealt to the 8 XCDs in turn.  Wavefronts side by side have neighbouring heads of one range, whose
// rows lie side by side in memory, and an XCD has consecutive ranges.  Range and head of wavefront `wave` of workgroup b
// of n (a multiple of 8); range >= W: none.
struct PagedPlace {
    int32_t range, head;
};
constexpr PagedPlace paged_place(uint32_t b, uint32_t n, uint32_t wave, int32_t heads) {
    const uint32_t q = (b % 8 * (n / 8) + b / 8) * kPagedWaves + wave;
    return {static_cast<int32_t>(q / heads), static_cast<int32_t>(q % heads)};
}

}  // namespace ppk
