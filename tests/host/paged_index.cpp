// Asks csrc/paged.h on the CPU.  Lines in:
//   split W len len ...   -> of every range its first step, then -1 and for every sequence with keys the ranges of its
//                            first and last step
//   places heads          -> groups, ranges, then "range head" of every wavefront of the grid
//   rows n_pages shift max_pages page ...  (one sequence's table) -> row of every position up to the span + 2
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>
#include <vector>

#include "paged.h"

using namespace ppk;

int main() {
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        std::string what;
        in >> what;
        if (what == "split") {
            int W, n;
            in >> W;
            std::vector<int> steps;
            int64_t S = 0;
            while (in >> n) steps.push_back(paged_steps(n)), S += steps.back();
            for (int w = 0; w <= W; ++w) std::printf("%lld ", static_cast<long long>(paged_start(w, S, W)));
            std::printf("-1 ");
            int64_t s0 = 0;
            for (int t : steps) {
                if (t) std::printf("%d %d ", paged_range(s0, S, W), paged_range(s0 + t - 1, S, W));
                s0 += t;
            }
            std::printf("\n");
        } else if (what == "places") {
            int heads;
            in >> heads;
            const int n = paged_groups(heads);
            std::printf("%d %d ", n, paged_ranges(heads));
            for (int b = 0; b < n; ++b)
                for (int w = 0; w < kPagedWaves; ++w) {
                    const PagedPlace p = paged_place(b, n, w, heads);
                    std::printf("%d %d ", p.range, p.head);
                }
            std::printf("\n");
        } else {
            int n_pages, shift, max_pages, page;
            in >> n_pages >> shift >> max_pages;
            std::vector<int> table;
            while (in >> page) table.push_back(page);
            const int span = paged_span(max_pages, shift);
            for (int pos = -1; pos < span + 2; ++pos) {
                const bool in_table = pos >= 0 && pos < paged_len(span + 1, span);
                std::printf("%d ", in_table ? paged_row(table[pos >> shift], n_pages, pos, shift) : -1);
            }
            std::printf("%d %d %d\n", paged_len(-3, span), paged_len(0, span), paged_len(0x7fffffff, span));
        }
    }
}
