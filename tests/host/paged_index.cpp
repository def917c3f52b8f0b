// Asks csrc/paged.h on the CPU.  Lines in:
//   split target least heads len len ...   -> for every workgroup of the grid that has work: "seq head tile0 tile1 units"
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
            int target, least, heads, n;
            in >> target >> least >> heads;
            std::vector<int> tiles;
            int64_t all = 0;
            while (in >> n) tiles.push_back(paged_tiles(n)), all += tiles.back();
            const int unit = paged_unit(all, target, least);
            const uint32_t bound = target + tiles.size();
            for (uint32_t b = 0; b < (bound + 7) / 8 * 8 * heads; ++b) {
                const PagedPlace p = paged_place(b, heads);
                int first = 0;
                for (size_t i = 0; i < tiles.size(); ++i) {
                    const int u = paged_units(tiles[i], unit);
                    if (p.unit >= first && p.unit < first + u) {
                        const int t0 = (p.unit - first) * unit;
                        std::printf("%zu %d %d %d %d ", i, p.head, t0, std::min(t0 + unit, tiles[i]), u);
                    }
                    first += u;
                }
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
