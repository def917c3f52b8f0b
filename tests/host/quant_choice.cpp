// Lines of "M N K entries" (entries of a row-tile list, -1: no list) in, and the 8-bit GEMM's choice of
// kernel for each out: kind (0 few rows, 1 tiles, 2 192 x 192, 3 192 x 256, 4 256 x 256), tile or column
// blocks, shares of K, leading 256-row tiles.  32 CUs an XCD.
#include <cstdio>

#include "gemm_quant_choice.h"

int main() {
    int M, N, K, list;
    while (std::scanf("%d %d %d %d", &M, &N, &K, &list) == 4) {
        const ppk::QuantChoice c = ppk::quant_choose(M, N, K, list, 32);
        std::printf("%d %d %d %d\n", static_cast<int>(c.kind), c.tile, c.splits, c.big);
    }
}
