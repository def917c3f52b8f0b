// Which kernel of the 8-bit GEMM takes a call.  Host code without a GPU's headers, so that a program
// without one can ask it too.
#pragma once
#include <algorithm>
#include <cstdint>

constexpr int kQuantStep = 128;       // bytes (= values) of K in a step: whole cache lines, two MFMAs deep

namespace ppk {

constexpr int kQuantFewRows = 64;   // most rows of the kernel for few rows
constexpr int quant_few_waves(int blocks) { return blocks == 4 ? 4 : 8; }   // of a workgroup of `blocks` column blocks

// Tiles of the kernel for medium batches.
constexpr int kQuantTiles = 5;
constexpr int kQuantTileRows[kQuantTiles] = {32, 64, 64, 128, 128};
constexpr int kQuantTileCols[kQuantTiles] = {64, 64, 128, 128, 256};

template <typename T>
T quant_div(T a, int b) { return a / b + (a % b != 0); }

// Output tiles of the XCD that takes most, by either division of the tile list.
struct QuantXcdSplit {
    int balanced;
    int64_t tiles;
};
inline QuantXcdSplit quant_xcd_split(int tiles_m, int tiles_n, int wg_per_xcd) {
    const int64_t blocked = int64_t(quant_div(tiles_m, 8)) * tiles_n, even = quant_div(int64_t(tiles_m) * tiles_n, 8);
    const int balanced = quant_div(even, wg_per_xcd) < quant_div(blocked, wg_per_xcd) ? 1 : 0;
    return QuantXcdSplit{balanced, balanced ? even : blocked};
}

// Which kernel takes which rows.  An estimate in us, for the CU with the most tiles: a launch and its first
// loads, then each tile's steps of K and its epilogue; at least the time of the call's bytes at the
// memory's rate and of what the tiles fetch from L2 together.  The constants are fitted to timings of 340
// sizes (1 to 28,000 rows, N 256 to 28,800, K 256 to 14,400) on every kernel, half of them also with weights
// that come from memory instead of the last-level cache.  On 110 other sizes, with the kernels as they now
// stand, the choice costs 3% of the best kernel's time on average, 34% at worst.
// The 192-row tiles are for the rounds that 256 x 256 ones leave part empty: 2000 rows, N 4096, K 11008 in
// 242 of 192 x 192 83 us, in 128 of 256 x 256 113; 2926 rows, N 4096, K 14336 in 256 of 192 x 256 150 and 169 us.
struct QuantChoice {
    enum Kind { kFew, kTile, k192x192, k192x256, k256x256 } kind;
    int tile, splits;   // kFew: column blocks in `tile`
    int big;            // kTile: 256-row tiles that the 256 x 256 kernel takes before it
};

namespace quant_fit {
constexpr int kBigRows = 256;   // of the largest tile, rows and columns
constexpr float kStart = 3.13f, kBigEpilogue = 6.94f, kBigStep = 1.39f, kStep192 = 1.16f, kStepSquare192 = 0.83f;
constexpr float kMemory = 6.0e6f, kFabric = 66.4e6f;   // bytes per us
// few rows: a launch, a round of workgroups, what a CU receives (bytes per us), weights (four column blocks: they
// have half the wavefronts) and the activations that all workgroups read
constexpr float kFewStart = 1.99f, kFewRound = 0.218f, kFewCu = 40.1e3f, kFewWeights = 5.16e6f, kFewWeights4 = 4.95e6f,
                kFewShared = 12.7e6f;
// a CU's only tile, and each of several (two or three of the smallest at a time)
constexpr float kTileAlone[kQuantTiles] = {0.20f, 0.263f, 0.339f, 0.34f, 0.868f};
constexpr float kTileStep[kQuantTiles] = {0.171f, 0.244f, 0.341f, 0.617f, 1.08f};
constexpr float kTileEpilogue[kQuantTiles] = {0.677f, 1.09f, 1.99f, 3.39f, 6.75f};
// a second launch, and its sums written and read
constexpr float kFinish = 4.24f, kFinishShare = 0.457f, kFinishBytes = 4.71e6f;
}  // namespace quant_fit

// n_mt < 0: every row of M; else the entries of a row-tile list.  wg: CUs of an XCD.
inline QuantChoice quant_choose(int M, int N, int K, int n_mt, int wg) {
    using namespace quant_fit;
    const bool list = n_mt >= 0;
    const int nk = quant_div(K, kQuantStep), tiles_n = quant_div(N, kBigRows);
    if (!list) n_mt = quant_div(M, kBigRows);
    const int rows = list ? static_cast<int>(std::min<int64_t>(M, int64_t(n_mt) * kBigRows)) : M;
    const float bytes = (float(rows) + N) * K + 4.f * rows * N;
    QuantChoice best{QuantChoice::kTile, 0, 1, 0};
    float best_time = 1e30f;
    auto consider = [&](float time, const QuantChoice& c) {
        if (time < best_time) {
            best_time = time;
            best = c;
        }
    };
    if (rows <= kQuantFewRows) {
        const int row_blocks = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
        for (int blocks : {1, 2, 4}) {
            if (blocks == 4 && row_blocks > 1) continue;   // (the registers)
            const int wgs = quant_div(N, 16 * blocks), rounds = quant_div(wgs, 8 * wg);
            if (int64_t(wgs) * 64 * quant_few_waves(blocks) > UINT32_MAX) continue;   // (more than a launch holds)
            const float cu = rounds * (kFewRound + 16.f * (blocks + row_blocks) * K / kFewCu);
            const float mem = bytes / (blocks == 4 ? kFewWeights4 : kFewWeights) + float(wgs) * rows * K / kFewShared;
            consider(kFewStart + std::max(cu, mem), QuantChoice{QuantChoice::kFew, blocks, 1, 0});
        }
    }
    auto tile_time = [&](int t, int m, int splits) {
        const int64_t tiles = int64_t(quant_div(m, kQuantTileRows[t])) * quant_div(N, kQuantTileCols[t]);
        const int64_t per_cu = ((tiles * splits + 7) / 8 + wg - 1) / wg;
        const float fetched = float(tiles) * (kQuantTileRows[t] + kQuantTileCols[t]) * K;
        const float work = per_cu * kTileEpilogue[t] + quant_div(nk, splits) * (per_cu == 1 ? kTileAlone[t] : per_cu * kTileStep[t]);
        const float mem = ((float(m) + N) * K + 4.f * m * N) / kMemory + fetched / kFabric;
        return kStart + std::max(work, mem) + (splits > 1 ? kFinish + splits * (kFinishShare + 4.f * m * N / kFinishBytes) : 0.f);
    };
    for (int t = 0; t < kQuantTiles; ++t) {
        consider(tile_time(t, rows, 1), QuantChoice{QuantChoice::kTile, t, 1, 0});
        if (list) continue;
        const int64_t tiles = int64_t(quant_div(M, kQuantTileRows[t])) * quant_div(N, kQuantTileCols[t]);
        for (int s : {2, 3, 4, 6, 8})   // shares of K, up to three workgroups per CU
            if (s <= nk && tiles * s <= 24 * wg) consider(tile_time(t, M, s), QuantChoice{QuantChoice::kTile, t, s, 0});
    }
    if (rows <= kQuantFewRows || K < kQuantStep) return best;   // (the large tiles need a whole step)
    auto big_time = [&](int mt, int tile_rows, float step, int tile_cols = kBigRows) {
        const int64_t per_cu = quant_div(quant_xcd_split(mt, quant_div(N, tile_cols), wg).tiles, wg);
        const float mem = (float(mt) * tile_rows * K + float(N) * K + 4.f * mt * tile_rows * N) / kMemory;
        return kStart + std::max(per_cu * (nk * step + kBigEpilogue), mem);
    };
    if (n_mt == quant_div(M, kBigRows)) {   // (a list must name every tile: it counts in 256 rows)
        consider(big_time(quant_div(M, 192), 192, kStep192), QuantChoice{QuantChoice::k192x256, 0, 1, 0});
        consider(big_time(quant_div(M, 192), 192, kStepSquare192, 192), QuantChoice{QuantChoice::k192x192, 0, 1, 0});
    }
    consider(big_time(n_mt, kBigRows, kBigStep), QuantChoice{QuantChoice::k256x256, 0, 1, 0});
    // whole rounds of 256 x 256 tiles and the other rows on small ones; a split has to promise 5%
    const int64_t rounds = int64_t(n_mt) * tiles_n / (8 * wg);
    for (int64_t r = rounds; r > 0 && r >= rounds - 1; --r) {
        const int big = static_cast<int>(r * 8 * wg / tiles_n), rest = rows - big * kBigRows;
        if (big <= 0 || rest <= 0) continue;
        for (int t = 0; t < kQuantTiles; ++t)
            consider((big_time(big, kBigRows, kBigStep) + tile_time(t, rest, 1)) * 1.05f, QuantChoice{QuantChoice::kTile, t, 1, big});
    }
    return best;
}

}  // namespace ppk
