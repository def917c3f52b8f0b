// The 8-bit GEMM on smaller output tiles than 256 x 256, for batches whose large tiles are too few, or
// too badly divided, for the CUs.
//
// One workgroup per tile, persistent, its tiles one stream of 128-value steps of K through an LDS ring of
// NS slots (A rows, then B rows of a step) filled NS - 1 steps ahead with direct-to-LDS loads of whole
// 128-byte row segments.  Per step one barrier, after which a wavefront refills the slot whose fragments
// it has, requests the next step's fragments, and runs the step's MFMAs meanwhile.  Ragged K and N as
// in k_gemm_quant.hip, but that any K will do.
//
// What bounds it is what a CU receives.  A direct-to-LDS load of 1 KB holds its wavefront's next one back
// for 140 cycles (17 GB/s a wavefront), so a CU wants 8 wavefronts at work: one workgroup of 8 where
// the ring takes the LDS, or several of 4 (64 rows, N 4096, K 8192 on 128 x 128 tiles: 43 us with 4
// wavefronts, 37 with 8).  In the 32 x 64, 64 x 64 and 128 x 128 tiles two wavefronts share a
// sub-tile, each with half of every step's K, so that they read a third less from LDS (35 us; 64 x 64
// tiles 19.8 to 17.8); on 64 x 128 and 128 x 256 tiles that gave nothing or lost.  Lines that another CU
// of the XCD wants too come at up to 98 GB/s, the others at 70.  Deeper rings are no faster.
// Measured (us; 256 x 256 tiles, the tile chosen): 344 rows, N 2048, K 5504: 70, 14.4 (64 x 64); 1309 rows:
// 72, 27.4 (128 x 128); 100 rows, N 4096, K 4096: 51, 10.3 (32 x 64); 64 rows, N 4096, K 14336: 158, 22.3
// (64 x 64 in shares of K); 48 rows, N 28672, K 4096: 53, 25.2, 4.7 TB/s (64 x 128).
#include <algorithm>

#include "gemm_quant.h"

namespace {

constexpr int ROW_B = kQuantStep;

// WM x WN x WK wavefronts: wavefront (wm, wn, wk) holds MB x NB blocks of 16 x 16 and, where WK is 2,
// takes the half wk of every step's K (XB: blocks that each hands over at a time when the halves are
// added at the end of a tile).
template <int BM_, int BN_, int WM_, int WN_, int WK_, int NS_, int XB_>
struct Geom {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WK = WK_, NS = NS_, XB = XB_;
    static constexpr int NW = WM * WN * WK, NT = 64 * NW, KS = 2 / WK;   // KS: MFMAs deep in a step, per wavefront
    static constexpr int MB = BM / 16 / WM, NB = BN / 16 / WN;
    static constexpr int A_LD = BM * ROW_B / 1024 / NW, B_LD = BN * ROW_B / 1024 / NW;   // 1 KB loads per wavefront
    static constexpr int STEP_LD = A_LD + B_LD;
    static constexpr int SLOT_B = (BM + BN) * ROW_B;
    static constexpr int LDS = NS * SLOT_B + (WK == 2 ? NW * XB * 1024 : 0);
    static_assert(NB >= 2 && NB % 2 == 0, "gate and up blocks of a pair in one wavefront");
    static_assert(WK == 1 || (MB % 2 == 0 && MB / 2 * NB % XB == 0), "each of the two keeps half of the rows");
    static_assert(A_LD * NW * 1024 == BM * ROW_B && B_LD * NW * 1024 == BN * ROW_B, "whole loads");
    static_assert(NS >= 3 && LDS <= 160 * 1024 && (NS - 1) * STEP_LD <= 63, "ring");
};

// Entries mt_first .. mt_first + n_mt - 1 of the row-tile list (or of the 256-row tiles of M), each of
// kQuantListRows / BM row tiles; those of the batch's last entry that start past M are left out.  The (row
// tile, column tile) list goes column by column in groups of at most GM row tiles and is cut into 8
// contiguous ranges, one per XCD (workgroup id mod 8).
template <int EPI, typename TO, class G, int WGS>
__global__ __launch_bounds__(G::NT, WGS * G::NW / 4) void gemm_quant_tiles_kernel(ppk::QuantGemm q, int mt_first, int n_mt) {
    constexpr int BM = G::BM, BN = G::BN, NS = G::NS, MB = G::MB, NB = G::NB, KS = G::KS;
    constexpr int SUB = kQuantListRows / BM, GM = 2048 / BM;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    const int last0 = q.mtile_m0 ? q.mtile_m0[mt_first + n_mt - 1] : (mt_first + n_mt - 1) * kQuantListRows;
    const int tiles_m = (n_mt - 1) * SUB + min(SUB, (q.M - last0 + BM - 1) / BM);
    const int tiles_n = (q.N + BN - 1) / BN;
    const int xcd = blockIdx.x & 7, slot0 = blockIdx.x >> 3, n_slots = gridDim.x >> 3;
    const int total = tiles_m * tiles_n, per = (total + 7) / 8;
    const int g_begin = xcd * per, n_local = min(per, total - g_begin);
    const int n_groups = (tiles_m + GM - 1) / GM, gm = (tiles_m + n_groups - 1) / n_groups;
    if (slot0 >= n_local) return;
    auto tile_m0n0 = [&](int local, int& m0, int& n0) {
        const int gi = g_begin + local;
        const int group = gi / (gm * tiles_n), within = gi - group * gm * tiles_n;
        const int first = group * gm, gsz = min(tiles_m - first, gm);
        const int mt = first + within % gsz;
        const int entry = mt_first + mt / SUB;
        m0 = (q.mtile_m0 ? q.mtile_m0[entry] : entry * kQuantListRows) + mt % SUB * BM;
        n0 = within / gsz * BN;
    };
    // this workgroup's steps of K: all of them, or one of kPartial's gridDim.y shares
    const int all = (q.K + kQuantStep - 1) / kQuantStep;
    const int k_first = EPI == ppk::kPartial ? static_cast<int>(int64_t(all) * blockIdx.y / gridDim.y) : 0;
    const int nk = EPI == ppk::kPartial ? static_cast<int>(int64_t(all) * (blockIdx.y + 1) / gridDim.y) - k_first : all;
    const int tail = k_first + nk == all ? q.K % kQuantStep : 0;   // values of the last step, 0: a whole one

    // Where in K this workgroup starts (and goes round): every XCD at another eighth.  At rows of some
    // strides, multiples of 4096 bytes among them, workgroups at the same K wait for the same few channels of
    // the memory; those of an XCD stay together, for the lines that they share in its L2.  us, all together
    // and so: 48 rows, N 28672, K 4096 32.3, 26.3; 8192 50.7, 45.5; 11008 78.3, 68.4; 4224 27.3, 27.7; 1309
    // rows, N 2048, K 5504 35.0, 31.9 (from the 256 MB of last-level cache 29.2, 29.2).
    const int k_rot = xcd * nk / 8;

    // ---- direct memory -> LDS loads: 1 KB = 8 rows x 128 bytes each; every address in range
    const int lda = static_cast<int>(q.lda), ldb = static_cast<int>(q.ldb);
    const int lrow = lane >> 3;
    // chunk fetched by this lane in loads of even and odd groups of 8 rows.  The last step of K is its last
    // 128 values; of a K below that, lanes past it fetch the row's last 16 values again
    int chunk_off[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) chunk_off[t] = min(16 * ((lane & 7) ^ quant_swz(8 * t + lrow)), q.K - 16);
    int voff_a[G::A_LD], voff_b[G::B_LD];
    // the parity of a load's first row group: wavefront w's t-th load starts at row 8 (LD w + t)
    const int odd_a = G::A_LD * wave & 1, odd_b = G::B_LD * wave & 1;
    // load cursor: the step being requested, into slot l_slot; past the last one its loads go
    // through an empty descriptor (they read nothing and land in slots that are not read again)
    int l_local = slot0, l_k = k_rot, l_slot = 0, l_off;   // l_k: step of K, l_off: its first value
    auto set_cursor_step = [&]() { l_off = min((k_first + l_k) * ROW_B, max(q.K - ROW_B, 0)); };
    set_cursor_step();
    __amdgpu_buffer_rsrc_t rsrc_a, rsrc_b;
    const __amdgpu_buffer_rsrc_t rsrc_0 = quant_rsrc(q.A, 0);
    auto set_cursor_tile = [&]() {
        if (l_local < n_local) {
            int m0, n0;
            tile_m0n0(l_local, m0, n0);
            const int a_rows = min(q.M - m0, BM), b_rows = min(q.N - n0, BN);
            rsrc_a = quant_rsrc(q.A + int64_t(m0) * lda, (a_rows - 1) * lda + q.K);
            rsrc_b = quant_rsrc(q.B + int64_t(n0) * ldb, (b_rows - 1) * ldb + q.K);
#pragma unroll
            for (int t = 0; t < G::A_LD; ++t)
                voff_a[t] = min(8 * (G::A_LD * wave + t) + lrow, a_rows - 1) * lda + ((t + odd_a) & 1 ? chunk_off[1] : chunk_off[0]);
#pragma unroll
            for (int t = 0; t < G::B_LD; ++t)
                voff_b[t] = min(8 * (G::B_LD * wave + t) + lrow, b_rows - 1) * ldb + ((t + odd_b) & 1 ? chunk_off[1] : chunk_off[0]);
        } else {
            rsrc_a = rsrc_0;
            rsrc_b = rsrc_0;
        }
    };
    set_cursor_tile();
    auto load = [&](int t) {   // t of the step's STEP_LD loads: A first
        const bool is_a = t < G::A_LD;
        char* dst = smem + l_slot * G::SLOT_B + (is_a ? (G::A_LD * wave + t) * 1024
                                                      : BM * ROW_B + (G::B_LD * wave + t - G::A_LD) * 1024);
        const int voff = is_a ? voff_a[is_a ? t : 0] : voff_b[is_a ? 0 : t - G::A_LD];
        __builtin_amdgcn_raw_ptr_buffer_load_lds(is_a ? rsrc_a : rsrc_b, (lds_void*)dst, 16, voff, l_off, 0, 0);
    };
    auto advance_cursor = [&]() {
        l_slot = l_slot == NS - 1 ? 0 : l_slot + 1;
        if (l_local >= n_local) return;
        l_k = l_k == nk - 1 ? 0 : l_k + 1;
        set_cursor_step();
        if (l_k == k_rot) {
            l_local += n_slots;
            set_cursor_tile();
        }
    };

    const int wn = wave % G::WN, wm = wave / G::WN % G::WM, wk = wave / (G::WN * G::WM);
    int a_lds[KS], b_lds[KS];
    bool past[KS];   // this lane's 16 values of the last step's half belong to the step before, or lie past K
#pragma unroll
    for (int h = 0; h < KS; ++h) {
        const int ks = G::WK == 2 ? wk : h;
        const int phys = ((4 * ks + (lane >> 4)) ^ quant_swz(lane & 15)) * 16;
        a_lds[h] = (wm * 16 * MB + (lane & 15)) * ROW_B + phys;
        b_lds[h] = (BM + wn * 16 * NB + (lane & 15)) * ROW_B + phys;
        const int v = 64 * ks + 16 * (lane >> 4);
        past[h] = tail && (q.K < ROW_B ? v >= tail : v < ROW_B - tail);
    }
    struct Frags { i32x4 w[KS][NB], a[KS][MB]; };   // a whole step's
    auto read_all = [&](int slot, Frags& f) {
        const char* base = smem + slot * G::SLOT_B;
#pragma unroll
        for (int h = 0; h < KS; ++h) {
#pragma unroll
            for (int i = 0; i < NB; ++i) f.w[h][i] = *reinterpret_cast<const i32x4*>(base + b_lds[h] + i * 16 * ROW_B);
#pragma unroll
            for (int j = 0; j < MB; ++j) f.a[h][j] = *reinterpret_cast<const i32x4*>(base + a_lds[h] + j * 16 * ROW_B);
        }
    };
    i32x4 acc[NB][MB];
    // One step: `cur` is on its way from slot c_slot.  Once it is there and the next step has landed (at
    // most the NS - 2 steps requested after it are pending; everything, once the last steps' loads are
    // dead), and all wavefronts agree, the slot is refilled, the next step's fragments are requested, and
    // the MFMAs run over both.
    auto step = [&](Frags& cur, Frags& nxt, int& c_slot, bool cut) {
        if (l_local < n_local) __builtin_amdgcn_s_waitcnt(quant_wait((NS - 2) * G::STEP_LD));
        else __builtin_amdgcn_s_waitcnt(quant_wait(0));
        quant_barrier();
        c_slot = c_slot == NS - 1 ? 0 : c_slot + 1;
#pragma unroll
        for (int t = 0; t < G::STEP_LD; ++t) load(t);
        read_all(c_slot, nxt);
        advance_cursor();
        if (cut) {
#pragma unroll
            for (int h = 0; h < KS; ++h)
#pragma unroll
                for (int j = 0; j < MB; ++j) cur.a[h][j] = past[h] ? i32x4{} : cur.a[h][j];
        }
#pragma unroll
        for (int h = 0; h < KS; ++h)
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j) acc[i][j] = quant_mfma(cur.w[h][i], cur.a[h][j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };

    // ---- prologue: the first NS steps requested, the first one awaited
#pragma unroll
    for (int p = 0; p < NS; ++p) {
#pragma unroll
        for (int t = 0; t < G::STEP_LD; ++t) load(t);
        advance_cursor();
    }
    if (l_local < n_local) __builtin_amdgcn_s_waitcnt(quant_wait((NS - 1) * G::STEP_LD));
    else __builtin_amdgcn_s_waitcnt(quant_wait(0));
    quant_barrier();
    Frags F0, F1;
    int c_slot = 0, c_local = slot0;
    read_all(0, F0);

    while (true) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] = i32x4{};
        const int cut = tail ? nk - 1 - k_rot : -1;   // the step that K ends in
        int kt = 0;
        for (; kt + 2 <= nk; kt += 2) {
            step(F0, F1, c_slot, kt == cut);
            step(F1, F0, c_slot, kt + 1 == cut);
        }
        if (kt < nk) {
            step(F0, F1, c_slot, kt == cut);
            F0 = F1;
        }
        int m0, n0;
        tile_m0n0(c_local, m0, n0);
        // block (i, j): row m0 + .. + l % 16 and columns n .. n + 3 of 16-column block i
        const int n_base = n0 + wn * 16 * NB + 4 * (lane >> 4);
        auto finish_row = [&](int j, const i32x4 (&a)[NB]) {
            const int m = m0 + wm * 16 * MB + 16 * j + (lane & 15);
            float as = 0.f;
            if constexpr (EPI != ppk::kPartial) as = q.a_scale[min(m, q.M - 1)];
            if (m >= q.M) return;
#pragma unroll
            for (int i = 0; i < NB; i += EPI == ppk::kSwiGLU ? 2 : 1) {
                if (n_base + 16 * i >= q.N) continue;
                if constexpr (EPI == ppk::kPartial)
                    *reinterpret_cast<i32x4*>(q.part + (int64_t(blockIdx.y) * q.M + m) * q.N + n_base + 16 * i) = a[i];
                else quant_finish4<EPI, TO>(q, m, n_base + 16 * i, as, a[i], a[EPI == ppk::kSwiGLU ? i + 1 : i]);
            }
        };
        if constexpr (G::WK == 1) {
#pragma unroll
            for (int j = 0; j < MB; ++j) {
                i32x4 a[NB];
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    if constexpr (NB * MB >= 16) asm volatile("" : "+a"(acc[i][j]) : : "memory");
                    a[i] = acc[i][j];
                }
                finish_row(j, a);
            }
        } else {
            // the two halves of K: wavefront wk keeps the block rows 2 t + wk and hands over the others,
            // XB blocks at a time through LDS of their own (the ring is full of the next tile)
            i32x4* mine = reinterpret_cast<i32x4*>(smem + NS * G::SLOT_B + wave * G::XB * 1024) + lane;
            const i32x4* other = reinterpret_cast<const i32x4*>(smem + NS * G::SLOT_B + (wave ^ (G::NW / 2)) * G::XB * 1024) + lane;
            i32x4 sum[MB / 2][NB];
#pragma unroll
            for (int r = 0; r < MB / 2 * NB; r += G::XB) {
                if (r > 0) {
                    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): what was handed over has been read
                    quant_barrier();
                }
#pragma unroll
                for (int x = 0; x < G::XB; ++x) {
                    const int t = (r + x) / NB, i = (r + x) % NB;
                    mine[x * 64] = wk ? acc[i][2 * t] : acc[i][2 * t + 1];
                    sum[t][i] = wk ? acc[i][2 * t + 1] : acc[i][2 * t];
                }
                __builtin_amdgcn_s_waitcnt(0xc07f);
                quant_barrier();
#pragma unroll
                for (int x = 0; x < G::XB; ++x) sum[(r + x) / NB][(r + x) % NB] += other[x * 64];
            }
#pragma unroll
            for (int t = 0; t < MB / 2; ++t) finish_row(2 * t + wk, sum[t]);
        }
        // waited for once, here: otherwise the compiler waits for the epilogue's loads inside the next K
        // loop, in every step, where that empties the ring
        __builtin_amdgcn_s_waitcnt(quant_wait(0));
        c_local += n_slots;
        if (c_local >= n_local) break;
    }
    __builtin_amdgcn_s_waitcnt(0);   // no load may still be writing LDS when the workgroup ends
}

// kPartial's sums of `splits` shares of K and the epilogue: one run of four results (SwiGLU: and the four
// sums of the other block) per thread.
template <int EPI, typename TO>
__global__ __launch_bounds__(256) void quant_finish_kernel(ppk::QuantGemm q, int splits) {
    constexpr int PER = EPI == ppk::kSwiGLU ? 8 : 4;   // columns of the product per thread
    const int64_t t = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int per_row = q.N / PER;
    const int m = static_cast<int>(t / per_row), r = static_cast<int>(t % per_row);
    if (m >= q.M) return;
    const int n = EPI == ppk::kSwiGLU ? r / 4 * 32 + r % 4 * 4 : r * 4;
    i32x4 a{}, b{};
    const int32_t* p = q.part + int64_t(m) * q.N + n;
    for (int s = 0; s < splits; ++s, p += int64_t(q.M) * q.N) {
        a += *reinterpret_cast<const i32x4*>(p);
        if constexpr (EPI == ppk::kSwiGLU) b += *reinterpret_cast<const i32x4*>(p + 16);
    }
    quant_finish4<EPI, TO>(q, m, n, q.a_scale[m], a, b);
}

// WGS: workgroups per CU.
template <int EPI, typename TO, class G, int WGS>
void launch(const ppk::QuantGemm& g, int mt_first, int n_mt, int splits, hipStream_t s) {
    static_assert(WGS * G::LDS <= 160 * 1024, "LDS of a CU's workgroups");
    static std::atomic<uint64_t> done{0};
    ppk::quant_allow_lds(reinterpret_cast<const void*>(&gemm_quant_tiles_kernel<EPI, TO, G, WGS>), G::LDS, done);
    const int64_t tiles = int64_t(n_mt) * (kQuantListRows / G::BM) * ((g.N + G::BN - 1) / G::BN);   // at least the kernel's count
    const int64_t grid = 8 * std::min<int64_t>((tiles + 7) / 8, WGS * (ppk::cu_count() / 8));
    gemm_quant_tiles_kernel<EPI, TO, G, WGS><<<dim3(static_cast<unsigned>(grid), splits), G::NT, G::LDS, s>>>(g, mt_first, n_mt);
}

template <int EPI, typename TO>
void launch_tile(int tile, const ppk::QuantGemm& g, int mt_first, int n_mt, int splits, hipStream_t s) {
    switch (tile) {
        case 0: return launch<EPI, TO, Geom<32, 64, 1, 2, 2, 4, 1>, 3>(g, mt_first, n_mt, splits, s);
        case 1: return launch<EPI, TO, Geom<64, 64, 2, 2, 2, 4, 2>, 2>(g, mt_first, n_mt, splits, s);
        case 2: return launch<EPI, TO, Geom<64, 128, 2, 4, 1, 3, 0>, 2>(g, mt_first, n_mt, splits, s);
        case 3: return launch<EPI, TO, Geom<128, 128, 2, 2, 2, 4, 4>, 1>(g, mt_first, n_mt, splits, s);
        default: return launch<EPI, TO, Geom<128, 256, 2, 4, 1, 3, 0>, 1>(g, mt_first, n_mt, splits, s);
    }
}

// K in `splits` shares: their sums first, then the epilogue in a launch of its own.
template <int EPI, typename TO>
void run(int tile, const ppk::QuantGemm& g, int mt_first, int n_mt, int splits, hipStream_t s) {
    if (splits == 1) return launch_tile<EPI, TO>(tile, g, mt_first, n_mt, 1, s);
    launch_tile<ppk::kPartial, float>(tile, g, mt_first, n_mt, splits, s);
    const int64_t threads = int64_t(g.M) * (g.N / (EPI == ppk::kSwiGLU ? 8 : 4));
    quant_finish_kernel<EPI, TO><<<static_cast<unsigned>((threads + 255) / 256), 256, 0, s>>>(g, splits);
}

}  // namespace

namespace ppk {

void quant_gemm_tiles(int epi, bool out_f32, int tile, const QuantGemm& g, int mt_first, int n_mt, int splits, hipStream_t s) {
    if (epi == kResidual) return run<kResidual, float>(tile, g, mt_first, n_mt, splits, s);
    if (epi == kSwiGLU)
        return out_f32 ? run<kSwiGLU, float>(tile, g, mt_first, n_mt, splits, s)
                       : run<kSwiGLU, bf16>(tile, g, mt_first, n_mt, splits, s);
    return out_f32 ? run<kStore, float>(tile, g, mt_first, n_mt, splits, s)
                   : run<kStore, bf16>(tile, g, mt_first, n_mt, splits, s);
}

}  // namespace ppk
