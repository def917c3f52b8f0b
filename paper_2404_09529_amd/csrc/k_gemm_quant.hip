// Projection GEMM of 8-bit codes: C[M, N] = A[M, K] B[N, K]^T with a scale for each row of A (token)
// and of B (output channel), exact int32 sums on the matrix cores, and the epilogues of a decoder
// layer.  This file: the 256 x 256, 192 x 256 and 192 x 192 tiles of large batches, and the calls of
// the kernels that gemm_quant_choice.h picks.
//
// The arrangement is k_gemm_bf16.hip's, whose 64-value steps of K are 128 bytes as the 128-value
// steps here are: one 256-thread workgroup (4 wavefronts, one per SIMD) per tile, a quarter of it to
// each wavefront (of the largest tile 128 x 128 values, 8 x 8 blocks of the 16x16x64 int8 MFMA: twice the
// products of the bf16 one in the same time), accumulators in the accumulation registers; operand
// tiles go from memory straight into an LDS ring of 5 slots of 32 KB (A and B of a step are one slot
// each), two in flight while a step is read; the workgroup's tiles are one stream of steps, whose loads cross
// tile boundaries; persistent, one workgroup per CU, every XCD on a compact block of tiles.
//
// What bounds it: 27,721 rows, N 22016, K 4096 with SwiGLU take 1.85 to 1.89 ms, 2.65 to 2.70 POP/s (a large int8 product of
// the vendor's library 2.43); the matrix cores are 67% busy at 1.93 GHz.  The MFMAs alone reach 3.9 POP/s on
// random codes and 4.75 on zeros: power holds the clock.  A step takes 1.54 us, 1.17 without the
// loads of operands (zeros: 1.21 and 1.12); with every operand in L2 the call would be 4% faster.  One
// wavefront a SIMD has to issue everything between its MFMAs, so nothing else may stand in the loop: moving
// the last step's offsets for a ragged K (instead of the step as a whole) cost 10%.  Weights through registers
// instead of direct loads: 4% slower.
//
// K need only be a multiple of 16 and 128 at least: the last step is the last 128 values, and the
// activations' fragments are zeroed where the step before had them already (what the weights hold then
// does not matter: the values are integers).  N a multiple of 16: rows of B past N are read as its last one.
#include <algorithm>

#include "gemm_quant.h"
#include "prepack.h"

namespace {

constexpr int BM = 256, BN = 256, NT = 256;   // of the largest tile
constexpr int ROW_B = kQuantStep, SLOT_B = BM * ROW_B, NSLOT = 5, LDS_BYTES = NSLOT * SLOT_B;

// The epilogue of one wavefront's 16 MB rows x 16 NB columns, 16 rows at a time (float32 rows in halves,
// which bounds the registers): lanes put their runs of four results into the staging area
// (LDS, this wavefront's own) and take back 16-byte chunks of whole rows, so that memory is read and
// written in whole lines.  Block (i, j): row mb + 16 j + l % 16, columns nb0 + 16 i + 4 (l / 16) + 0..3.
// Staging row r's chunk c sits at c ^ (r % chunks); a row of 6 blocks is staged in the room of 8.
template <int EPI, typename TO, int MB, int NB>
__device__ __forceinline__ void epilogue(i32x4 (&acc)[NB][MB], const ppk::QuantGemm& q, int mb, int nb0, int lane, char* stg) {
    constexpr bool PAIRS = EPI == ppk::kSwiGLU;
    constexpr int HALVES = !PAIRS && sizeof(TO) == 4 ? 2 : 1, IB = NB / HALVES;   // passes over a block row, blocks of each
    constexpr int COLS = PAIRS ? 8 * NB : 16 * NB / HALVES;                 // columns of a pass
    constexpr int RB = (PAIRS ? 64 : 128 / HALVES) * static_cast<int>(sizeof(TO)), CH = RB / 16;   // bytes, chunks of a staged row
    constexpr int RPI = 64 / CH, NI = 16 / RPI;                             // rows per instruction, instructions
    constexpr int PER = 16 / static_cast<int>(sizeof(TO));                  // values of a chunk
    const int lr = lane & 15, g = lane >> 4;
    const int n_out = PAIRS ? q.N / 2 : q.N;
    const int col0 = (PAIRS ? nb0 / 2 : nb0) + lane % CH * PER;
    const bool in_row = lane % CH * PER < COLS;   // (chunks past a row of 6 blocks hold nothing)
    f32x4 bs[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) bs[i] = quant_scales4(q.b_scale + min(nb0 + 16 * i, q.N - 16) + 4 * g);
    float as[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) as[j] = q.a_scale[min(mb + 16 * j + lr, q.M - 1)];
    u32x4 cbuf[2][NI];
    auto load_rows = [&](int t, u32x4 (&b)[NI]) {   // kResidual: addresses past M or N are the last ones again
#pragma unroll
        for (int k = 0; k < NI; ++k) {
            const int m = mb + 16 * (t / HALVES) + RPI * k + lane / CH;
            const int64_t at = int64_t(min(m, q.M - 1)) * q.ldc + min(col0 + COLS * (t % HALVES), n_out - PER);
            b[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const TO*>(q.C) + at));
        }
    };
    if constexpr (EPI == ppk::kResidual) load_rows(0, cbuf[0]);
#pragma unroll
    for (int t = 0; t < HALVES * MB; ++t) {
        const int j = t / HALVES, i0 = t % HALVES * IB;
        if constexpr (EPI == ppk::kResidual) {
            if (t + 1 < HALVES * MB) load_rows(t + 1, cbuf[(t + 1) & 1]);
        }
        i32x4 a[IB];
#pragma unroll
        for (int i = 0; i < IB; ++i) {   // out of the accumulation registers one block row at a time
            asm volatile("" : "+a"(acc[i0 + i][j]) : : "memory");
            a[i] = acc[i0 + i][j];
        }
#pragma unroll
        for (int i = 0; i < IB; i += PAIRS ? 2 : 1) {
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = quant_scaled(a[i][e], as[j], bs[i0 + i][e]);
                if constexpr (PAIRS) v[e] = quant_swiglu<TO>(v[e], quant_scaled(a[i + 1][e], as[j], bs[i + 1][e]));
            }
            const int at = (PAIRS ? 8 * i : 16 * i) + 4 * g, ch = at / PER;   // column and chunk of the run
            quant_store4(reinterpret_cast<TO*>(stg + lr * RB + (ch ^ (lr % CH)) * 16) + at % PER, v);
        }
        u32x4 o[NI];
#pragma unroll
        for (int k = 0; k < NI; ++k) {
            const int r = RPI * k + lane / CH;
            o[k] = *reinterpret_cast<const u32x4*>(stg + r * RB + ((lane % CH) ^ (r % CH)) * 16);
        }
#pragma unroll
        for (int k = 0; k < NI; ++k) {
            const int m = mb + 16 * j + RPI * k + lane / CH, col = col0 + COLS * (t % HALVES);
            if (m < q.M && col < n_out && in_row) {
                u32x4* p = reinterpret_cast<u32x4*>(static_cast<TO*>(q.C) + int64_t(m) * q.ldc + col);
                if constexpr (EPI == ppk::kResidual) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[k][e] = __float_as_uint(quant_add(__uint_as_float(cbuf[t & 1][k][e]), __uint_as_float(o[k][e])));
                    __builtin_nontemporal_store(o[k], p);
                } else {
                    *p = o[k];
                }
            }
        }
    }
    // The loads of C and the stores are waited for once, here: otherwise the compiler protects their
    // registers with waits inside the next K loop, where they would stand behind its loads.  The staging area
    // is refilled by this wavefront's own loads right after.
    __builtin_amdgcn_s_waitcnt(quant_wait(0));
}

// MB, NB: 16-row and 16-column blocks of a wavefront, so tiles of 32 MB x 32 NB (6: 192, rows without a
// row-tile list).
template <int EPI, typename TO, int MB, int NB>
__global__ __launch_bounds__(NT, 1) void gemm_quant_kernel(ppk::QuantGemm q, int tiles_m, int tiles_n, int balanced) {
    constexpr int TM = 32 * MB, TN = 32 * NB, GM = 64 / MB;   // of a tile; M-tiles of a group
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // ---- schedule.  XCD x (workgroup id mod 8) takes the contiguous M-tiles [x pm, x pm + pm) in groups of
    // at most GM sweeping N, or (balanced) an eighth of the same list over all M-tiles where the
    // first leaves an XCD a round of tiles more.
    const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, n_slots = gridDim.x >> 3;
    int m_begin, m_cnt, g_begin, n_local;
    if (balanced) {
        const int total = tiles_m * tiles_n, per = (total + 7) / 8;
        m_begin = 0;
        m_cnt = tiles_m;
        g_begin = xcd * per;
        n_local = min(per, total - g_begin);
    } else {
        const int pm = (tiles_m + 7) / 8;
        m_begin = xcd * pm;
        m_cnt = min(pm, tiles_m - m_begin);
        g_begin = 0;
        n_local = m_cnt * tiles_n;
    }
    if (m_cnt <= 0 || slot >= n_local) return;
    const int n_groups = (m_cnt + GM - 1) / GM, gm = (m_cnt + n_groups - 1) / n_groups;
    auto tile_m0n0 = [&](int local, int& m0, int& n0) {
        const int gi = g_begin + local;
        const int group = gi / (gm * tiles_n), within = gi - group * gm * tiles_n;
        const int first = group * gm, gsz = min(m_cnt - first, gm);
        const int mt = m_begin + first + within % gsz;
        m0 = q.mtile_m0 ? q.mtile_m0[mt] : mt * TM;
        n0 = within / gsz * TN;
    };
    const int nk = (q.K + kQuantStep - 1) / kQuantStep;
    // Every XCD starts at another eighth of K and goes round, so that not all wait for the same channels of
    // the memory.  Weights from memory, us together and so: 2926 rows, N 6144, K 4096 81, 73; 2000 rows, N 4096,
    // K 11008 93, 88; 6000 rows, N 6144, K 5120 166, 160; where the products bound it no difference.
    const int k_rot = xcd * nk / 8;
    const int tail = q.K % kQuantStep;   // values of the last step, 0: a whole one

    // ---- direct memory -> LDS loads: each fills 1 KB = 8 rows x 128 bytes of a slot, lane l landing at
    // physical chunk l % 8 of row l / 8 and fetching the logical chunk that the swizzle puts there.
    // Rows past M or N are read as the last one: every load is in range, so loads complete in
    // the order in which they were issued.
    const int lda = static_cast<int>(q.lda), ldb = static_cast<int>(q.ldb);
    const int lrow = lane >> 3;
    int chunk_off[2];   // of even and odd loads
#pragma unroll
    for (int t = 0; t < 2; ++t) chunk_off[t] = 16 * ((lane & 7) ^ quant_swz(8 * t + lrow));
    int voff_a[MB], voff_b[NB];
    // load cursor: the step being requested, into slots l_sa (A) and l_sb (B); l_local >= n_local once the
    // stream is exhausted (its loads are then dead: they read nothing, into slots that are not read again)
    int l_local = slot, l_kt = k_rot, l_sa = 0, l_sb = 1, l_k = min(k_rot * kQuantStep, q.K - kQuantStep);   // l_kt: step of K, l_k: its first value
    __amdgpu_buffer_rsrc_t rsrc_a, rsrc_b;
    const __amdgpu_buffer_rsrc_t rsrc_0 = quant_rsrc(q.A, 0);
    auto set_cursor_tile = [&]() {
        if (l_local < n_local) {
            int m0, n0;
            tile_m0n0(l_local, m0, n0);
            const int a_rows = min(q.M - m0, TM), b_rows = min(q.N - n0, TN);
            rsrc_a = quant_rsrc(q.A + int64_t(m0) * lda, (a_rows - 1) * lda + q.K);
            rsrc_b = quant_rsrc(q.B + int64_t(n0) * ldb, (b_rows - 1) * ldb + q.K);
#pragma unroll
            for (int t = 0; t < MB; ++t) voff_a[t] = min(8 * (MB * wave + t) + lrow, a_rows - 1) * lda + chunk_off[t & 1];
#pragma unroll
            for (int t = 0; t < NB; ++t) voff_b[t] = min(8 * (NB * wave + t) + lrow, b_rows - 1) * ldb + chunk_off[t & 1];
        } else {
            rsrc_a = rsrc_0;
            rsrc_b = rsrc_0;
        }
    };
    set_cursor_tile();
    auto load_a = [&](int t) {
        char* dst = smem + l_sa * SLOT_B + (wave * MB + t) * 1024;
        const int voff = voff_a[t];
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_a, (lds_void*)dst, 16, voff, l_k, 0, 0);
    };
    auto load_b = [&](int t) {
        char* dst = smem + l_sb * SLOT_B + (wave * NB + t) * 1024;
        const int voff = voff_b[t];
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_b, (lds_void*)dst, 16, voff, l_k, 0, 0);
    };
    // in two parts: scalar arithmetic that issues between MFMAs, and the rare step to another tile
    bool l_wrap = false;
    auto advance_cursor = [&]() {
        l_sa = l_sa >= NSLOT - 2 ? l_sa + 2 - NSLOT : l_sa + 2;
        l_sb = l_sb >= NSLOT - 2 ? l_sb + 2 - NSLOT : l_sb + 2;
        l_kt = l_kt == nk - 1 ? 0 : l_kt + 1;
        l_wrap = l_kt == k_rot;
        l_k = min(l_kt * kQuantStep, q.K - kQuantStep);
    };
    auto advance_tile = [&]() {
        if (l_wrap && l_local < n_local) {
            l_local += n_slots;
            set_cursor_tile();
        }
    };

    // ---- fragments.  Block i of sub-step ks: row base + 16 i + l % 16, logical chunk 4 ks + l / 16
    const int wn = wave & 1, wm = wave >> 1;
    int a_lds[2], b_lds[2];
    bool again[2];   // this lane's 16 values of the last step's sub-step belong to the step before
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        const int phys = ((4 * ks + (lane >> 4)) ^ quant_swz(lane & 15)) * 16;
        a_lds[ks] = (wm * 16 * MB + (lane & 15)) * ROW_B + phys;
        b_lds[ks] = (wn * 16 * NB + (lane & 15)) * ROW_B + phys;
        again[ks] = tail && 64 * ks + 16 * (lane >> 4) < kQuantStep - tail;
    }
    struct Frags { i32x4 w[NB], a[MB]; };
    auto read_one = [&](int sa, int sb, int ks, int p, Frags& f) {   // w0, a0 .., w1 ..: as the MFMAs need them
        if (p == 0) f.w[0] = *reinterpret_cast<const i32x4*>(smem + sb * SLOT_B + b_lds[ks]);
        else if (p <= MB) f.a[p - 1] = *reinterpret_cast<const i32x4*>(smem + sa * SLOT_B + a_lds[ks] + (p - 1) * 16 * ROW_B);
        else f.w[p - MB] = *reinterpret_cast<const i32x4*>(smem + sb * SLOT_B + b_lds[ks] + (p - MB) * 16 * ROW_B);
    };
    auto zero_again = [&](int ks, Frags& f) {
#pragma unroll
        for (int j = 0; j < MB; ++j) f.a[j] = again[ks] ? i32x4{} : f.a[j];
    };

    // ---- the stream of steps.  Step g holds slots 2g % 5 (A) and (2g+1) % 5 (B).  Per step:
    //   sub-step 0: MFMAs (g, 0); read (g, 1); A tile of step g+2 (into the slot of B of g-1)
    //   wait until step g+1 has landed and this wavefront's reads of step g are done; barrier
    //   sub-step 1: MFMAs (g, 1); read (g+1, 0); B tile of step g+2 (into the slot of A of g)
    // The loads issued after B of g+1 are the MB of the A tile of g+2: vmcnt(MB) waits for g+1.
    int c_local = l_local;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
#pragma unroll
        for (int t = 0; t < MB; ++t) load_a(t);
#pragma unroll
        for (int t = 0; t < NB; ++t) load_b(t);
        advance_cursor();
        advance_tile();
    }
    __builtin_amdgcn_s_waitcnt(0);
    quant_barrier();
    Frags F0, F1;
    int c_sa = 0, c_sb = 1;
#pragma unroll
    for (int p = 0; p < NB + MB; ++p) read_one(c_sa, c_sb, 0, p, F0);
    while (true) {
        i32x4 acc[NB][MB];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] = i32x4{};
        // One sub-step: the MFMAs on `cur`, with the fragment reads of the next one (into `nxt`) and a
        // load per row of blocks, in a fixed order.  The first sub-step ends at the barrier: its
        // reads go among the first three quarters of the MFMAs, so they have landed by then.
        auto substep = [&](const Frags& cur, Frags& nxt, int rsa, int rsb, int rks, bool first) {
#pragma unroll
            for (int m = 0; m < NB * MB; ++m) {
                const int i = m / MB, j = m % MB;
                acc[i][j] = quant_mfma(cur.w[i], cur.a[j], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
                const int span = first ? NB * MB * 3 / 4 : NB * MB;
#pragma unroll
                for (int p = (m * (NB + MB) + span - 1) / span;
                     p < ((m + 1) * (NB + MB) + span - 1) / span && p < NB + MB; ++p)
                    read_one(rsa, rsb, rks, p, nxt);
                if (first) {
                    if (m % NB == 2) load_a(m / NB);
                } else {
                    if (m % MB == 2) load_b(m / MB);
                    if (m == (NB - 1) * MB + 3) advance_cursor();   // the cursor moves to step g+3
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        for (int kt = 0; kt < nk; ++kt) {
            const int n_sa = c_sa >= NSLOT - 2 ? c_sa + 2 - NSLOT : c_sa + 2;
            const int n_sb = c_sb >= NSLOT - 2 ? c_sb + 2 - NSLOT : c_sb + 2;
            const bool cut = tail && kt == nk - 1 - k_rot;
            if (cut) zero_again(0, F0);
            substep(F0, F1, c_sa, c_sb, 1, true);    // A tile of g+2
            if (l_local >= n_local) __builtin_amdgcn_s_waitcnt(quant_wait(0));   // dead loads may end out of turn
            __builtin_amdgcn_s_waitcnt(quant_wait(MB));
            quant_barrier();
            if (cut) zero_again(1, F1);
            substep(F1, F0, n_sa, n_sb, 0, false);   // B tile of g+2
            advance_tile();
            c_sa = n_sa;
            c_sb = n_sb;
        }
        // The slot of the last step's B tile is free until the A tile of step g+3 (its next user) is
        // requested in the next step's first sub-step; wavefront w's staging area is exactly the part of it
        // that w's own loads refill.
        int m0, n0;
        tile_m0n0(c_local, m0, n0);
        const int free_slot = c_sb >= 2 ? c_sb - 2 : c_sb + NSLOT - 2;
        epilogue<EPI, TO, MB, NB>(acc, q, m0 + wm * 16 * MB, n0 + wn * 16 * NB, lane, smem + free_slot * SLOT_B + wave * MB * 1024);
        c_local += n_slots;
        if (c_local >= n_local) break;
    }
    __builtin_amdgcn_s_waitcnt(0);   // no load may still be writing LDS when the workgroup ends
}

}  // namespace

namespace ppk {
namespace {

// The first n_mt tiles of 32 MB rows on this kernel.
template <int EPI, typename TO, int MB, int NB>
void launch(const QuantGemm& g, int n_mt, hipStream_t s) {
    static std::atomic<uint64_t> done{0};
    quant_allow_lds(reinterpret_cast<const void*>(&gemm_quant_kernel<EPI, TO, MB, NB>), LDS_BYTES, done);
    const int tiles_n = quant_div(g.N, 32 * NB), wg_per_xcd = cu_count() / 8;
    const QuantXcdSplit x = quant_xcd_split(n_mt, tiles_n, wg_per_xcd);
    QuantGemm q = g;
    if (MB == 8 && !g.mtile_m0) q.M = std::min<int64_t>(g.M, int64_t(n_mt) * BM);
    gemm_quant_kernel<EPI, TO, MB, NB><<<8 * static_cast<int>(std::min<int64_t>(wg_per_xcd, x.tiles)), NT, LDS_BYTES, s>>>(q, n_mt, tiles_n, x.balanced);
}

template <int EPI, typename TO>
void gemm(QuantGemm g, hipStream_t s) {
    if (g.M <= BM) g.mtile_m0 = nullptr;   // (a list of one tile then, which is all of M)
    const int n_mt = g.mtile_m0 ? g.n_mtiles : quant_div(g.M, BM);
    const QuantChoice c = quant_choose(g.M, g.N, g.K, g.mtile_m0 ? n_mt : -1, cu_count() / 8);
    if (c.kind == QuantChoice::kFew) return quant_gemm_few(EPI, sizeof(TO) == 4, c.tile, g, s);
    if (c.kind == QuantChoice::k256x256) return launch<EPI, TO, 8, 8>(g, n_mt, s);
    if (c.kind == QuantChoice::k192x256 || c.kind == QuantChoice::k192x192) {
        g.mtile_m0 = nullptr;   // (it names every tile)
        return c.kind == QuantChoice::k192x256 ? launch<EPI, TO, 6, 8>(g, quant_div(g.M, 192), s)
                                          : launch<EPI, TO, 6, 6>(g, quant_div(g.M, 192), s);
    }
    if (c.big > 0) launch<EPI, TO, 8, 8>(g, c.big, s);
    quant_gemm_tiles(EPI, sizeof(TO) == 4, c.tile, g, c.big, n_mt - c.big, c.splits, s);
}

}  // namespace

size_t quant_gemm_workspace(int M, int N, int K) {
    if (M == 0) return 0;
    const QuantChoice c = quant_choose(M, N, K, -1, cu_count() / 8);   // (a row-tile list is never split)
    return c.kind == QuantChoice::kTile && c.splits > 1 ? size_t(c.splits) * M * N * sizeof(int32_t) : 0;
}

void quant_gemm(int epi, bool out_f32, const QuantGemm& g, hipStream_t s) {
    if (epi == kResidual) return gemm<kResidual, float>(g, s);
    if (epi == kSwiGLU) return out_f32 ? gemm<kSwiGLU, float>(g, s) : gemm<kSwiGLU, bf16>(g, s);
    return out_f32 ? gemm<kStore, float>(g, s) : gemm<kStore, bf16>(g, s);
}

}  // namespace ppk
