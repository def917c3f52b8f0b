// The 8-bit GEMM for few rows (decode steps): the weights are nearly all that a call reads, so they go
// straight from memory to the registers, once.
//
// A workgroup takes 16 NB columns and every row; its NW wavefronts deal the 128-value steps of K among
// themselves (wavefront w takes steps w, w + NW, ..: at any time the workgroup reads one contiguous stretch
// of each of its rows), and their int32 sums, exact in any order, are added through LDS.  The activations
// (16 MB rows, read again by every workgroup) come from L2 the same way.  No workgroup waits for another:
// no workspace, no second launch.  More steps in flight per wavefront are no faster (10 rows, N 4096,
// K 11008: 10.7 us, with two steps 4% more, with 16 wavefronts 5%): the CU's requests are what is bounded.
// What counts is few rounds of workgroups (16 rows, N 6144, K 4096: 384 workgroups of 16 columns 10.3 us, 192
// of 32 8.1; one row, N 12288: 192 of 64 10.7 us, 4.7 TB/s, 384 of 32 13.1; one row, N 28672: 896 of 32
// 23.1, 5.1 TB/s).  Tiles overtake it with the activations that every workgroup reads: 16 rows, N 28672 29 us, on
// 64 x 128 tiles 25.
//
// The weight block is the MFMA's first operand: a lane ends with 4 consecutive columns of one row.
#include "gemm_quant.h"

namespace {

template <int EPI, typename TO, int NB, int MB, int NW>
__global__ __launch_bounds__(64 * NW) void gemm_few_kernel(ppk::QuantGemm q) {
    __shared__ i32x4 sums[NW > 1 ? NW : 1][NB * MB][64];
    const int lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16 * NB;
    const int lda = static_cast<int>(q.lda), ldb = static_cast<int>(q.ldb);
    const int nk = (q.K + kQuantStep - 1) / kQuantStep;
    const int b_rows = min(q.N - n0, 16 * NB);
    const int bytes_a = (q.M - 1) * lda + q.K, bytes_b = (b_rows - 1) * ldb + q.K;
    const int8_t* B = q.B + int64_t(n0) * ldb;
    int ra[MB], rb[NB];   // byte offsets of this lane's rows; rows past the last are read as the last
#pragma unroll
    for (int j = 0; j < MB; ++j) ra[j] = min(16 * j + lr, q.M - 1) * lda;
#pragma unroll
    for (int i = 0; i < NB; ++i) rb[i] = min(16 * i + lr, b_rows - 1) * ldb;

    // Where in K the workgroup starts (and goes round), so that not all wait for the same channels of the
    // memory: in one round of workgroups those of an XCD together, which then find the activations in its
    // L2, and the XCDs apart; in several all of them apart.  Weights from memory, us without and with: 10
    // rows, N 4096, K 11008 13.9, 12.4; one row, N 12288, K 4096 13.0, 12.4; N 28672, K 8192 56.4, 51.5.
    const int k_rot = static_cast<int>((gridDim.x <= 256 ? (blockIdx.x & 7) * 32 : blockIdx.x & 255) * nk >> 8);
    auto place = [&](int s) { return s + k_rot >= nk ? s + k_rot - nk : s + k_rot; };   // of the s-th step, in K
    struct Step { i32x4 b[2][NB], a[2][MB]; };
    auto load = [&](int s, Step& f) {   // steps past the last read nothing (an empty descriptor) and give zeros
        const __amdgpu_buffer_rsrc_t r_a = quant_rsrc(q.A, s < nk ? bytes_a : 0), r_b = quant_rsrc(B, s < nk ? bytes_b : 0);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            // lanes past K read the row's last 16 values again; the activations are then zeroed
            const int k = place(s) * kQuantStep + 64 * ks + 16 * g, kc = min(k, q.K - 16);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int at = rb[i] + kc;
                f.b[ks][i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r_b, at, 0, 0));
            }
#pragma unroll
            for (int j = 0; j < MB; ++j) {
                const int at = ra[j] + kc;
                f.a[ks][j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r_a, at, 0, 0));
            }
        }
    };
    i32x4 acc[NB][MB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j) acc[i][j] = i32x4{};
    auto add = [&](int s, Step& f) {
        s = place(s);
        if ((s + 1) * kQuantStep > q.K) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int j = 0; j < MB; ++j)
                    f.a[ks][j] = s * kQuantStep + 64 * ks + 16 * g >= q.K ? i32x4{} : f.a[ks][j];
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j) acc[i][j] = quant_mfma(f.b[ks][i], f.a[ks][j], acc[i][j]);
    };
    Step f;
    load(wave, f);
    for (int st = wave; st < nk; st += NW) {
        add(st, f);
        load(st + NW, f);
    }
    // ---- the wavefronts' sums, added by as many of them as there are blocks (gate and up together)
    constexpr int PER = EPI == ppk::kSwiGLU ? 2 : 1, BLOCKS = NB * MB / PER;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j) sums[wave][j * NB + i][lane] = acc[i][j];
    __syncthreads();
    for (int b = wave; b < BLOCKS; b += NW) {
        const int j = b / (NB / PER), i = b % (NB / PER) * PER;
        const int m = 16 * j + lr, n = n0 + 16 * i + 4 * g;
        i32x4 t[PER];
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            t[x] = sums[0][j * NB + i + x][lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) t[x] += sums[w][j * NB + i + x][lane];
        }
        if (m < q.M && n < q.N) quant_finish4<EPI, TO>(q, m, n, q.a_scale[m], t[0], t[PER - 1]);
    }
}

template <int EPI, typename TO, int NB, int MB>
void launch(const ppk::QuantGemm& g, hipStream_t s) {
    constexpr int NW = ppk::quant_few_waves(NB);
    gemm_few_kernel<EPI, TO, NB, MB, NW><<<(g.N + 16 * NB - 1) / (16 * NB), 64 * NW, 0, s>>>(g);
}

template <int EPI, typename TO, int MB>
void columns(int blocks, const ppk::QuantGemm& g, hipStream_t s) {
    if constexpr (EPI != ppk::kSwiGLU) {   // (its gate and up blocks go together)
        if (blocks == 1) return launch<EPI, TO, 1, MB>(g, s);
    }
    if constexpr (MB == 1) {
        if (blocks == 4) return launch<EPI, TO, 4, MB>(g, s);
    }
    launch<EPI, TO, 2, MB>(g, s);
}

template <int EPI, typename TO>
void rows(int blocks, const ppk::QuantGemm& g, hipStream_t s) {
    if (g.M <= 16) return columns<EPI, TO, 1>(blocks, g, s);
    if (g.M <= 32) return columns<EPI, TO, 2>(blocks, g, s);
    columns<EPI, TO, 4>(blocks, g, s);
}

}  // namespace

namespace ppk {

void quant_gemm_few(int epi, bool out_f32, int blocks, const QuantGemm& g, hipStream_t s) {
    if (epi == kResidual) return rows<kResidual, float>(blocks, g, s);
    if (epi == kSwiGLU) return out_f32 ? rows<kSwiGLU, float>(blocks, g, s) : rows<kSwiGLU, bf16>(blocks, g, s);
    return out_f32 ? rows<kStore, float>(blocks, g, s) : rows<kStore, bf16>(blocks, g, s);
}

}  // namespace ppk
