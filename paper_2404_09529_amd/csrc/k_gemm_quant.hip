// Projection GEMM of 8-bit codes: C = (A B^T) with a scale for each row of A and of B, int32 sums.
//
// One wavefront per 16 rows x 16 (SwiGLU: 32) columns, operands straight from memory: the simplest form
// that is right for every size.  It reads both operands once per block, so it is bound by L2.
#include "device.h"
#include "kernels.h"

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
constexpr int kListRows = 256;   // rows of one entry of a plan's row-tile list

template <typename TO>
__device__ __forceinline__ void store4(TO* p, const float* v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = static_cast<TO>(v[e]);
}

template <int EPI, typename TO>
__global__ __launch_bounds__(64) void gemm_quant_kernel(ppk::QuantGemm g, int64_t tiles_m, int64_t tiles) {
    constexpr int NB = EPI == ppk::kSwiGLU ? 2 : 1;
    const int lane = threadIdx.x, lr = lane & 15, lg = lane >> 4;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int mt = static_cast<int>(tile % tiles_m), nt = static_cast<int>(tile / tiles_m);
        const int m0 = g.mtile_m0 ? g.mtile_m0[mt / (kListRows / 16)] + mt % (kListRows / 16) * 16 : mt * 16;
        if (m0 >= g.M) continue;
        const int n0 = nt * 16 * NB, m = m0 + lr;
        const int8_t* a = g.A + int64_t(min(m, g.M - 1)) * g.lda + 16 * lg;
        const int8_t* b = g.B + int64_t(n0 + lr) * g.ldb + 16 * lg;
        i32x4 acc[NB] = {};
        for (int k = 0; k < g.K; k += 64) {
            const bool in = k + 16 * lg < g.K;
            const i32x4 av = in ? *reinterpret_cast<const i32x4*>(a + k) : i32x4{};
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const i32x4 bv = in ? *reinterpret_cast<const i32x4*>(b + 16 * i * g.ldb + k) : i32x4{};
                acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bv, av, acc[i], 0, 0, 0);
            }
        }
        if (m >= g.M) continue;
        const float as = g.a_scale[m];
        float v[NB][4];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[i][e] = static_cast<float>(acc[i][e]) * as * g.b_scale[n0 + 16 * i + 4 * lg + e];
        if constexpr (EPI == ppk::kResidual) {
            float* c = static_cast<float*>(g.C) + int64_t(m) * g.ldc + n0 + 4 * lg;
            f32x4 o = *reinterpret_cast<const f32x4*>(c);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += v[0][e];
            *reinterpret_cast<f32x4*>(c) = o;
        } else if constexpr (EPI == ppk::kSwiGLU) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[0][e] = v[0][e] / (1.0f + expf(-v[0][e])) * v[1][e];
            store4(static_cast<TO*>(g.C) + int64_t(m) * g.ldc + n0 / 2 + 4 * lg, v[0]);
        } else {
            store4(static_cast<TO*>(g.C) + int64_t(m) * g.ldc + n0 + 4 * lg, v[0]);
        }
    }
}

template <int EPI, typename TO>
void launch(const ppk::QuantGemm& g, hipStream_t s) {
    const int64_t tiles_m = g.mtile_m0 ? int64_t(g.n_mtiles) * (kListRows / 16) : (int64_t(g.M) + 15) / 16;
    const int64_t tiles = tiles_m * (g.N / (EPI == ppk::kSwiGLU ? 32 : 16));
    gemm_quant_kernel<EPI, TO><<<static_cast<unsigned>(tiles < 16384 ? tiles : 16384), 64, 0, s>>>(g, tiles_m, tiles);
}

}  // namespace

namespace ppk {

size_t quant_gemm_workspace(int, int, int) { return 0; }

void quant_gemm(int epi, bool out_f32, const QuantGemm& g, hipStream_t s) {
    if (epi == kResidual) return launch<kResidual, float>(g, s);
    if (epi == kSwiGLU) return out_f32 ? launch<kSwiGLU, float>(g, s) : launch<kSwiGLU, bf16>(g, s);
    return out_f32 ? launch<kStore, float>(g, s) : launch<kStore, bf16>(g, s);
}

}  // namespace ppk
