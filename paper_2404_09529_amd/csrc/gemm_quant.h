// What the 8-bit GEMM's kernels share: operand types, their place in LDS and the element-wise
// arithmetic of the epilogues, so that a result does not depend on which kernel computed it (the
// int32 sums are exact in any order).
#pragma once
#include <atomic>

#include "device.h"
#include "gemm_quant_choice.h"
#include "kernels.h"

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kQuantListRows = 256;   // rows of one entry of a plan's row-tile list
// Buffer descriptor word 3 for raw (unstructured) 32-bit-offset loads on gfx9-family parts.
constexpr int kQuantRsrcWord3 = 0x00020000;

// s_waitcnt immediate: vmcnt(n) and lgkmcnt(0), expcnt not waited for (gfx9 encoding).
constexpr int quant_wait(int n) { return ((n >> 4) << 14) | (n & 15) | 0x0070; }

typedef __attribute__((address_space(3))) void lds_void;

// LDS swizzle of 128-byte rows: 16-byte chunk c of row r at chunk c ^ swz(r).  A fragment read
// takes chunk 4 ks + l / 16 of rows l % 16, lanes i and i + 32 served together: 8 rows x chunks
// {c, c ^ 2} on distinct banks (the derivation stands in k_gemm_bf16.hip: the rows are as long).
__device__ __forceinline__ int quant_swz(int r) { return ((r >> 1) & 1) | (((r >> 3) & 1) << 1) | (r & 4); }

__device__ __forceinline__ void quant_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t quant_rsrc(const int8_t* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p), 0, bytes, kQuantRsrcWord3);
}

__device__ __forceinline__ i32x4 quant_mfma(i32x4 w, i32x4 a, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, a, c, 0, 0, 0);
}

// A sum with its scales.  One order of roundings everywhere, no fused multiply-add.
__device__ __forceinline__ float quant_scaled(int32_t acc, float as, float bs) {
#pragma clang fp contract(off)
    return static_cast<float>(acc) * as * bs;
}
// SiLU(gate) * up: for a bf16 result with the hardware's exponential and reciprocal, whose errors are
// far below its rounding; for float32 with the library's.
template <typename TO>
__device__ __forceinline__ float quant_swiglu(float gate, float up) {
#pragma clang fp contract(off)
    if constexpr (sizeof(TO) == 2) return gate * __builtin_amdgcn_rcpf(1.0f + __expf(-gate)) * up;
    else return gate / (1.0f + expf(-gate)) * up;
}
__device__ __forceinline__ float quant_add(float c, float v) {
#pragma clang fp contract(off)
    return c + v;
}

// Four scales, which start at any float.
__device__ __forceinline__ f32x4 quant_scales4(const float* p) {
    typedef f32x4 unaligned __attribute__((aligned(4)));
    return *reinterpret_cast<const unaligned*>(p);
}

// Four consecutive results to memory (8- or 16-byte store; rows start on 8-byte boundaries at least).
__device__ __forceinline__ void quant_store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void quant_store4(bf16* p, f32x4 v) {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = static_cast<bf16>(v[e]);
    *reinterpret_cast<bf16x4*>(p) = o;
}

// The epilogue of 4 consecutive columns n .. n + 3 of row m straight from the registers.  kSwiGLU: acc
// the gate's sums and up those of the column block 16 further.
template <int EPI, typename TO>
__device__ __forceinline__ void quant_finish4(const ppk::QuantGemm& g, int m, int n, float as, i32x4 acc, i32x4 up) {
    const f32x4 bs = quant_scales4(g.b_scale + n);
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = quant_scaled(acc[e], as, bs[e]);
    if constexpr (EPI == ppk::kResidual) {
        float* c = static_cast<float*>(g.C) + int64_t(m) * g.ldc + n;
        const f32x4 o = *reinterpret_cast<const f32x4*>(c);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = quant_add(o[e], v[e]);
        quant_store4(c, v);
    } else if constexpr (EPI == ppk::kSwiGLU) {
        const f32x4 bu = quant_scales4(g.b_scale + n + 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = quant_swiglu<TO>(v[e], quant_scaled(up[e], as, bu[e]));
        // columns 32 j + c (gate) become 16 j + c
        quant_store4(static_cast<TO*>(g.C) + int64_t(m) * g.ldc + (n >> 5) * 16 + (n & 15), v);
    } else {
        quant_store4(static_cast<TO*>(g.C) + int64_t(m) * g.ldc + n, v);
    }
}

namespace ppk {

int cu_count();   // CUs of the GPU, rounded down to a multiple of 8

// Lets a kernel have `bytes` of dynamic LDS on the current GPU; `done` holds a bit for each GPU on which it may.
inline void quant_allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    (void)hipGetDevice(&dev);
    const uint64_t bit = uint64_t(1) << (dev & 63);
    if (done.load(std::memory_order_relaxed) & bit) return;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess) done.fetch_or(bit);
}

// Up to 64 rows: weights straight from memory to the registers, 16 * blocks columns (blocks 1, 2, or
// up to 16 rows 4) and all of K per workgroup.
void quant_gemm_few(int epi, bool out_f32, int blocks, const QuantGemm& g, hipStream_t s);

// Tiles of kQuantTileRows x kQuantTileCols: entries mt_first .. mt_first + n_mt - 1 of the row-tile list
// (without one: of the 256-row tiles of M).  splits > 1 (without a list, every row): K in that many
// shares, whose sums go to g.part [splits][M][N], and a second launch for the epilogue.
void quant_gemm_tiles(int epi, bool out_f32, int tile, const QuantGemm& g, int mt_first, int n_mt, int splits,
                      hipStream_t s);

}  // namespace ppk
