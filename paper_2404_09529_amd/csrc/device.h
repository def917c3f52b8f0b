// Device-side helpers shared by the gfx950 kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

typedef __bf16 bf16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
    return v;
}

// 8 consecutive elements <-> float, for either storage type.
__device__ __forceinline__ void load8(const float* p, float* v) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p);
    const f32x4 b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[i + 4] = b[i]; }
}
__device__ __forceinline__ void load8(const bf16* p, float* v) {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(a[i]);
}
__device__ __forceinline__ void store8(float* p, const float* v) {
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = v[i]; b[i] = v[i + 4]; }
    *reinterpret_cast<f32x4*>(p) = a;
    *reinterpret_cast<f32x4*>(p + 4) = b;
}
__device__ __forceinline__ void store8(bf16* p, const float* v) {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = static_cast<bf16>(v[i]);
    *reinterpret_cast<bf16x8*>(p) = a;
}

__device__ __forceinline__ float silu(float x) { return x / (1.0f + __expf(-x)); }
// SiLU with the hardware reciprocal (1 ulp) in place of the correctly rounded division: for
// results that are rounded to bf16 (8 significant bits) the difference is invisible.
__device__ __forceinline__ float silu_rcp(float x) { return x * __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

// One rotate-half pair (x, y) at angle (c, s): the products are fused in a fixed order.
__device__ __forceinline__ float rope_lo(float x, float y, float c, float s) { return fmaf(x, c, -(y * s)); }
__device__ __forceinline__ float rope_hi(float x, float y, float c, float s) { return fmaf(x, s, y * c); }
// The upper half as pp_rope and the float32 QKV epilogue form it: a float32 prefill's caches are
// those of pp_gemm, pp_rope and pp_kv_scatter bit for bit.
__device__ __forceinline__ float rope_hi_step(float x, float y, float c, float s) { return fmaf(y, c, x * s); }

// cos and sin of position * theta^(-2i/D), evaluated in float64.
__device__ __forceinline__ float2 rope_entry(int64_t position, int i, int D, double theta) {
    const double inv_freq = pow(theta, -2.0 * i / static_cast<double>(D));
    const double a = static_cast<double>(position) * inv_freq;
    return make_float2(static_cast<float>(cos(a)), static_cast<float>(sin(a)));
}
