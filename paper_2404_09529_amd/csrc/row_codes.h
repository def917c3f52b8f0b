// The 8-bit form of a row: its scale and its codes, shared by the kernels that write them.
#pragma once
#include "device.h"

// What turns a row's values into codes.  The largest magnitude is kept as the bits of its absolute
// value: as unsigned integers they are ordered as the magnitudes are, infinities above every
// number and NaN above them, so no NaN is lost on the way.
struct RowCode {
    float scale, pre, s, inv;   // s = scale * pre, inv = 1 / s
    uint32_t mask;   // 0 where the codes are 0 whatever the values (zero rows, rows with NaN or inf)
};

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ RowCode row_code(uint32_t top) {
    const bool finite = top < 0x7f800000u;
    RowCode c;
    c.scale = finite ? __uint_as_float(top) * (1.0f / 127.0f) : __uint_as_float(0x7fc00000u);
    // the reciprocal of a scale below 2^-126 would overflow: a power of two brings both into range
    c.pre = c.scale < 0x1p-100f ? 0x1p64f : 1.0f;
    c.s = c.scale * c.pre;
    c.inv = 1.0f / c.s;
    c.mask = finite && c.scale > 0.f ? 0xffffffffu : 0u;
    return c;
}

// Codes of four values in the bytes of a word.  The quotient is the product with the reciprocal and
// one correction by its remainder, so that values next to a border fall on the division's side (equal to it at
// 1.9 billion pairs within two float32 steps of a border).  Adding 1.5 * 2^23 leaves the nearest integer (ties to even) in the
// low bits of the sum, as two's complement; the clamp matters only to scales that are themselves denormal.
__device__ __forceinline__ uint32_t codes4(const float* v, const RowCode& c) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y = v[i] * c.pre, t = y * c.inv, u = fmaf(fmaf(-t, c.s, y), c.inv, t);
        b[i] = __float_as_uint(__builtin_amdgcn_fmed3f(u, -127.0f, 127.0f) + 12582912.0f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u) & c.mask;
}
