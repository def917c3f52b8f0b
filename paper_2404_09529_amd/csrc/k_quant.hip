// Rows in 8-bit codes with a scale for each row: quantize_rows, and rmsnorm_quant (residual
// addition, RMSNorm and the codes of its result).
//
// scale = max|y| * (1 / 127), code = round(y / scale).  Both need the whole row before the first code
// is written, so a row stays in registers between its one read and its one write: memory bounds
// both kernels (27,721 x 4096, back to back: quantize_rows of bf16 59 us, 5.8 TB/s; rmsnorm_quant with a bf16 residual
// 218, 5.7 TB/s; dequantize_rows to bf16 62, 5.5 TB/s, to float32 144, 3.9 TB/s; quantize_rows behind a kernel that wrote 227 MB
// 74 us, 4.6 TB/s).
//
// A row of up to four 16-byte chunks per lane is one wavefront's, a longer one a workgroup's: 20,000 rows
// of 688 bf16 values 9.3 us and 19.4, of 4096 46.2 and 43.5.  Six chunks a thread beside eight, for the
// registers: rmsnorm_quant of 300 x 5120 5.6 -> 5.2 us, 3951 x 5120 21.4 -> 21.1, 27,721 x 5120 127 -> 125 (with a bf16
// residual 279 -> 282).
// quantize_rows has workgroups of 16 wavefronts too, for the rows of a wide layer's second weight (up to
// 65,536 float32 or 131,072 bf16 values): 4096 x 28,672 float32 106 us, 5.5 TB/s, instead of 156 with two reads.
#include "device.h"
#include "kernels.h"
#include "prepack.h"

namespace {

constexpr int kThreads = 256;
constexpr int kRsrcWord3 = 0x00020000;   // raw buffer descriptors, word 3 (gfx9 family)

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------------------- codes
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

__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o, kWave)));
    return v;
}

// Threads of a workgroup whose rows have W wavefronts each: kThreads, or those of one row.
template <int W>
constexpr int kBlock = kWave * W > kThreads ? kWave * W : kThreads;

// Over the W wavefronts of a row (W = 1: each wavefront of the workgroup has a row of its own); T: float
// or double.
template <int W, typename T>
__device__ __forceinline__ T row_sum(T v, T* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    if constexpr (W > 1) {
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v += lds[w];
    }
    return v;
}
template <int W>
__device__ __forceinline__ uint32_t row_umax(uint32_t v, uint32_t* lds) {
    v = wave_umax(v);
    if constexpr (W > 1) {
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = max(v, lds[w]);
    }
    return v;
}

// ------------------------------------------------------------------------------- row access
// A row's bytes behind a buffer descriptor of its length: lanes past its end read zeros, which
// change neither the sum nor the maximum, and their stores go nowhere.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_rsrc(const void* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, kRsrcWord3);
}

template <typename T>
struct Add4;   // four consecutive values of a row as float, at element offset e
template <>
struct Add4<float> {
    u32x4 raw;
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int e) {
        raw = __builtin_amdgcn_raw_buffer_load_b128(r, e * 4, 0, 0);
    }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(raw[i]); }
};
template <>
struct Add4<bf16> {
    u32x2 raw;
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int e) {
        raw = __builtin_amdgcn_raw_buffer_load_b64(r, e * 2, 0, 0);
    }
    __device__ __forceinline__ float at(int i) const {
        return __uint_as_float(i & 1 ? raw[i >> 1] & 0xffff0000u : raw[i >> 1] << 16);
    }
};

__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ f32x4 load4(const bf16* p) {
    const bf16x4 v = *reinterpret_cast<const bf16x4*>(p);
    return f32x4{static_cast<float>(v[0]), static_cast<float>(v[1]), static_cast<float>(v[2]), static_cast<float>(v[3])};
}

// Row of this thread's W wavefronts, uniform in each of them.
template <int W>
__device__ __forceinline__ int64_t my_row() {
    constexpr int per_block = kBlock<W> / kWave / W;
    return (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * per_block + __builtin_amdgcn_readfirstlane(threadIdx.x / (kWave * W));
}

// ------------------------------------------------------------------------------- norm
// NC chunks of four elements per lane: rows of up to NC * 256 * W elements.
template <typename T, bool ADD, int W, int NC>
__global__ __launch_bounds__(kThreads) void rmsnorm_quant_kernel(float* __restrict__ x, const T* __restrict__ add,
                                                                 const float* __restrict__ g, int rows, int d,
                                                                 float eps, int8_t* __restrict__ q,
                                                                 float* __restrict__ scale) {
    __shared__ float sums[kThreads / kWave];
    __shared__ uint32_t tops[kThreads / kWave];
    const int64_t row = my_row<W>();
    if (row >= rows) return;   // whole wavefronts, and with W > 1 a workgroup has one row
    const int t = threadIdx.x % (kWave * W);
    const __amdgpu_buffer_rsrc_t rx = row_rsrc(x + row * d, d * 4), rg = row_rsrc(g, d * 4), rq = row_rsrc(q + row * d, d);
    auto at = [&](int c) { return (c * kWave * W + t) * 4; };
    u32x4 xr[NC];
    Add4<T> ar[ADD ? NC : 1];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        xr[c] = __builtin_amdgcn_raw_buffer_load_b128(rx, at(c) * 4, 0, 0);
    }
    if constexpr (ADD) {
        const __amdgpu_buffer_rsrc_t ra = row_rsrc(add + row * d, d * static_cast<int>(sizeof(T)));
#pragma unroll
        for (int c = 0; c < NC; ++c) ar[c].load(ra, at(c));
    }
    u32x4 gr[NC];   // requested with the rest, so that they are there when the sum is
#pragma unroll
    for (int c = 0; c < NC; ++c) gr[c] = __builtin_amdgcn_raw_buffer_load_b128(rg, at(c) * 4, 0, 0);
    float v[NC][4], ss = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[c][i] = __uint_as_float(xr[c][i]);
            if constexpr (ADD) v[c][i] += ar[c].at(i);
            ss += v[c][i] * v[c][i];
        }
        if constexpr (ADD) {
            const u32x4 o = {__float_as_uint(v[c][0]), __float_as_uint(v[c][1]), __float_as_uint(v[c][2]), __float_as_uint(v[c][3])};
            __builtin_amdgcn_raw_buffer_store_b128(o, rx, at(c) * 4, 0, 0);
        }
    }
    ss = row_sum<W>(ss, sums);
    const float r = rsqrtf(ss / static_cast<float>(d) + eps);
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[c][i] = v[c][i] * r * __uint_as_float(gr[c][i]);
            top = max(top, magnitude(v[c][i]));
        }
    }
    top = row_umax<W>(top, tops);
    const RowCode rc = row_code(top);
#pragma unroll
    for (int c = 0; c < NC; ++c) __builtin_amdgcn_raw_buffer_store_b32(codes4(v[c], rc), rq, at(c), 0, 0);
    if (t == 0) scale[row] = rc.scale;
}

// Rows too long for the registers: one workgroup each, a thread's four values at a time, read three times
// (a thread reads again what it wrote itself; 4096 rows of 28,672 values, bf16 residual: 335 us,
// 3.9 TB/s).  Four squares are added in float32 and their sums in float64: a thread has up to 2^23
// squares, and with float32 sums the scale of 4,000,016 equal values was off by 8e-5 of itself (as fast).
template <typename T>
__global__ __launch_bounds__(kThreads) void rmsnorm_quant_long_kernel(float* __restrict__ x, const T* __restrict__ add,
                                                                      const float* __restrict__ g, int rows, int d,
                                                                      float eps, int8_t* __restrict__ q,
                                                                      float* __restrict__ scale) {
    __shared__ double sums[kThreads / kWave];
    __shared__ uint32_t tops[kThreads / kWave];
    const int64_t row = my_row<kThreads / kWave>();
    if (row >= rows) return;
    float* xr = x + row * d;
    const T* ar = add ? add + row * d : nullptr;
    double ss = 0.0;
#pragma unroll 4
    for (int64_t e = 4 * threadIdx.x; e < d; e += 4 * kThreads) {
        f32x4 v = load4(xr + e);
        if (ar) {
            v += load4(ar + e);
            *reinterpret_cast<f32x4*>(xr + e) = v;
        }
        ss += (v[0] * v[0] + v[1] * v[1]) + (v[2] * v[2] + v[3] * v[3]);
    }
    ss = row_sum<kThreads / kWave>(ss, sums);
    const float r = rsqrtf(static_cast<float>(ss / d) + eps);
    uint32_t top = 0;
#pragma unroll 4
    for (int64_t e = 4 * threadIdx.x; e < d; e += 4 * kThreads) {
        const f32x4 v = load4(xr + e) * r * load4(g + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, magnitude(v[i]));
    }
    top = row_umax<kThreads / kWave>(top, tops);
    const RowCode rc = row_code(top);
#pragma unroll 4
    for (int64_t e = 4 * threadIdx.x; e < d; e += 4 * kThreads) {
        const f32x4 y = load4(xr + e) * r * load4(g + e);
        const float v[4] = {y[0], y[1], y[2], y[3]};
        *reinterpret_cast<uint32_t*>(q + row * d + e) = codes4(v, rc);
    }
    if (threadIdx.x == 0) scale[row] = rc.scale;
}

// ------------------------------------------------------------------------------- rows as they are
template <typename T, int W, int NC>
__global__ __launch_bounds__(kBlock<W>) void quantize_kernel(const T* __restrict__ x, int64_t ldx, int rows, int d,
                                                            int8_t* __restrict__ q, int64_t ldq,
                                                            float* __restrict__ scale) {
    __shared__ uint32_t tops[kBlock<W> / kWave];
    const int64_t row = my_row<W>();
    if (row >= rows) return;
    const int t = threadIdx.x % (kWave * W);
    constexpr int E = 16 / sizeof(T);   // elements of a lane's 16-byte chunk
    const __amdgpu_buffer_rsrc_t rx = row_rsrc(x + row * ldx, d * static_cast<int>(sizeof(T))), rq = row_rsrc(q + row * ldq, d);
    u32x4 raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) raw[c] = __builtin_amdgcn_raw_buffer_load_b128(rx, (c * kWave * W + t) * 16, 0, 0);
    uint32_t top = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = max(top, raw[c][i] & 0x7fffffffu);
    } else {
        uint32_t lo = 0, hi = 0;   // magnitudes of the even and the odd elements, in the upper half of a word
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo = max(lo, raw[c][i] << 17);
                hi = max(hi, raw[c][i] & 0x7fff0000u);
            }
        top = max(lo >> 1, hi);
    }
    top = row_umax<W>(top, tops);
    const RowCode rc = row_code(top);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float v[E];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(raw[c][i]);
            __builtin_amdgcn_raw_buffer_store_b32(codes4(v, rc), rq, (c * kWave * W + t) * E, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(raw[c][i] << 16);
                v[2 * i + 1] = __uint_as_float(raw[c][i] & 0xffff0000u);
            }
            const u32x2 o = {codes4(v, rc), codes4(v + 4, rc)};
            __builtin_amdgcn_raw_buffer_store_b64(o, rq, (c * kWave * W + t) * E, 0, 0);
        }
    }
    if (t == 0) scale[row] = rc.scale;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_long_kernel(const T* __restrict__ x, int64_t ldx, int rows, int d,
                                                                 int8_t* __restrict__ q, int64_t ldq,
                                                                 float* __restrict__ scale) {
    __shared__ uint32_t tops[kThreads / kWave];
    const int64_t row = my_row<kThreads / kWave>();
    if (row >= rows) return;
    const T* xr = x + row * ldx;
    uint32_t top = 0;
#pragma unroll 4
    for (int64_t e = 4 * threadIdx.x; e < d; e += 4 * kThreads) {
        const f32x4 v = load4(xr + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, magnitude(v[i]));
    }
    top = row_umax<kThreads / kWave>(top, tops);
    const RowCode rc = row_code(top);
#pragma unroll 4
    for (int64_t e = 4 * threadIdx.x; e < d; e += 4 * kThreads) {
        const f32x4 y = load4(xr + e);
        const float v[4] = {y[0], y[1], y[2], y[3]};
        *reinterpret_cast<uint32_t*>(q + row * ldq + e) = codes4(v, rc);
    }
    if (threadIdx.x == 0) scale[row] = rc.scale;
}

// ------------------------------------------------------------------------------- back to values
// 16 codes per thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(const int8_t* __restrict__ q, int64_t ldq,
                                                              const float* __restrict__ scale, int64_t n, uint32_t per_row,
                                                              T* __restrict__ x, int64_t ldx) {
    const int64_t t = (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * kThreads + threadIdx.x;
    if (t >= n) return;
    int64_t row;
    uint32_t c;
    if (n <= UINT32_MAX) {   // (a 32-bit division where it will do)
        row = static_cast<uint32_t>(t) / per_row;
        c = static_cast<uint32_t>(t) % per_row;
    } else {
        row = t / per_row;
        c = static_cast<uint32_t>(t % per_row);
    }
    const u32x4 codes = *reinterpret_cast<const u32x4*>(q + row * ldq + int64_t(c) * 16);
    const float s = scale[row];
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = static_cast<float>(static_cast<int8_t>(codes[i / 4] >> (8 * (i % 4)))) * s;
    T* o = x + row * ldx + int64_t(c) * 16;
    store8(o, v);
    store8(o + 8, v + 8);
}

// ------------------------------------------------------------------------------- dispatch
constexpr int kW = kThreads / kWave;   // wavefronts of a row that a whole workgroup takes

// Workgroups for the rows, in two dimensions: one may hold 2^32 threads at most.
template <int W>
dim3 row_blocks(int rows) {
    constexpr int per = kBlock<W> / kWave / W;
    const int64_t n = (int64_t(rows) + per - 1) / per, x = n < (1 << 20) ? n : 1 << 20;
    return dim3(static_cast<unsigned>(x), static_cast<unsigned>((n + x - 1) / x));
}

template <typename T, bool ADD, int W, int NC>
void launch_norm(float* x, const T* add, const float* g, int rows, int d, float eps, int8_t* q, float* scale, hipStream_t s) {
    rmsnorm_quant_kernel<T, ADD, W, NC><<<row_blocks<W>(rows), kThreads, 0, s>>>(x, add, g, rows, d, eps, q, scale);
}

template <typename T, bool ADD>
void norm_dispatch(float* x, const T* add, const float* g, int rows, int d, float eps, int8_t* q, float* scale, hipStream_t s) {
    const int of_wave = (d - 1) / (kWave * 4) + 1;    // chunks of a lane of one wavefront
    if (of_wave <= 1) return launch_norm<T, ADD, 1, 1>(x, add, g, rows, d, eps, q, scale, s);
    if (of_wave <= 2) return launch_norm<T, ADD, 1, 2>(x, add, g, rows, d, eps, q, scale, s);
    if (of_wave <= 4) return launch_norm<T, ADD, 1, 4>(x, add, g, rows, d, eps, q, scale, s);
    const int nc = (d - 1) / (kThreads * 4) + 1;   // and of a whole workgroup
    if (nc <= 2) return launch_norm<T, ADD, kW, 2>(x, add, g, rows, d, eps, q, scale, s);
    if (nc <= 4) return launch_norm<T, ADD, kW, 4>(x, add, g, rows, d, eps, q, scale, s);
    if (nc <= 6) return launch_norm<T, ADD, kW, 6>(x, add, g, rows, d, eps, q, scale, s);
    if (nc <= 8) return launch_norm<T, ADD, kW, 8>(x, add, g, rows, d, eps, q, scale, s);
    if (nc <= 16) return launch_norm<T, ADD, kW, 16>(x, add, g, rows, d, eps, q, scale, s);
    rmsnorm_quant_long_kernel<T><<<row_blocks<kW>(rows), kThreads, 0, s>>>(x, add, g, rows, d, eps, q, scale);
}

template <typename T, int W, int NC>
void launch_rows(const T* x, int64_t ldx, int rows, int d, int8_t* q, int64_t ldq, float* scale, hipStream_t s) {
    quantize_kernel<T, W, NC><<<row_blocks<W>(rows), kBlock<W>, 0, s>>>(x, ldx, rows, d, q, ldq, scale);
}

template <typename T>
void rows_dispatch(const T* x, int64_t ldx, int rows, int d, int8_t* q, int64_t ldq, float* scale, hipStream_t s) {
    constexpr int E = 16 / sizeof(T);
    const int of_wave = (d - 1) / (kWave * E) + 1;
    if (of_wave <= 1) return launch_rows<T, 1, 1>(x, ldx, rows, d, q, ldq, scale, s);
    if (of_wave <= 2) return launch_rows<T, 1, 2>(x, ldx, rows, d, q, ldq, scale, s);
    if (of_wave <= 4) return launch_rows<T, 1, 4>(x, ldx, rows, d, q, ldq, scale, s);
    const int nc = (d - 1) / (kThreads * E) + 1;
    if (nc <= 2) return launch_rows<T, kW, 2>(x, ldx, rows, d, q, ldq, scale, s);
    if (nc <= 4) return launch_rows<T, kW, 4>(x, ldx, rows, d, q, ldq, scale, s);
    if (nc <= 6) return launch_rows<T, kW, 6>(x, ldx, rows, d, q, ldq, scale, s);
    if (nc <= 8) return launch_rows<T, kW, 8>(x, ldx, rows, d, q, ldq, scale, s);
    if (nc <= 16) return launch_rows<T, kW, 16>(x, ldx, rows, d, q, ldq, scale, s);
    const int nc16 = (d - 1) / (16 * kWave * E) + 1;          // and of one of 16 wavefronts
    if (nc16 <= 8) return launch_rows<T, 16, 8>(x, ldx, rows, d, q, ldq, scale, s);
    if (nc16 <= 16) return launch_rows<T, 16, 16>(x, ldx, rows, d, q, ldq, scale, s);
    quantize_long_kernel<T><<<row_blocks<kW>(rows), kThreads, 0, s>>>(x, ldx, rows, d, q, ldq, scale);
}

template <typename T>
void dequantize(const int8_t* q, int64_t ldq, const float* scale, int rows, int d, T* x, int64_t ldx, hipStream_t s) {
    const int64_t n = int64_t(rows) * (d / 16), blocks = (n + kThreads - 1) / kThreads;
    const int64_t bx = blocks < (1 << 20) ? blocks : 1 << 20;
    dequantize_kernel<T><<<dim3(static_cast<unsigned>(bx), static_cast<unsigned>((blocks + bx - 1) / bx)), kThreads, 0, s>>>(
        q, ldq, scale, n, static_cast<uint32_t>(d / 16), x, ldx);
}

}  // namespace

namespace ppk {

void dequantize_rows(int dtype, const int8_t* q, int64_t ldq, const float* scale, int rows, int d, void* x, int64_t ldx,
                     hipStream_t s) {
    if (dtype == PP_BF16)
        dequantize(q, ldq, scale, rows, d, static_cast<bf16*>(x), ldx, s);
    else
        dequantize(q, ldq, scale, rows, d, static_cast<float*>(x), ldx, s);
}

void quantize_rows(int dtype, const void* x, int64_t ldx, int rows, int d, int8_t* q, int64_t ldq, float* scale,
                   hipStream_t s) {
    if (dtype == PP_BF16)
        rows_dispatch(static_cast<const bf16*>(x), ldx, rows, d, q, ldq, scale, s);
    else
        rows_dispatch(static_cast<const float*>(x), ldx, rows, d, q, ldq, scale, s);
}

void rmsnorm_quant(int dtype, float* x, const void* add, const float* g, int rows, int d, float eps, int8_t* q,
                   float* scale, hipStream_t s) {
    if (!add)
        norm_dispatch<float, false>(x, nullptr, g, rows, d, eps, q, scale, s);
    else if (dtype == PP_BF16)
        norm_dispatch<bf16, true>(x, static_cast<const bf16*>(add), g, rows, d, eps, q, scale, s);
    else
        norm_dispatch<float, true>(x, static_cast<const float*>(add), g, rows, d, eps, q, scale, s);
}

}  // namespace ppk
