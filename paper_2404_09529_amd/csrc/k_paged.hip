// A paged cache's rows: written from dense rows (a prefill's caches), read back, and appended to by a
// decode step with the rotation of its query and key (RESTART-PE: a sequence's positions are its own).
//
// A head's row of D values is D / 8 lanes' (16 for D = 128), 8 values each, so that its scale is a maximum over
// lanes that sit side by side.  Memory bounds the rows' kernels; the append is a few microseconds of latency.
#include "device.h"
#include "kernels.h"
#include "paged.h"
#include "prepack.h"
#include "row_codes.h"

namespace {

constexpr int kBlock = 256;

// The code of a head's row of LANES * N values, N a lane; its lanes sit side by side and all take part.
template <int LANES, int N>
__device__ __forceinline__ RowCode head_code(const float (&v)[N]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, magnitude(v[i]));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
        top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o, kWave)));
    return row_code(top);
}

template <typename T>
__device__ __forceinline__ void load_row8(const T* pages, const float*, int64_t src, int64_t, float* v) {
    load8(pages + src, v);
}
__device__ __forceinline__ void load_row8(const int8_t* pages, const float* scales, int64_t src, int64_t head_row, float* v) {
    const uint2 q = *reinterpret_cast<const uint2*>(pages + src);
    const float s = scales[head_row];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = static_cast<float>(static_cast<int8_t>(q.x >> (8 * i))) * s;
        v[i + 4] = static_cast<float>(static_cast<int8_t>(q.y >> (8 * i))) * s;
    }
}

__device__ __forceinline__ int32_t place(const ppk::PagedCache& c, int32_t seq, int32_t pos) {
    if (seq < 0 || seq >= c.k || pos < 0 || (pos >> c.shift) >= c.max_pages) return -1;
    return ppk::paged_row(c.table[int64_t(seq) * c.max_pages + (pos >> c.shift)], c.n_pages, pos, c.shift);
}

// Item = (row, keys or values, 8 values); one thread each.
template <int D, typename T, typename P, bool WRITE>
__global__ __launch_bounds__(kBlock) void paged_rows_kernel(ppk::PagedCache c, const int32_t* __restrict__ seq,
                                                            const int32_t* __restrict__ pos, int64_t items, T* k,
                                                            int64_t ldk, T* v, int64_t ldv) {
    constexpr int LANES = D / 8;
    const int per = c.Hkv * LANES;   // threads of a row of keys
    const int64_t step = int64_t(gridDim.x) * kBlock;
    for (int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x; i < items; i += step) {
        const int64_t r2 = i / per;
        const int at = static_cast<int>(i - r2 * per), head = at / LANES;
        const int64_t r = r2 >> 1;
        const bool val = r2 & 1;
        const int32_t row = place(c, seq[r], pos[r]);
        if (row < 0) continue;   // the lanes of a head's row go together
        T* x = (val ? v + r * ldv : k + r * ldk) + at * 8;
        P* pages = static_cast<P*>(val ? c.vp : c.kp);
        float* scales = val ? c.vs : c.ks;
        const int64_t off = int64_t(row) * c.Hkv * D + at * 8, head_row = int64_t(row) * c.Hkv + head;
        float y[8];
        if constexpr (WRITE) {
            load8(x, y);
            if constexpr (sizeof(P) == 1) {
                const RowCode rc = head_code<LANES>(y);
                *reinterpret_cast<uint2*>(pages + off) = make_uint2(codes4(y, rc), codes4(y + 4, rc));
                if (at % LANES == 0) scales[head_row] = rc.scale;
            } else {
                store8(pages + off, y);
            }
        } else {
            load_row8(pages, scales, off, head_row, y);
            store8(x, y);
        }
    }
}

// One workgroup: sequence blockIdx.x, 256 / (D / 16) heads from blockIdx.y on.  A thread rotates 8 pairs
// (x_j, x_{j + D/2}) of a head; the heads after H + Hkv are values, which stay as they are.
template <int D, typename T, typename P>
__global__ __launch_bounds__(kBlock) void paged_append_kernel(ppk::PagedCache c, const int32_t* __restrict__ lens,
                                                              const T* qkv, int64_t ldqkv, T* q_out, int64_t ldq,
                                                              double theta) {
    constexpr int LANES = D / 16, HEADS = kBlock / LANES, HALF = D / 2;
    __shared__ float2 angle[HALF];
    const int i = blockIdx.x, pos = lens[i] - 1;
    if (pos < 0) return;
    const int head = blockIdx.y * HEADS + threadIdx.x / LANES, j = threadIdx.x % LANES * 8;
    const bool live = head < c.H + 2 * c.Hkv;
    float lo[8], hi[8];
    if (live) {
        const T* x = qkv + i * ldqkv + int64_t(head) * D + j;
        load8(x, lo);
        load8(x + HALF, hi);
    }
    if (threadIdx.x < HALF) angle[threadIdx.x] = rope_entry(pos, threadIdx.x, D, theta);
    __syncthreads();
    if (!live) return;
    if (head < c.H + c.Hkv) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double x = lo[e], y = hi[e], cs = angle[j + e].x, sn = angle[j + e].y;
            lo[e] = static_cast<float>(x * cs - y * sn);
            hi[e] = static_cast<float>(y * cs + x * sn);
        }
    }
    if (head < c.H) {
        T* q = q_out + i * ldq + int64_t(head) * D + j;
        store8(q, lo);
        store8(q + HALF, hi);
        return;
    }
    const int32_t row = place(c, i, pos);
    if (row < 0) return;
    const bool val = head >= c.H + c.Hkv;
    const int h = head - c.H - (val ? c.Hkv : 0);
    const int64_t head_row = int64_t(row) * c.Hkv + h;
    P* dst = static_cast<P*>(val ? c.vp : c.kp) + head_row * D + j;
    if constexpr (sizeof(P) == 1) {
        float both[16];
#pragma unroll
        for (int e = 0; e < 8; ++e) both[e] = lo[e], both[e + 8] = hi[e];
        const RowCode rc = head_code<LANES>(both);
        *reinterpret_cast<uint2*>(dst) = make_uint2(codes4(lo, rc), codes4(lo + 4, rc));
        *reinterpret_cast<uint2*>(dst + HALF) = make_uint2(codes4(hi, rc), codes4(hi + 4, rc));
        if (j == 0) (val ? c.vs : c.ks)[head_row] = rc.scale;
    } else {
        store8(dst, lo);
        store8(dst + HALF, hi);
    }
}

template <bool WRITE>
void rows(int dtype, const ppk::PagedCache& c, const int32_t* seq, const int32_t* pos, int n, void* k, int64_t ldk,
          void* v, int64_t ldv, hipStream_t s) {
    const int64_t items = int64_t(n) * 2 * c.Hkv * (c.D / 8);
    const unsigned blocks = static_cast<unsigned>(min((items + kBlock - 1) / kBlock, int64_t(1) << 22));
    auto go = [&](auto d, auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        paged_rows_kernel<decltype(d)::value, T, P, WRITE><<<blocks, kBlock, 0, s>>>(
            c, seq, pos, items, static_cast<T*>(k), ldk, static_cast<T*>(v), ldv);
    };
    const std::integral_constant<int, 64> d64;
    const std::integral_constant<int, 128> d128;
    if (dtype == PP_BF16) {
        if (c.kv_type == PP_KV_I8) go(d128, bf16{}, int8_t{});
        else go(d128, bf16{}, bf16{});
    } else if (c.kv_type == PP_KV_I8) {
        if (c.D == 64) go(d64, 0.f, int8_t{});
        else go(d128, 0.f, int8_t{});
    } else {
        if (c.D == 64) go(d64, 0.f, 0.f);
        else go(d128, 0.f, 0.f);
    }
}

}  // namespace

namespace ppk {

void paged_write(int dtype, const PagedCache& c, const int32_t* seq, const int32_t* pos, int n, const void* k,
                 int64_t ldk, const void* v, int64_t ldv, hipStream_t s) {
    rows<true>(dtype, c, seq, pos, n, const_cast<void*>(k), ldk, const_cast<void*>(v), ldv, s);
}

void paged_read(int dtype, const PagedCache& c, const int32_t* seq, const int32_t* pos, int n, void* k, int64_t ldk,
                void* v, int64_t ldv, hipStream_t s) {
    rows<false>(dtype, c, seq, pos, n, k, ldk, v, ldv, s);
}

void paged_append(int dtype, const PagedCache& c, const int32_t* lens, const void* qkv, int64_t ldqkv, void* q_out,
                  int64_t ldq, float theta, hipStream_t s) {
    auto go = [&](auto d, auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr int D = decltype(d)::value, heads = kBlock / (D / 16);
        const dim3 grid(c.k, (c.H + 2 * c.Hkv + heads - 1) / heads);
        paged_append_kernel<D, T, P><<<grid, kBlock, 0, s>>>(c, lens, static_cast<const T*>(qkv), ldqkv,
                                                             static_cast<T*>(q_out), ldq, static_cast<double>(theta));
    };
    const std::integral_constant<int, 64> d64;
    const std::integral_constant<int, 128> d128;
    if (dtype == PP_BF16) {
        if (c.kv_type == PP_KV_I8) go(d128, bf16{}, int8_t{});
        else go(d128, bf16{}, bf16{});
    } else if (c.kv_type == PP_KV_I8) {
        if (c.D == 64) go(d64, 0.f, int8_t{});
        else go(d128, 0.f, int8_t{});
    } else {
        if (c.D == 64) go(d64, 0.f, 0.f);
        else go(d128, 0.f, 0.f);
    }
}

}  // namespace ppk
