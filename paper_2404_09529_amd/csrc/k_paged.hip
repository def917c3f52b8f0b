// A paged cache's rows: written from dense rows (a prefill's caches), read back, and appended to by a
// decode step with the rotation of its query and key (RESTART-PE: a sequence's positions are its own).
//
// A head's row of D values is D / 16 lanes' (8 for D = 128), side by side, so that its scale is a maximum over few
// lanes; a lane has 8 values of each half of the row, the pairs that are rotated together, and every load is of whole lines.
// Memory bounds the rows' kernels.  24,349 rows of 32 heads of 128: into 8-bit pages (604 MB) 125 us by itself, 4.8 TB/s, and 143
// behind a kernel whose 403 MB are still on their way to memory; back 102 us, 5.9 TB/s; 20,140 rows of 8 heads back 27-28 us, 4.5
// TB/s.  The append is latency: 2.9 us for one sequence, 4.4 for 64 (32 heads, 8-bit pages).
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
    // the neighbour, the other pair, then the lane opposite in 8 and in 16
    auto with = [&](auto control) {
        top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(top), control(), 0xf, 0xf, true)));
    };
    with([] { return 0xb1; });
    with([] { return 0x4e; });
    if constexpr (LANES >= 8) with([] { return 0x141; });
    if constexpr (LANES >= 16) with([] { return 0x140; });
    return row_code(top);
}

// A lane's 16 values of a head's row, 8 from dst on and 8 half a row behind; `lane` of the head's.
template <int LANES, typename P>
__device__ __forceinline__ void store_head(P* dst, float* scale, const float (&v)[16], int lane) {
    constexpr int HALF = 8 * LANES;
    if constexpr (sizeof(P) == 1) {
        const RowCode rc = head_code<LANES>(v);
        *reinterpret_cast<uint2*>(dst) = make_uint2(codes4(v, rc), codes4(v + 4, rc));
        *reinterpret_cast<uint2*>(dst + HALF) = make_uint2(codes4(v + 8, rc), codes4(v + 12, rc));
        if (lane == 0) *scale = rc.scale;
    } else {
        store8(dst, v);
        store8(dst + HALF, v + 8);
    }
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

// The table has an entry.  (It is read at a place that exists, whatever is asked for: a load behind a branch is waited for
// at once.)
__device__ __forceinline__ int32_t place(const ppk::PagedCache& c, int32_t seq, int32_t pos) {
    const bool in = seq >= 0 && seq < c.k && pos >= 0 && (pos >> c.shift) < c.max_pages;
    const int32_t page = c.table[in ? int64_t(seq) * c.max_pages + (pos >> c.shift) : 0];
    return in ? ppk::paged_row(page, c.n_pages, pos, c.shift) : -1;
}

// A thread has dims j .. j + 7 and D / 2 + j .. + 7 of a head's row (one of 2 Hkv D / 16 columns, those of the keys first)
// and kAhead rows on the way at once; a workgroup has `wide` columns of kBlock / wide rows, kAhead times.  In us, the rows of 32
// heads written and read back in turn: 8 values a thread and one row at a time 149 and 120, two 156 and 151, four 156 and 117,
// eight 154 and 108; 16 values and two rows 144 and 102, four 148 and 101, and few rows are slower then (459 rows of 16 heads into bf16
// pages: 3.8 and 4.1); 16 neighbouring values, codes in whole pieces of 16 bytes, 143 and 120.
constexpr int kAhead = 2;
template <int D, typename T, typename P, bool WRITE>
__global__ __launch_bounds__(kBlock) void paged_rows_kernel(ppk::PagedCache c, const int32_t* __restrict__ seq,
                                                            const int32_t* __restrict__ pos, int rows, T* k, int64_t ldk,
                                                            T* v, int64_t ldv, int wide, int col_blocks) {
    constexpr int LANES = D / 16, HALF = D / 2;
    const int half = c.Hkv * LANES, tall = kBlock / wide, local = threadIdx.x / wide;
    const int col = blockIdx.x % col_blocks * wide + threadIdx.x - local * wide;
    const int64_t first = int64_t(blockIdx.x / col_blocks) * tall * kAhead + local;
    if (local >= tall || col >= 2 * half || first >= rows) return;   // (heads as a whole)
    const bool val = col >= half;
    const int lane = col % LANES, head = (val ? col - half : col) / LANES, in_row = head * D + lane * 8;
    T* dense = (val ? v : k) + in_row;
    const int64_t ld = val ? ldv : ldk;
    P* pages = static_cast<P*>(val ? c.vp : c.kp) + in_row;
    float* scales = (val ? c.vs : c.ks) + head;
    float y[kAhead][16];
    int32_t s[kAhead], p[kAhead], row[kAhead];
    int64_t r[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        r[u] = min(first + int64_t(u) * tall, int64_t(rows) - 1);   // (loads stay in range)
        s[u] = seq[r[u]];
        p[u] = pos[r[u]];
    }
    if constexpr (WRITE) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            load8(dense + r[u] * ld, y[u]);
            load8(dense + r[u] * ld + HALF, y[u] + 8);
        }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) row[u] = place(c, s[u], p[u]);
    if constexpr (!WRITE) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t at = int64_t(max(row[u], 0)) * c.Hkv;
            load_row8(pages, scales, at * D, at, y[u]);
            load_row8(pages, scales, at * D + HALF, at, y[u] + 8);
        }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        if (row[u] < 0 || first + int64_t(u) * tall >= rows) continue;
        const int64_t at = int64_t(row[u]) * c.Hkv;
        if constexpr (!WRITE) {
            store8(dense + r[u] * ld, y[u]);
            store8(dense + r[u] * ld + HALF, y[u] + 8);
        } else {
            store_head<LANES>(pages + at * D, scales + at, y[u], lane);
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
    float x[16];
    if (live) {
        const T* src = qkv + i * ldqkv + int64_t(head) * D + j;
        load8(src, x);
        load8(src + HALF, x + 8);
    }
    if (threadIdx.x < HALF) angle[threadIdx.x] = rope_entry(pos, threadIdx.x, D, theta);
    __syncthreads();
    if (!live) return;
    if (head < c.H + c.Hkv) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double lo = x[e], hi = x[e + 8], cs = angle[j + e].x, sn = angle[j + e].y;
            x[e] = static_cast<float>(lo * cs - hi * sn);
            x[e + 8] = static_cast<float>(hi * cs + lo * sn);
        }
    }
    if (head < c.H) {
        T* q = q_out + i * ldq + int64_t(head) * D + j;
        store8(q, x);
        store8(q + HALF, x + 8);
        return;
    }
    if (c.max_pages == 0) return;
    const int32_t row = place(c, i, pos);
    if (row < 0) return;
    const bool val = head >= c.H + c.Hkv;
    const int64_t head_row = int64_t(row) * c.Hkv + head - c.H - (val ? c.Hkv : 0);
    store_head<LANES>(static_cast<P*>(val ? c.vp : c.kp) + head_row * D + j, (val ? c.vs : c.ks) + head_row, x, j / 8);
}

template <bool WRITE>
void rows(int dtype, const ppk::PagedCache& c, const int32_t* seq, const int32_t* pos, int n, void* k, int64_t ldk,
          void* v, int64_t ldv, hipStream_t s) {
    if (c.max_pages == 0) return;   // no row has a place
    // columns of a workgroup: whole heads
    const int cols = 2 * c.Hkv * (c.D / 16), wide = min(cols, kBlock), col_blocks = (cols + wide - 1) / wide;
    const int64_t per_block = int64_t(kBlock / wide) * kAhead;
    const unsigned blocks = static_cast<unsigned>((n + per_block - 1) / per_block * col_blocks);
    auto go = [&](auto d, auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        paged_rows_kernel<decltype(d)::value, T, P, WRITE><<<blocks, kBlock, 0, s>>>(
            c, seq, pos, n, static_cast<T*>(k), ldk, static_cast<T*>(v), ldv, wide, col_blocks);
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
