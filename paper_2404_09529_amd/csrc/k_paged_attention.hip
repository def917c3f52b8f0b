// Attention of one query row per sequence over a paged cache: out = softmax(q k^T / sqrt(D)) v over the
// first lens[i] keys of sequence i, in whatever pages they lie.
//
// One wavefront per (sequence, query head), keys in tiles of 64: lane j holds key j's score, one maximum and one sum
// across the lanes per tile, then lane d accumulates dims d (and d + 64).
#include "device.h"
#include "kernels.h"
#include "paged.h"
#include "prepack.h"

namespace {

constexpr int kBlock = 256;

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(bf16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float value(int8_t x) { return static_cast<float>(x); }

template <int D, typename T, typename P>
__global__ __launch_bounds__(kBlock) void paged_attention_kernel(ppk::PagedCache c, const int32_t* __restrict__ lens,
                                                                 const T* __restrict__ q, int64_t ldq,
                                                                 T* __restrict__ out, float scale) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t wid = int64_t(blockIdx.x) * (kBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = static_cast<int>(wid / c.H), h = static_cast<int>(wid % c.H), g = h / (c.H / c.Hkv);
    if (i >= c.k) return;
    const int n = ppk::paged_len(lens[i], ppk::paged_span(c.max_pages, c.shift));
    const T* qr = q + i * ldq + int64_t(h) * D;
    const P* K = static_cast<const P*>(c.kp) + int64_t(g) * D;
    const P* V = static_cast<const P*>(c.vp) + int64_t(g) * D + lane;
    const int64_t ld = int64_t(c.Hkv) * D;
    float m = -INFINITY, l = 0.f, acc[E] = {};
    bool any = false;
    for (int j0 = 0; j0 < n; j0 += 64) {
        const int j = j0 + lane;
        const int row = j < n ? ppk::paged_row(c.table[int64_t(i) * c.max_pages + (j >> c.shift)], c.n_pages, j, c.shift) : -1;
        float s = -INFINITY, vs = 1.f;
        if (row >= 0) {
            const P* k = K + row * ld;
            float d4[4] = {0.f, 0.f, 0.f, 0.f};
            for (int e = 0; e < D; e += 4)
#pragma unroll
                for (int u = 0; u < 4; ++u) d4[u] = fmaf(value(qr[e + u]), value(k[e + u]), d4[u]);
            s = (d4[0] + d4[1]) + (d4[2] + d4[3]);
            if constexpr (sizeof(P) == 1) {
                s *= c.ks[int64_t(row) * c.Hkv + g];
                vs = c.vs[int64_t(row) * c.Hkv + g];
            }
            s *= scale;
        }
        const uint64_t here = __ballot(row >= 0);
        if (!here) continue;
        any = true;
        const float m_new = fmaxf(m, wave_max(s));
        const float corr = m == m_new ? 1.f : expf(m - m_new);
        // scores of -inf alone add nothing yet; if none follows, 0 / 0 is no number, as the formula has it
        const float p = row < 0 || m_new == -INFINITY ? 0.f : expf(s - m_new);
        l = l * corr + wave_sum(p);
        m = m_new;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= corr;
        const float pv = row < 0 ? 0.f : p * vs;
        for (int t = 0; t < 64; ++t) {
            const int r = __builtin_amdgcn_readlane(row, t);
            if (r < 0) continue;
            const float pt = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(pv), t));
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(pt, value(V[r * ld + 64 * e]), acc[e]);
        }
    }
    T* o = out + (int64_t(i) * c.H + h) * D + lane;
#pragma unroll
    for (int e = 0; e < E; ++e) o[64 * e] = static_cast<T>(any ? acc[e] / l : 0.f);
}

}  // namespace

namespace ppk {

size_t paged_attention_workspace(int, int, int, int) { return 0; }

void paged_attention(int dtype, const PagedCache& c, const int32_t* lens, const void* q, int64_t ldq, void* out, void*,
                     hipStream_t s) {
    const unsigned blocks = static_cast<unsigned>((int64_t(c.k) * c.H + kBlock / kWave - 1) / (kBlock / kWave));
    const float scale = 1.0f / sqrtf(static_cast<float>(c.D));
    auto go = [&](auto d, auto t, auto p) {
        using T = decltype(t);
        paged_attention_kernel<decltype(d)::value, T, decltype(p)><<<blocks, kBlock, 0, s>>>(
            c, lens, static_cast<const T*>(q), ldq, static_cast<T*>(out), scale);
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
