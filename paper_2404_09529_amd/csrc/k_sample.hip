// Sampling: a token of every row of logits with temperature, top-k, top-p and min-p, from a given random
// number.
//
// With the row's ids in order (largest logit first, ties lowest id first) every step asks for the first place where a
// running count or sum passes a bound: top-k by count, top-p by sum, and the token itself by sum.  Weights are
// multiples of 2^-44 of the largest, so sums are exact, whatever their order, and no sort is needed: a place is found by
// descent through the logit's bits.
//
// One workgroup per row, eight bits of the logit at a time: a histogram of counts and sums, the bin in which the bound is
// passed, then the next eight bits of that bin's ids; equal logits have equal weights, and the id among them is counted off.
#include "device.h"
#include "kernels.h"
#include "prepack.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr double kUnit = 0x1p44;
typedef unsigned long long u64;

enum Bound { kCount, kReaches, kExceeds };   // count >= bound; sum >= bound; sum > bound

struct Totals {
    u64 sum;
    uint32_t count;
};

// Integers ordered as the logits are (NaN excepted); both zeros are one.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}

struct Row {
    const float* x;
    int vocab;
    float top;       // the largest logit
    double inv_t;

    __device__ __forceinline__ u64 weight(float v) const {
        if (!(v > -INFINITY)) return 0;
        if (v == top) return static_cast<u64>(kUnit);
        if (top == INFINITY) return 0;
        return static_cast<u64>(rint(exp((static_cast<double>(v) - static_cast<double>(top)) * inv_t) * kUnit));
    }
};

struct Lds {
    u64 sum[256];
    uint32_t count[256];
    Totals wave[kWaves];
    float top[kWaves];
    int id[kWaves];
    // what one wavefront found for all
    int digit;
    u64 above_sum;
    uint32_t above_count;
    int found;
};

__device__ __forceinline__ bool passes(Bound b, u64 sum, uint32_t count, double bound) {
    return b == kCount ? count >= bound : b == kReaches ? static_cast<double>(sum) >= bound : static_cast<double>(sum) > bound;
}

struct Place {
    int id;
    u64 sum;   // of the ids up to this one
    float x;
};

// The first place, in order, where the running count or sum passes the bound; there is one.
__device__ Place find(const Row& r, Bound what, double bound, Lds& lds) {
    const int tid = threadIdx.x, lane = tid & 63;
    uint32_t prefix = 0, mask = 0;
    u64 above = 0;
    uint32_t above_n = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) lds.sum[tid] = 0, lds.count[tid] = 0;
        __syncthreads();
        for (int v = tid; v < r.vocab; v += kThreads) {
            const float x = r.x[v];
            const u64 w = r.weight(x);
            const uint32_t k = key_of(x);
            if (w && (k & mask) == prefix) {
                atomicAdd(&lds.sum[(k >> shift) & 255], w);
                atomicAdd(&lds.count[(k >> shift) & 255], 1u);
            }
        }
        __syncthreads();
        if (tid < 64) {   // digits from 255 down, four a lane
            u64 s[4], ls = 0;
            uint32_t n[4], ln = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ls += s[e] = lds.sum[255 - 4 * lane - e];
                ln += n[e] = lds.count[255 - 4 * lane - e];
            }
            u64 is = ls;
            uint32_t in = ln;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const u64 os = __shfl_up(is, o, 64);
                const uint32_t on = __shfl_up(in, o, 64);
                if (lane >= o) is += os, in += on;
            }
            u64 rs = above + is - ls;
            uint32_t rn = above_n + in - ln;
            if (!passes(what, rs, rn, bound) && passes(what, above + is, above_n + in, bound)) {   // one lane
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u64 ns = rs + s[e];
                    const uint32_t nn = rn + n[e];
                    if (!passes(what, rs, rn, bound) && passes(what, ns, nn, bound))
                        lds.digit = 255 - 4 * lane - e, lds.above_sum = rs, lds.above_count = rn;
                    rs = ns, rn = nn;
                }
            }
        }
        __syncthreads();
        above = lds.above_sum, above_n = lds.above_count;
        prefix |= static_cast<uint32_t>(lds.digit) << shift;
        mask |= 255u << shift;
    }
    // equal logits: the number of them that passes the bound, then the id
    const float x = __uint_as_float(prefix >> 31 ? prefix ^ 0x80000000u : ~prefix);
    const u64 w = r.weight(x);
    uint32_t lo = 1, hi = r.vocab;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (passes(what, above + w * mid, above_n + mid, bound)) hi = mid;
        else lo = mid + 1;
    }
    uint32_t before = 0;
    for (int v0 = 0; v0 < r.vocab; v0 += kThreads) {
        const bool is = v0 + tid < r.vocab && r.x[v0 + tid] == x;
        const u64 b = __ballot(is);
        __syncthreads();
        if (lane == 0) lds.count[tid >> 6] = __popcll(b);
        __syncthreads();
        uint32_t mine = before, all = 0;
        for (int k = 0; k < kWaves; ++k) {
            if (k < (tid >> 6)) mine += lds.count[k];
            all += lds.count[k];
        }
        if (is && mine + __popcll(b & ((1ull << lane) - 1)) == lo - 1) lds.found = v0 + tid;
        before += all;
        if (before >= lo) break;
    }
    __syncthreads();
    const int id = lds.found;
    __syncthreads();
    return {id, above + w * lo, x};
}

__device__ Totals block_totals(Totals t, Lds& lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t.sum += __shfl_xor(t.sum, o, 64), t.count += __shfl_xor(t.count, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds.wave[threadIdx.x >> 6] = t;
    __syncthreads();
    Totals a{0, 0};
    for (int k = 0; k < kWaves; ++k) a.sum += lds.wave[k].sum, a.count += lds.wave[k].count;
    return a;
}

__global__ __launch_bounds__(kThreads) void sample_kernel(ppk::Sample a) {
    __shared__ Lds lds;
    const int row = blockIdx.x, tid = threadIdx.x;
    Row r{a.logits + row * a.ldl, a.vocab, -INFINITY, 1.0};
    // the largest logit, and the lowest id that has it
    int id = INT32_MAX;
    float top = -INFINITY;
    for (int v = tid; v < a.vocab; v += kThreads) {
        const float x = r.x[v];
        if (x > top || (x == top && id == INT32_MAX)) top = x, id = v;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float ot = __shfl_xor(top, o, 64);
        const int oi = __shfl_xor(id, o, 64);
        if (ot > top || (ot == top && oi < id)) top = ot, id = oi;
    }
    if ((tid & 63) == 0) lds.top[tid >> 6] = top, lds.id[tid >> 6] = id;
    __syncthreads();
    for (int k = 0; k < kWaves; ++k)
        if (lds.top[k] > top || (lds.top[k] == top && lds.id[k] < id)) top = lds.top[k], id = lds.id[k];
    const float t = a.temperature ? a.temperature[row] : 1.0f;
    const bool greedy = !(t > 0.f);
    if (greedy || top == -INFINITY) {
        if (tid == 0) {
            const bool none = id == INT32_MAX || !greedy;
            a.tokens[row] = none ? -1 : id;
            if (a.prob) a.prob[row] = none ? 0.f : 1.f;
        }
        return;
    }
    r.top = top;
    r.inv_t = 1.0 / static_cast<double>(t);
    const float mp = a.min_p ? a.min_p[row] : 0.f;
    const double min_p = mp > 0.f ? fmin(static_cast<double>(mp), 1.0) : 0.0;
    Totals all{0, 0}, likely{0, 0};
    for (int v = tid; v < a.vocab; v += kThreads) {
        const float x = r.x[v];
        const u64 w = r.weight(x);
        if (w) {
            all.sum += w, ++all.count;
            if (x == top || exp((static_cast<double>(x) - static_cast<double>(top)) * r.inv_t) >= min_p)
                likely.sum += w, ++likely.count;
        }
    }
    all = block_totals(all, lds);
    likely = block_totals(likely, lds);
    u64 kept = all.sum;
    const int top_k = a.top_k ? a.top_k[row] : 0;
    if (top_k > 0 && static_cast<uint32_t>(top_k) < all.count) kept = find(r, kCount, top_k, lds).sum;
    const float tp = a.top_p ? a.top_p[row] : 1.f;
    if (tp < 1.f) kept = find(r, kReaches, fmax(static_cast<double>(tp) * static_cast<double>(kept), 1.0), lds).sum;
    kept = min(kept, likely.sum);
    const float uf = a.u[row];
    const double u = uf >= 0.f ? uf : 0.0, sum = static_cast<double>(kept);
    const Place p = find(r, kExceeds, u < 1.0 ? fmin(u * sum, nextafter(sum, 0.0)) : nextafter(sum, 0.0), lds);
    if (tid == 0) {
        a.tokens[row] = p.id;
        if (a.prob) {
            const double w = p.x == top ? 1.0 : exp((static_cast<double>(p.x) - static_cast<double>(top)) * r.inv_t);
            a.prob[row] = static_cast<float>(w * (kUnit / sum));
        }
    }
}

}  // namespace

namespace ppk {

size_t sample_workspace(int, int) { return 0; }

void sample(const Sample& a, hipStream_t s) { sample_kernel<<<a.k, kThreads, 0, s>>>(a); }

}  // namespace ppk
