// Sampling: a token of every row of logits with temperature, top-k, top-p and min-p, from a given random
// number.
//
// With the row's ids in order (largest logit first, ties lowest id first) every setting, and the choice itself, asks for
// the first place where a running count or sum passes a bound.  No row is sorted for that.  In powers of two, y =
// x log2(e) / T, the weight 2^y is cut into bins of 1/32 octave below an integer exponent E; sums of weights are integers,
// multiples of 2^(E - 44), the same in whatever order they are formed.
//   hist_kernel    a part of a row: its largest logit, E = ceil of its y, and the sum (and for top-k the count) of
//                  every bin.  E is the part's own: parts differ by whole octaves, that is by shifts, so no pass over the
//                  row has to come before to find its largest logit.
//   gather_kernel  the parts' bins together; the bins in which the bounds are passed, or several where one bound depends
//                  on another's exact place; the part's ids in these bins into the row's list.
//   pick_kernel    the list in order, running sums behind what the bins before hold, and the places themselves.  A list that is
//                  too long (thousands of nearly equal logits) is resolved by descent through the logit's bits instead.
// Rows are split into up to 16 parts, so that a few rows fill the chip: the logits are read three times, twice of them
// from L2 (MEASURED).
#include <algorithm>

#include "device.h"
#include "kernels.h"
#include "prepack.h"

namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kUnitBits = 44, kPerOctave = 32;
constexpr int kBins = 46 * kPerOctave;          // weights below 2^-45 are none
constexpr int kScan = 3 * kThreads;             // bins as the threads hold them, three each
constexpr int kList = 4096, kMaxParts = 16;
static_assert(kScan >= kBins, "three bins a thread");
typedef unsigned long long u64;

// Integers ordered as the logits are (NaN excepted); both zeros are one.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k >> 31 ? k ^ 0x80000000u : ~k); }

// ------------------------------------------------------------------------------- weights
// 2^(i / 64), filled by the first wavefront; a barrier follows.
struct Powers {
    double at[64];
    __device__ __forceinline__ void fill() {
        if (threadIdx.x < 64) at[threadIdx.x] = exp2(threadIdx.x / 64.0);
    }
};

struct Scale {
    double c;   // log2(e) / T
    double E;   // exponent of the unit's 2^44
    // How far x's y is below E, in octaves; NaN and -inf and what is too far below give no number below 46.
    __device__ __forceinline__ double depth(float x) const {
#pragma clang fp contract(off)
        if (E == INFINITY) return x == INFINITY ? 0.0 : 64.0;
        return E - y_of(x, c);
    }
    // Rounded, here and in E: one unrounded in a fused operation would not be E's own y where that is large.
    static __device__ __forceinline__ double y_of(float x, double c) {
#pragma clang fp contract(off)
        const double y = static_cast<double>(x) * c;
        return y;
    }
};
__device__ __forceinline__ double exponent_of(float top, double c) { return top == INFINITY ? INFINITY : ceil(Scale::y_of(top, c)); }
__device__ __forceinline__ double scale_of(float t) { return 1.4426950408889634 / static_cast<double>(t); }
__device__ __forceinline__ int bin_of(double depth) { return static_cast<int>(depth * kPerOctave); }
__device__ __forceinline__ bool live(double depth) { return depth < 45.0; }   // false for NaN

// 2^(44 - depth) rounded: a 64th of an octave from the table, the rest, |r| <= ln 2 / 128, by the exponential's
// series to the fifth power (the next term is below 2^-54); adding 2^52 leaves the integer in the low bits.
__device__ __forceinline__ double power(double depth, const Powers& p) {
    const double z = -64.0 * depth, n = rint(z), r = (z - n) * (0.69314718055994531 / 64.0);
    const int i = static_cast<int>(n);
    double s = fma(r, 1.0 / 120.0, 1.0 / 24.0);
    s = fma(s, r, 1.0 / 6.0);
    s = fma(s, r, 0.5);
    s = fma(s, r, 1.0);
    const double t = p.at[i & 63];
    return ldexp(fma(t, s * r, t), i >> 6);   // 2^-depth
}
__device__ __forceinline__ u64 weight(double depth, const Powers& p) {
    const double w = fma(power(depth, p), static_cast<double>(1ull << kUnitBits), 0x1p52);
    return static_cast<u64>(__double_as_longlong(w)) & ((1ull << 52) - 1);
}

// ------------------------------------------------------------------------------- a row's settings and workspace
struct Settings {
    float t;
    int top_k;
    double top_p, min_p, u;   // 1 and more: no limit; 0: no limit; in [0, 1]
    bool greedy;
};
__device__ __forceinline__ Settings settings_of(const ppk::Sample& a, int row) {
    Settings s;
    s.t = a.temperature ? a.temperature[row] : 1.f;
    s.greedy = !(s.t > 0.f);
    s.top_k = a.top_k ? max(a.top_k[row], 0) : 0;
    const float p = a.top_p ? a.top_p[row] : 1.f, m = a.min_p ? a.min_p[row] : 0.f, u = a.u[row];
    s.top_p = p < 1.f ? static_cast<double>(p) : 1.0;
    s.min_p = m > 0.f ? fmin(static_cast<double>(m), 1.0) : 0.0;
    s.u = u >= 0.f ? static_cast<double>(u) : 0.0;
    return s;
}
// The bound that the chosen id's running sum exceeds; it is below the sum.
__device__ __forceinline__ double choice_bound(double u, double sum) {
    const double below = nextafter(sum, 0.0);
    return u < 1.0 ? fmin(u * sum, below) : below;
}

struct Part {   // of a row, by hist_kernel
    double E;   // -inf: no id that may be chosen
    float top;
    int id;     // the lowest that has the largest logit; INT32_MAX: every logit is NaN
};
struct Plan {   // of a row, by gather_kernel
    double E;
    float top;
    int listed;       // ids in the list, also those that found no room; cleared by hist_kernel
    int k_bin;        // top-k's bin (-1: no limit), and the ids before it
    int k_before;
    int m_bin;        // first bin in which min_p's border may lie
    u64 all;
    u64 before[kBins];
    u64 list[kList];
};
struct Space {
    u64* sum;         // [k][parts][kBins]
    uint32_t* count;  // [k][parts][kBins]
    Part* part;       // [k][parts]
    Plan* plan;       // [k]
};
size_t space_bytes(int k, int parts) {
    return size_t(k) * parts * (kBins * 12 + sizeof(Part)) + size_t(k) * sizeof(Plan);
}
Space space_at(void* ws, int k, int parts) {
    Space s;
    s.plan = static_cast<Plan*>(ws);
    s.sum = reinterpret_cast<u64*>(s.plan + k);
    s.part = reinterpret_cast<Part*>(s.sum + size_t(k) * parts * kBins);
    s.count = reinterpret_cast<uint32_t*>(s.part + size_t(k) * parts);
    return s;
}

// f(x, id) for the ids v0 <= id < v1 of a row, eight loads of a thread in flight.
template <typename F>
__device__ __forceinline__ void over(const float* x, int v0, int v1, F f) {
    int v = v0 + threadIdx.x;
    for (; v + 7 * kThreads < v1; v += 8 * kThreads) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[v + i * kThreads];
#pragma unroll
        for (int i = 0; i < 8; ++i) f(y[i], v + i * kThreads);
    }
    for (; v < v1; v += kThreads) f(x[v], v);
}

__device__ __forceinline__ bool above(float t, int i, float u, int j) { return t > u || (t == u && i < j); }

__global__ __launch_bounds__(kThreads) void hist_kernel(ppk::Sample a, Space s, int parts, int size) {
    __shared__ u64 sum[kBins];
    __shared__ uint32_t count[kBins];
    __shared__ Powers powers;
    __shared__ float tops[kWaves];
    __shared__ int ids[kWaves];
    const int row = blockIdx.x / parts, tid = threadIdx.x, v0 = blockIdx.x % parts * size, v1 = min(v0 + size, a.vocab);
    const float* x = a.logits + row * a.ldl;
    const Settings set = settings_of(a, row);
    for (int b = tid; b < kBins; b += kThreads) sum[b] = 0, count[b] = 0;
    powers.fill();
    float top = -INFINITY;
    int id = INT32_MAX;
    over(x, v0, v1, [&](float y, int v) {
        if (y > top || (y == top && id == INT32_MAX)) top = y, id = v;   // (a thread's ids ascend)
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float t = __shfl_xor(top, o, kWave);
        const int i = __shfl_xor(id, o, kWave);
        if (above(t, i, top, id)) top = t, id = i;
    }
    if (tid % kWave == 0) tops[tid / kWave] = top, ids[tid / kWave] = id;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (above(tops[w], ids[w], top, id)) top = tops[w], id = ids[w];
    const double c = scale_of(set.t);
    const bool none = set.greedy || top == -INFINITY;
    const Scale sc = {c, none ? -INFINITY : exponent_of(top, c)};
    if (tid == 0) {
        s.part[blockIdx.x] = {sc.E, top, id};
        if (blockIdx.x % parts == 0) s.plan[row].listed = 0;
    }
    if (none) return;
    const bool counted = set.top_k > 0;
    over(x, v0, v1, [&](float y, int) {
        const double d = sc.depth(y);
        if (!live(d)) return;
        const u64 w = weight(d, powers);
        atomicAdd(&sum[bin_of(d)], w);
        if (counted) atomicAdd(&count[bin_of(d)], 1u);
    });
    __syncthreads();
    const int64_t out = int64_t(blockIdx.x) * kBins;
    for (int b = tid; b < kBins; b += kThreads) {
        s.sum[out + b] = sum[b];
        if (counted) s.count[out + b] = count[b];
    }
}

// ------------------------------------------------------------------------------- scans of a workgroup
template <typename T>
__device__ __forceinline__ T block_scan(T mine, T* waves) {   // up to and including this thread
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const T y = __shfl_up(mine, o, kWave);
        if (lane >= o) mine += y;
    }
    __syncthreads();
    if (lane == kWave - 1) waves[w] = mine;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
        if (i < w) mine += waves[i];
    return mine;
}

// The whole row's parts.
struct Whole {
    double E;
    float top;
    int id;
};
__device__ __forceinline__ Whole whole_of(const Part* p, int parts) {
    Whole w = {-INFINITY, -INFINITY, INT32_MAX};
    for (int i = 0; i < parts; ++i) {
        const Part q = p[i];
        if (above(q.top, q.id, w.top, w.id)) w.top = q.top, w.id = q.id;
        w.E = fmax(w.E, q.E);
    }
    return w;
}
// Octaves from one exponent down to another, both whole numbers.
__device__ __forceinline__ int octaves(double E, double part) { return E == part ? 0 : static_cast<int>(fmin(E - part, 64.0)); }

__global__ __launch_bounds__(kThreads) void gather_kernel(ppk::Sample a, Space s, int parts, int size) {
    __shared__ u64 sums[kScan + 1];        // of the bins before each
    __shared__ uint32_t counts[kScan + 1];
    __shared__ u64 found[kList / 2];
    __shared__ u64 wave_sums[kWaves];
    __shared__ uint32_t wave_counts[kWaves];
    __shared__ int at[6], listed, base;
    const int row = blockIdx.x / parts, part = blockIdx.x % parts, tid = threadIdx.x;
    const Settings set = settings_of(a, row);
    if (set.greedy) return;
    const Part* ps = s.part + int64_t(row) * parts;
    const Whole w = whole_of(ps, parts);
    if (w.E == -INFINITY) return;
    // the bins of all parts: three neighbours a thread
    u64 sum[3] = {0, 0, 0};
    uint32_t count[3] = {0, 0, 0};
    for (int p = 0; p < parts; ++p) {
        if (ps[p].E == -INFINITY) continue;
        const int shift = octaves(w.E, ps[p].E);
        const int64_t src = (int64_t(row) * parts + p) * kBins - kPerOctave * shift;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int b = 3 * tid + i;
            if (shift >= 46 || b >= kBins || b < kPerOctave * shift) continue;
            sum[i] += s.sum[src + b] >> shift;
            if (set.top_k) count[i] += s.count[src + b];
        }
    }
    const u64 se = block_scan(sum[0] + sum[1] + sum[2], wave_sums);
    const uint32_t ce = block_scan(count[0] + count[1] + count[2], wave_counts);
    sums[3 * tid + 3] = se, sums[3 * tid + 2] = se - sum[2], sums[3 * tid + 1] = se - sum[2] - sum[1];
    counts[3 * tid + 3] = ce, counts[3 * tid + 2] = ce - count[2], counts[3 * tid + 1] = ce - count[2] - count[1];
    if (tid == 0) sums[0] = 0, counts[0] = 0, listed = 0;
    if (tid < 6) at[tid] = kBins - 1;
    __syncthreads();
    const u64 all = sums[kScan];
    // at[slot]: the bin in which the sum (or count) passes the bound
    auto passing = [&](int slot, auto before, auto bound) {
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int b = 3 * tid + i;
            if (!bound(before[b]) && bound(before[b + 1])) at[slot] = b;   // one thread
        }
        __syncthreads();
    };
    // bins: top-k's; top-p's first and last; min-p's first and last; the choice's first and last
    const bool has_k = set.top_k > 0 && static_cast<uint32_t>(set.top_k) < counts[kScan], has_p = set.top_p < 1.0;
    u64 lo = all, hi = all;   // of what is kept
    int bk = -1;
    if (has_k) {
        passing(0, counts, [&](uint32_t n) { return n >= static_cast<uint32_t>(set.top_k); });
        bk = at[0];
        lo = sums[bk], hi = sums[bk + 1];
    }
    int p0 = 0, p1 = -1, m0 = 0, m1 = -1;
    if (has_p) {
        const double t0 = fmax(set.top_p * static_cast<double>(lo), 1.0), t1 = fmax(set.top_p * static_cast<double>(hi), 1.0);
        passing(1, sums, [&](u64 n) { return static_cast<double>(n) >= t0; });
        passing(2, sums, [&](u64 n) { return static_cast<double>(n) >= t1; });
        p0 = at[1], p1 = at[2];
        lo = min(lo, sums[p0]), hi = min(hi, sums[p1 + 1]);
    }
    if (set.min_p > 0.0) {
        // 2^-depth = min_p 2^-depth(top), one bin more on both sides
        const double d = Scale{scale_of(set.t), w.E}.depth(w.top) - log2(set.min_p);
        const int b = static_cast<int>(fmin(d, 46.0) * kPerOctave);
        m0 = min(max(b - 1, 0), kBins - 1), m1 = min(b + 1, kBins - 1);
        lo = min(lo, sums[m0]), hi = min(hi, sums[m1 + 1]);
    }
    const double u0 = choice_bound(set.u, fmax(static_cast<double>(lo), 1.0)), u1 = choice_bound(set.u, static_cast<double>(hi));
    passing(3, sums, [&](u64 n) { return static_cast<double>(n) > u0; });
    passing(4, sums, [&](u64 n) { return static_cast<double>(n) > u1; });
    const int s0 = at[3], s1 = at[4];

    Plan* plan = s.plan + row;
    if (part == 0) {
        for (int b = tid; b < kBins; b += kThreads) plan->before[b] = sums[b];
        if (tid == 0) {
            plan->E = w.E, plan->top = w.top, plan->m_bin = m0, plan->all = all;
            plan->k_bin = bk, plan->k_before = bk >= 0 ? static_cast<int>(counts[bk]) : 0;
        }
    }
    if (ps[part].E == -INFINITY) return;
    const Scale sc = {scale_of(set.t), ps[part].E};
    const int shift = octaves(w.E, sc.E) * kPerOctave;
    const int v0 = part * size;
    over(a.logits + row * a.ldl, v0, min(v0 + size, a.vocab), [&](float y, int v) {
        const double d = sc.depth(y);
        if (!live(d)) return;
        const int b = bin_of(d) + shift;
        if (b == bk || (b >= p0 && b <= p1) || (b >= m0 && b <= m1) || (b >= s0 && b <= s1)) {
            const int n = atomicAdd(&listed, 1);
            if (n < kList / 2) found[n] = u64(~key_of(y)) << 32 | static_cast<uint32_t>(v);
        }
    });
    __syncthreads();
    // a part with more than half the list's room: the list is too long, or is taken to be
    const int n = listed;
    if (tid == 0 && n) base = atomicAdd(&plan->listed, n > kList / 2 ? kList + 1 : n);
    __syncthreads();
    for (int i = tid; i < min(n, kList / 2); i += kThreads)
        if (base + i < kList) plan->list[base + i] = found[i];
}

// ------------------------------------------------------------------------------- descent
// Where the list is too long: eight bits of the logit at a time, a histogram of counts and sums, the bin in which the
// bound is passed, then the next eight bits of that bin's ids; equal logits have equal weights, and the id among them is
// counted off.
enum Bound { kCount, kReaches, kExceeds };   // count >= bound; sum >= bound; sum > bound
__device__ __forceinline__ bool passes(Bound b, u64 sum, uint32_t count, double bound) {
    return b == kCount ? count >= bound : b == kReaches ? static_cast<double>(sum) >= bound : static_cast<double>(sum) > bound;
}

struct Place {
    int id;
    u64 sum;   // of the ids up to this one
    float x;
};
struct Descent {
    u64 sum[256];
    uint32_t count[256];
    u64 wave_sum[kWaves];
    uint32_t wave_count[kWaves];
    int digit, found;
    u64 above_sum;
    uint32_t above_count;
};

// The first place, in order, where the running count or sum passes the bound; there is one.
__device__ Place find(const float* x, int vocab, const Scale& sc, const Powers& powers, Bound what, double bound, Descent& lds) {
    const int tid = threadIdx.x, lane = tid % kWave;
    uint32_t prefix = 0, mask = 0, above_n = 0;
    u64 above_s = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) lds.sum[tid] = 0, lds.count[tid] = 0;
        __syncthreads();
        over(x, 0, vocab, [&](float y, int) {
            const uint32_t k = key_of(y);
            if ((k & mask) != prefix) return;
            const double d = sc.depth(y);
            if (!live(d)) return;
            atomicAdd(&lds.sum[(k >> shift) & 255], weight(d, powers));
            atomicAdd(&lds.count[(k >> shift) & 255], 1u);
        });
        __syncthreads();
        const u64 s = tid < 256 ? lds.sum[255 - tid] : 0;   // digits from 255 down
        const uint32_t n = tid < 256 ? lds.count[255 - tid] : 0;
        const u64 es = above_s + block_scan(s, lds.wave_sum);
        const uint32_t en = above_n + block_scan(n, lds.wave_count);
        if (tid < 256 && !passes(what, es - s, en - n, bound) && passes(what, es, en, bound))
            lds.digit = 255 - tid, lds.above_sum = es - s, lds.above_count = en - n;
        __syncthreads();
        above_s = lds.above_sum, above_n = lds.above_count;
        prefix |= static_cast<uint32_t>(lds.digit) << shift;
        mask |= 255u << shift;
    }
    const float v = of_key(prefix);
    const u64 w = weight(sc.depth(v), powers);
    uint32_t lo = 1, hi = vocab;   // the number of equal logits that passes
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (passes(what, above_s + w * mid, above_n + mid, bound)) hi = mid;
        else lo = mid + 1;
    }
    uint32_t before = 0;
    for (int v0 = 0; v0 < vocab; v0 += kThreads) {
        const bool is = v0 + tid < vocab && x[v0 + tid] == v;
        const u64 here = __ballot(is);
        __syncthreads();
        if (lane == 0) lds.wave_count[tid / kWave] = __popcll(here);
        __syncthreads();
        uint32_t mine = before, all = 0;
        for (int i = 0; i < kWaves; ++i) {
            if (i < tid / kWave) mine += lds.wave_count[i];
            all += lds.wave_count[i];
        }
        if (is && mine + __popcll(here & ((1ull << lane) - 1)) == lo - 1) lds.found = v0 + tid;
        before += all;
        if (before >= lo) break;
    }
    __syncthreads();
    const int id = lds.found;
    __syncthreads();
    return {id, above_s + w * lo, v};
}

__device__ Place descend(const float* x, int vocab, const Settings& set, const Scale& sc, float top, const Powers& powers,
                         Descent& lds) {
    u64 all = 0, likely = 0;
    uint32_t count = 0;
    over(x, 0, vocab, [&](float y, int) {
        const double d = sc.depth(y);
        if (!live(d)) return;
        const u64 w = weight(d, powers);
        all += w, ++count;
        if (y == top || power(d - sc.depth(top), powers) >= set.min_p) likely += w;
    });
    auto total = [&](auto v, auto* waves) {
        v = block_scan(v, waves);
        __syncthreads();
        if (threadIdx.x == kThreads - 1) waves[0] = v;
        __syncthreads();
        v = waves[0];
        __syncthreads();
        return v;
    };
    u64 kept = total(all, lds.wave_sum);
    likely = total(likely, lds.wave_sum);
    count = total(count, lds.wave_count);
    if (set.top_k && static_cast<uint32_t>(set.top_k) < count) kept = find(x, vocab, sc, powers, kCount, set.top_k, lds).sum;
    if (set.top_p < 1.0)
        kept = find(x, vocab, sc, powers, kReaches, fmax(set.top_p * static_cast<double>(kept), 1.0), lds).sum;
    kept = min(kept, likely);
    Place p = find(x, vocab, sc, powers, kExceeds, choice_bound(set.u, static_cast<double>(kept)), lds);
    p.sum = kept;
    return p;
}

// ------------------------------------------------------------------------------- the choice
__global__ __launch_bounds__(kThreads) void pick_kernel(ppk::Sample a, Space s, int parts) {
    __shared__ u64 list[kList];   // what of the order stands in the id's stead: ~key, id
    __shared__ u64 run[kList];    // running sums of the list's weights
    __shared__ union {
        Descent descent;
        u64 waves[kWaves];
    } lds;
    __shared__ Powers powers;
    __shared__ int first;
    __shared__ u64 likely;
    const int row = blockIdx.x, tid = threadIdx.x;
    const Settings set = settings_of(a, row);
    const Part* ps = s.part + int64_t(row) * parts;
    if (set.greedy || whole_of(ps, parts).E == -INFINITY) {
        const Whole w = whole_of(ps, parts);
        const bool none = w.id == INT32_MAX || !set.greedy;
        if (tid == 0) {
            a.tokens[row] = none ? -1 : w.id;
            if (a.prob) a.prob[row] = none ? 0.f : 1.f;
        }
        return;
    }
    powers.fill();
    const Plan* plan = s.plan + row;
    const Scale sc = {scale_of(set.t), plan->E};
    const float top = plan->top;
    const int n = plan->listed;
    auto write = [&](int id, float x, u64 kept) {   // by one thread
        a.tokens[row] = id;
        if (a.prob)
            a.prob[row] = static_cast<float>(power(sc.depth(x), powers) * (static_cast<double>(1ull << kUnitBits) / static_cast<double>(kept)));
    };
    if (n > kList || n == 0) {
        __syncthreads();
        const Place p = descend(a.logits + row * a.ldl, a.vocab, set, sc, top, powers, lds.descent);
        if (tid == 0) write(p.id, p.x, p.sum);
        return;
    }
    // bitonic sort of the next power of two, two values a thread and step at most kList / kThreads / 2 times
    int m = 64;
    while (m < n) m *= 2;
    for (int i = tid; i < m; i += kThreads) list[i] = i < n ? plan->list[i] : ~0ull;
    for (int size = 2; size <= m; size *= 2)
        for (int stride = size / 2; stride > 0; stride /= 2) {
            __syncthreads();
            for (int i = tid; i < m / 2; i += kThreads) {
                const int lo = 2 * i - (i & (stride - 1)), hi = lo + stride;
                const u64 x = list[lo], y = list[hi];
                if ((x > y) == ((lo & size) == 0)) list[lo] = y, list[hi] = x;
            }
        }
    __syncthreads();
    // running sums: eight neighbours a thread
    const int per = (m + kThreads - 1) / kThreads;
    auto x_of = [&](int i) { return of_key(~static_cast<uint32_t>(list[i] >> 32)); };
    u64 mine = 0;
    for (int i = tid * per; i < min(tid * per + per, n); ++i) mine += weight(sc.depth(x_of(i)), powers);
    u64 sum = block_scan(mine, lds.waves) - mine;
    for (int i = tid * per; i < min(tid * per + per, n); ++i) run[i] = sum += weight(sc.depth(x_of(i)), powers);
    if (tid == 0) likely = plan->before[plan->m_bin];
    __syncthreads();
    struct Sum {
        u64 sum;    // of all ids up to list entry i: the bins before its own, and the list's entries of its bin
        int bin, rank;   // among the bin's
    };
    auto upto = [&](int i) {
        const int b = bin_of(sc.depth(x_of(i)));
        int lo = 0, hi = i;   // the first entry of the bin
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (bin_of(sc.depth(x_of(mid))) < b) lo = mid + 1;
            else hi = mid;
        }
        return Sum{plan->before[min(b, kBins - 1)] + run[i] - (lo ? run[lo - 1] : 0), b, i - lo};
    };
    // The first entry that passes; the last one if a sum of parts and one of ids differ in their last bits just here.
    auto place = [&](auto bound) {
        __syncthreads();
        if (tid == 0) first = n - 1;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads)
            if (bound(i)) {
                atomicMin(&first, i);
                break;
            }
        __syncthreads();
        return first;
    };
    u64 kept = plan->all;
    if (plan->k_bin >= 0) {
        const int rank = set.top_k - plan->k_before - 1;
        kept = upto(place([&](int i) {
            const Sum e = upto(i);
            return e.bin == plan->k_bin && e.rank == rank;
        })).sum;
    }
    if (set.top_p < 1.0) {
        const double bound = fmax(set.top_p * static_cast<double>(kept), 1.0);
        kept = upto(place([&](int i) { return static_cast<double>(upto(i).sum) >= bound; })).sum;
    }
    if (set.min_p > 0.0) {
        for (int i = tid; i < n; i += kThreads)
            if (power(sc.depth(x_of(i)) - sc.depth(top), powers) >= set.min_p) atomicMax(&likely, upto(i).sum);
        __syncthreads();
        kept = min(kept, likely);
    }
    const double bound = choice_bound(set.u, static_cast<double>(kept));
    const int i = place([&](int j) { return static_cast<double>(upto(j).sum) > bound; });
    if (tid == 0) write(static_cast<int>(static_cast<uint32_t>(list[i])), x_of(i), kept);
}

constexpr int kRowsAtOnce = 1024;   // rows of a set of launches: the workspace's bound

// Parts of a row: about 512 workgroups, of 4096 ids at least.
int parts_of(int rows, int vocab) { return std::max(1, std::min({512 / rows, (vocab + 4095) / 4096, kMaxParts})); }

}  // namespace

namespace ppk {

size_t sample_workspace(int k, int vocab) {
    const int rows = min(k, kRowsAtOnce);
    return rows ? space_bytes(rows, parts_of(rows, vocab)) : 0;
}

void sample(const Sample& all, hipStream_t s) {
    const int most = min(all.k, kRowsAtOnce), parts = parts_of(most, all.vocab), size = (all.vocab + parts - 1) / parts;
    const Space space = space_at(all.ws, most, parts);
    for (int r = 0; r < all.k; r += most) {
        Sample a = all;
        a.k = min(most, all.k - r);
        a.logits += r * a.ldl;
        if (a.temperature) a.temperature += r;
        if (a.top_k) a.top_k += r;
        if (a.top_p) a.top_p += r;
        if (a.min_p) a.min_p += r;
        a.u += r, a.tokens += r;
        if (a.prob) a.prob += r;
        hist_kernel<<<a.k * parts, kThreads, 0, s>>>(a, space, parts, size);
        gather_kernel<<<a.k * parts, kThreads, 0, s>>>(a, space, parts, size);
        pick_kernel<<<a.k, kThreads, 0, s>>>(a, space, parts);
    }
}

}  // namespace ppk
