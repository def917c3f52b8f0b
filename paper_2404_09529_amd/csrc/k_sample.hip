// Sampling: a token of every row of logits with temperature, top-k, top-p and min-p, from a given random
// number.
//
// With the row's ids in order (largest logit first, ties lowest id first) every setting, and the choice itself, asks for
// the first place where a running count or sum passes a bound.  No row is sorted for that.  In powers of two, y =
// x log2(e) / T, the weight 2^y is cut into bins of 1/32 octave below an integer exponent E; sums of weights are integers,
// multiples of 2^(E - 44), the same in whatever order they are formed.  Ids 45 octaves below E are none.
//   hist_kernel    a part of a row: its largest logit, E = ceil of its y, and the sum (and for top-k the count) of
//                  every bin.  E is the part's own: parts differ by whole octaves, that is by shifts, so no pass over the
//                  row has to come before to find its largest logit.  (What a shift takes behind the row's last bin is none; sums are
//                  rounded, half a step a bin.)
//   sum_kernel     the parts' bins together; the bins in which the bounds are passed, or several where one bound depends
//                  on another's exact place.
//   gather_kernel  a part's ids in these bins.
//   pick_kernel    the list in order, running sums behind what the bins before hold, and the places themselves.  A list that is
//                  too long (thousands of nearly equal logits) is resolved by descent through the logit's bits instead.
// A row that fits one workgroup's registers goes all this way in one launch (row_kernel).  Other rows are split into up to 16
// parts, so that a few rows fill the chip: the logits are read twice, the second time from
// the caches.  64 rows of 128,256 logits (33 MB, 6.5 us at a large copy's rate) with settings of their own take 19.1, 10.2, 12.8
// and 16.7 us: about 35 instructions, a third of them float64, and an atomic for each logit, which all workgroups come to together
// behind their loads; the latency of a workgroup; loads, then prefix sums; the order of the longest list (1,325 ids: 2048
// entries through 66 comparisons on one CU; lists of a few ids take 6.4).  One row of 32,000: 5.9, 8.2, 4.4 and 6.7 us, each a
// launch and a chain of loads and barriers.
// (Every row by descent through the bits of its logits, a pass for each of eight bits, as long lists are: 1101 us and 222.)
#include <algorithm>

#include "device.h"
#include "kernels.h"
#include "prepack.h"

namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kUnitBits = 44, kPerOctave = 32;
constexpr int kLive = 45 * 64;                  // 64ths of an octave: weights below 2^-45 are none
constexpr int kBins = kLive / 2;                // of a part, and of the row: what falls behind is none, whatever part it is in
constexpr int kWide = 1024;                     // threads that sum a row's parts
constexpr int kScan = 2 * kWide;                // bins as they hold them, two each
constexpr int kPick = 512;                      // threads that choose
constexpr int kList = 4096, kMaxParts = 16;
static_assert(kScan >= kBins && 2 * kPerOctave == 64, "two bins a thread, two 64ths a bin");
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

// How far an id's y is below the exponent E, in 64ths of an octave: a whole number, and what is left of it (|rest| <= 1/2).
struct Depth {
    int whole;
    double rest;
};
constexpr int kNone = 1 << 30;   // as `whole`: NaN, -inf, or too far below
constexpr double kRound = 0x1.8p52;   // added to a number it leaves the nearest whole one in the low bits

// Rounded wherever E is large: unrounded in a fused operation it would not be E's own y.
__device__ __forceinline__ double y_of(float x, double c) {
#pragma clang fp contract(off)
    const double y = static_cast<double>(x) * c;
    return y;
}
__device__ __forceinline__ double exponent_of(float top, double c) { return top == INFINITY ? INFINITY : ceil(y_of(top, c)); }
// Where one rounding instead of two makes no difference to whole octaves.  Rows beyond go by descent, parts beyond in other
// rows have nothing that may be chosen.
__device__ __forceinline__ bool near(double E) { return fabs(E) < 0x1p30; }

struct Scale {
    double e64, c64;   // 64 E, -64 c with c = log2(e) / T
    __device__ __forceinline__ Scale(double c, double E) : e64(64.0 * E), c64(-64.0 * c) {}
    __device__ __forceinline__ double at(float x) const { return fma(static_cast<double>(x), c64, e64); }
    // (beyond 46 octaves the low bits are not asked for; -inf times 0 is no number, and dropped by the first comparison)
    __device__ __forceinline__ int whole(float x) const {
        const double d = at(x);
        return x > -INFINITY && d < 46.0 * 64.0 ? static_cast<int>(__double_as_longlong(d + kRound)) : kNone;
    }
    __device__ __forceinline__ Depth depth(float x) const {
        const double d = at(x), z = d + kRound;
        return {x > -INFINITY && d < 46.0 * 64.0 ? static_cast<int>(__double_as_longlong(z)) : kNone, d - (z - kRound)};
    }
};
// The same for any E.
struct AnyScale {
    double c, E;
    __device__ __forceinline__ Depth depth(float x) const {
        if (near(E)) return Scale(c, E).depth(x);
        if (E == INFINITY) return {x == INFINITY ? 0 : kNone, 0.0};
        const double d = 64.0 * (E - y_of(x, c)), n = rint(d);
        return {d < 46.0 * 64.0 ? static_cast<int>(n) : kNone, d - n};
    }
};
__device__ __forceinline__ double scale_of(float t) { return 1.4426950408889634 / static_cast<double>(t); }
__device__ __forceinline__ bool live(const Depth& d) { return d.whole < kLive; }
__device__ __forceinline__ int bin_of(const Depth& d) { return d.whole >> 1; }   // of a live id

// 2^-depth as `scaled` times a power of two: a 64th of an octave from the table, the rest, |r| <= ln 2 / 128, by the
// exponential's series to the fifth power (the next term is below 2^-54).
__device__ __forceinline__ double series(const Depth& d, const Powers& p) {
    constexpr double r = -0.69314718055994531 / 64.0;   // the rest times r is the exponent
    double s = fma(d.rest, r * r * r * r * r / 120.0, r * r * r * r / 24.0);
    s = fma(s, d.rest, r * r * r / 6.0);
    s = fma(s, d.rest, r * r / 2.0);
    s = fma(s, d.rest, r);
    const double t = p.at[-d.whole & 63];
    return fma(t, s * d.rest, t);
}
// whole = 64 q - i with 0 <= i < 64: 2^-(whole / 64) = 2^(i / 64) 2^-q
__device__ __forceinline__ int octave_of(const Depth& d) { return (d.whole + 63) >> 6; }
__device__ __forceinline__ double power(const Depth& d, const Powers& p) { return ldexp(series(d, p), -octave_of(d)); }
// 2^(44 - depth) rounded, 0 where there is none: adding 2^52 leaves the whole number in the low bits.
__device__ __forceinline__ u64 weight(const Depth& d, const Powers& p) {
    if (!live(d)) return 0;   // (the exponent below would wrap)
    const double unit = __hiloint2double((1023 + kUnitBits - octave_of(d)) << 20, 0);   // 2^(44 - octave)
    return static_cast<u64>(__double_as_longlong(fma(series(d, p), unit, 0x1p52))) & ((1ull << 52) - 1);
}

// ------------------------------------------------------------------------------- a row's settings and workspace
struct Settings {
    float t;
    int top_k;
    double top_p, min_p, u;   // 1 and more: no limit; 0: no limit; in [0, 1]
    bool greedy, last;        // last: u is 1 or more, the last kept id whatever the sums' last bits
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
    s.last = u >= 1.f;
    return s;
}
// exp((x - top) / T), as min-p asks for it.
__device__ __forceinline__ double share_of(float x, float top, const Settings& s) {
    return x == top ? 1.0 : exp((static_cast<double>(x) - static_cast<double>(top)) / static_cast<double>(s.t));
}
// Bounds in whole steps, which a running sum exceeds at its place: that of the shortest beginning that reaches top_p of `sum`, and
// of the chosen id (the last kept one: where all of the sum is there).  Both factors are at most 1 - 2^-24.
__device__ __forceinline__ u64 share_bound(double top_p, u64 sum) {
    return static_cast<u64>(ceil(fmax(top_p * static_cast<double>(sum), 1.0))) - 1;
}
__device__ __forceinline__ u64 choice_bound(const Settings& s, u64 sum) {
    return s.last ? sum - 1 : static_cast<u64>(s.u * static_cast<double>(sum));
}

struct Part {   // of a row, by hist_kernel
    double E;   // -inf: no id that may be chosen
    float top;
    int id;     // the lowest that has the largest logit; INT32_MAX: every logit is NaN
};
struct Plan {   // of a row, by sum_kernel
    double E;
    float top;
    int k_bin;        // top-k's bin (-1: no limit), and the ids before it
    int k_before;
    int p0, p1, m0, m1, s0, s1;   // first and last bin in which top-p's, min-p's and the choice's place may lie
    u64 all;
    u64 before[kBins];
};
struct Space {
    u64* sum;         // [k][parts][kBins]
    uint32_t* count;  // [k][parts][kBins]
    Part* part;       // [k][parts]
    Plan* plan;       // [k]
    u64* list;        // [k][parts][room]: a part's ids in the bins that matter
    int* listed;      // [k][parts]: how many there are, also those that found no room
};
// Room for a part's ids: a quarter of what pick_kernel takes, or all of it for a row that is one part.
__host__ __device__ constexpr int room_of(int parts) { return parts == 1 ? kList : kList / 4; }

size_t space_bytes(int rows, int parts, size_t room) {   // of `parts` parts in all
    return size_t(rows) * sizeof(Plan) + size_t(parts) * (kBins * 12 + sizeof(Part) + 4) + room * 8;
}
Space space_at(void* ws, int k, int parts) {
    Space s;
    s.plan = static_cast<Plan*>(ws);
    s.sum = reinterpret_cast<u64*>(s.plan + k);
    s.list = s.sum + size_t(k) * parts * kBins;
    s.part = reinterpret_cast<Part*>(s.list + size_t(k) * parts * room_of(parts));
    s.count = reinterpret_cast<uint32_t*>(s.part + size_t(k) * parts);
    s.listed = reinterpret_cast<int*>(s.count + size_t(k) * parts * kBins);
    return s;
}

// U logits of a thread of N, ids v0 + threadIdx.x + i N, all in flight at once; NaN, which is never chosen, from v1 on.
template <int U, int N = kThreads>
__device__ __forceinline__ void read(const float* x, int v0, int v1, float (&y)[U]) {
    const int v = v0 + threadIdx.x;
#pragma unroll
    for (int i = 0; i < U; ++i) y[i] = x[min(v + i * N, v1 - 1)];
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (v + i * N >= v1) y[i] = __uint_as_float(0x7fc00000u);
}
// f(x, id) for these ids, and some NaN.
template <int U, int N = kThreads, typename F>
__device__ __forceinline__ void over(const float* x, int v0, int v1, F f) {
    for (; v0 < v1; v0 += U * N) {
        float y[U];
        read<U, N>(x, v0, v1, y);
#pragma unroll
        for (int i = 0; i < U; ++i) f(y[i], v0 + static_cast<int>(threadIdx.x) + i * N);
    }
}

__device__ __forceinline__ bool above(float t, int i, float u, int j) { return t > u || (t == u && i < j); }

struct Bins {
    u64 sum[kBins];
    uint32_t count[kBins];
    float tops[kWaves];
    int ids[kWaves];
};
// Ids v0 .. v1 - 1 into bins, by kThreads threads.  A part of up to U kThreads ids is read once and stays in `held`.  Barriers
// around the powers and the bins are in here, the last one if there are bins: if E is near.
template <int U>
__device__ __forceinline__ Part part_of(const float* x, int v0, int v1, const Settings& set, Bins& lds, Powers& powers, float (&held)[U]) {
    const int tid = threadIdx.x;
    for (int b = tid; b < kBins; b += kThreads) lds.sum[b] = 0, lds.count[b] = 0;
    powers.fill();
    float top = -INFINITY;
    int id = INT32_MAX;
    const bool once = v1 - v0 <= U * kThreads;
    auto each = [&](auto f) {
        if (once) {
#pragma unroll
            for (int i = 0; i < U; ++i) f(held[i], v0 + tid + i * kThreads);
        } else {
            over<U>(x, v0, v1, f);
        }
    };
    if (once) read(x, v0, v1, held);
    each([&](float y, int v) {
        if (y > top || (y == top && id == INT32_MAX)) top = y, id = v;   // (a thread's ids ascend)
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float t = __shfl_xor(top, o, kWave);
        const int i = __shfl_xor(id, o, kWave);
        if (above(t, i, top, id)) top = t, id = i;
    }
    if (tid % kWave == 0) lds.tops[tid / kWave] = top, lds.ids[tid / kWave] = id;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (above(lds.tops[w], lds.ids[w], top, id)) top = lds.tops[w], id = lds.ids[w];
    const double c = scale_of(set.t);
    const bool none = set.greedy || top == -INFINITY;
    const double E = none ? -INFINITY : exponent_of(top, c);
    if (!near(E)) return {E, top, id};
    const Scale sc(c, E);
    const bool counted = set.top_k > 0;
    each([&](float y, int) {
        const Depth d = sc.depth(y);
        if (!live(d)) return;
        const u64 w = weight(d, powers);
        atomicAdd(&lds.sum[bin_of(d)], w);
        if (counted) atomicAdd(&lds.count[bin_of(d)], 1u);
    });
    __syncthreads();
    return {E, top, id};
}

template <int U>
__global__ __launch_bounds__(kThreads, 4) void hist_kernel(ppk::Sample a, Space s, int parts, int size) {
    __shared__ Bins lds;
    __shared__ Powers powers;
    const int row = blockIdx.x / parts, tid = threadIdx.x, v0 = blockIdx.x % parts * size, v1 = min(v0 + size, a.vocab);
    const Settings set = settings_of(a, row);
    float held[U];
    const Part part = part_of(a.logits + row * a.ldl, v0, v1, set, lds, powers, held);
    if (tid == 0) s.part[blockIdx.x] = part;
    if (!near(part.E)) return;
    const int64_t out = int64_t(blockIdx.x) * kBins;
    for (int b = tid; b < kBins; b += kThreads) {
        s.sum[out + b] = lds.sum[b];
        if (set.top_k > 0) s.count[out + b] = lds.count[b];
    }
}

// ------------------------------------------------------------------------------- scans of a workgroup
template <int W, typename T>
__device__ __forceinline__ T block_scan(T mine, T* waves) {   // up to and including this thread of W wavefronts
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
    for (int i = 0; i < W; ++i)
        if (i < w) mine += waves[i];
    return mine;
}

// The whole row's parts.
struct Whole {
    double E;
    float top;
    int id;
};
__device__ __forceinline__ Whole whole_of(const Part* p, int parts) {   // by every wavefront for itself
    const Part q = p[min(static_cast<int>(threadIdx.x % kMaxParts), parts - 1)];
    Whole w = {q.E, q.top, q.id};
#pragma unroll
    for (int o = kMaxParts / 2; o > 0; o >>= 1) {
        const float t = __shfl_xor(w.top, o, kWave);
        const int i = __shfl_xor(w.id, o, kWave);
        if (above(t, i, w.top, w.id)) w.top = t, w.id = i;
        w.E = fmax(w.E, __shfl_xor(w.E, o, kWave));
    }
    return w;
}
// Octaves from one exponent down to another, both whole numbers.
__device__ __forceinline__ int octaves(double E, double part) { return E == part ? 0 : static_cast<int>(fmin(E - part, 64.0)); }

// A row's bins, for their running sums.
struct Sums {
    u64 sum[kScan + 1];        // of a bin, then of the bins before each
    uint32_t count[kScan + 1];
    u64 wave_sums[kWide / kWave];
    uint32_t wave_counts[kWide / kWave];
    int at[5];
};
// The plan of a row from its bins in `lds`, by N threads; barriers at the beginning and, behind the plan, the caller's.
template <int N>
__device__ __forceinline__ void plan_of(const Settings& set, double E, float top, Sums& lds, Plan* plan) {
    constexpr int PER = kScan / N;   // neighbours that a thread adds up
    const int tid = threadIdx.x;
    if (tid < 5) lds.at[tid] = kBins - 1;
    __syncthreads();
    u64 sum[PER];
    uint32_t count[PER];
    u64 se = 0;
    uint32_t ce = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        sum[i] = se += lds.sum[PER * tid + i];
        count[i] = ce += lds.count[PER * tid + i];
    }
    se = block_scan<N / kWave>(se, lds.wave_sums) - se;
    ce = set.top_k ? block_scan<N / kWave>(ce, lds.wave_counts) - ce : 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) lds.sum[PER * tid + i + 1] = se + sum[i], lds.count[PER * tid + i + 1] = ce + count[i];
    if (tid == 0) lds.sum[0] = 0, lds.count[0] = 0;
    __syncthreads();
    const u64* sums = lds.sum;
    const uint32_t* counts = lds.count;
    const u64 all = sums[kScan];
    // at[slot]: the bin in which the sum (or count) passes the bound; a barrier follows
    auto passing = [&](int slot, auto before, auto bound) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int b = PER * tid + i;
            if (!bound(before[b]) && bound(before[b + 1])) lds.at[slot] = b;   // one thread
        }
    };
    u64 lo = all, hi = all;   // of what is kept
    int bk = -1;
    if (set.top_k > 0 && static_cast<uint32_t>(set.top_k) < counts[kScan]) {
        passing(0, counts, [&](uint32_t n) { return n >= static_cast<uint32_t>(set.top_k); });
        __syncthreads();
        bk = lds.at[0];
        lo = sums[bk], hi = sums[bk + 1];
    }
    int p0 = 0, p1 = -1, m0 = 0, m1 = -1;
    if (set.top_p < 1.0) {
        const u64 t0 = share_bound(set.top_p, lo), t1 = share_bound(set.top_p, hi);
        passing(1, sums, [&](u64 n) { return n > t0; });
        passing(2, sums, [&](u64 n) { return n > t1; });
        __syncthreads();
        p0 = lds.at[1], p1 = lds.at[2];
        lo = min(lo, sums[p0]), hi = min(hi, sums[p1 + 1]);
    }
    if (set.min_p > 0.0) {
        // 2^-depth = min_p 2^-depth(top), one bin more on both sides
        const double d = Scale(scale_of(set.t), E).at(top) / 64.0 - log2(set.min_p);
        const int b = static_cast<int>(fmin(d, 46.0) * kPerOctave);
        m0 = min(max(b - 1, 0), kBins - 1), m1 = min(b + 1, kBins - 1);
        lo = min(lo, sums[m0]), hi = min(hi, sums[m1 + 1]);
    }
    const u64 u0 = choice_bound(set, max(lo, u64(1))), u1 = choice_bound(set, hi);
    passing(3, sums, [&](u64 n) { return n > u0; });
    passing(4, sums, [&](u64 n) { return n > u1; });
    __syncthreads();
    for (int b = tid; b < kBins; b += N) plan->before[b] = sums[b];
    if (tid == 0) {
        plan->k_bin = bk, plan->k_before = bk >= 0 ? static_cast<int>(counts[bk]) : 0;
        plan->p0 = p0, plan->p1 = p1, plan->m0 = m0, plan->m1 = m1, plan->s0 = lds.at[3], plan->s1 = lds.at[4];
        plan->all = all;
    }
}

__global__ __launch_bounds__(kWide) void sum_kernel(ppk::Sample a, Space s, int parts) {
    __shared__ Sums lds;
    __shared__ int shifts[kMaxParts];
    const int row = blockIdx.x, tid = threadIdx.x;
    const Settings set = settings_of(a, row);
    const Part* ps = s.part + int64_t(row) * parts;
    const Whole w = whole_of(ps, parts);
    Plan* plan = s.plan + row;
    if (tid == 0) plan->E = w.E, plan->top = w.top;
    if (set.greedy || !near(w.E)) return;
    if (tid < kMaxParts) shifts[tid] = tid < parts && near(ps[tid].E) ? octaves(w.E, ps[tid].E) : 64;
    __syncthreads();
    // the bins of all parts, eight parts in one wait for memory (without branches: a part too many is the last one again)
    u64 t[2] = {0, 0};
    uint32_t n[2] = {0, 0};
    for (int p0 = 0; p0 < parts; p0 += 8) {
        const int64_t src = int64_t(row) * parts * kBins;
        u64 x[2][8];
        uint32_t c[2][8];
        auto from = [&](int i, int p) { return tid + i * kWide - kPerOctave * shifts[p0 + p]; };
        auto at_of = [&](int i, int p) { return src + min(p0 + p, parts - 1) * kBins + min(max(from(i, p), 0), kBins - 1); };
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int p = 0; p < 8; ++p) x[i][p] = s.sum[at_of(i, p)], c[i][p] = 0;
        if (set.top_k) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int p = 0; p < 8; ++p) c[i][p] = s.count[at_of(i, p)];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                // (a part without anything, 64 octaves down, has written no bins; a part's last bins may lie behind the row's)
                const bool has = from(i, p) >= 0 && from(i, p) < kBins && tid + i * kWide < kBins;
                const int down = shifts[p0 + p] & 63;   // to the nearest: a bin with an id in it is not 0
                t[i] += has ? (x[i][p] + ((1ull << down) >> 1)) >> down : 0;
                n[i] += has ? c[i][p] : 0;
            }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) lds.sum[tid + i * kWide] = t[i], lds.count[tid + i * kWide] = n[i];
    plan_of<kWide>(set, w.E, w.top, lds, plan);
}

// The bins whose ids matter.
struct Wanted {
    int bk, p0, p1, m0, m1, s0, s1;
    __device__ __forceinline__ explicit Wanted(const Plan* p)
        : bk(p->k_bin), p0(p->p0), p1(p->p1), m0(p->m0), m1(p->m1), s0(p->s0), s1(p->s1) {}
    __device__ __forceinline__ bool has(int b) const {
        return b == bk || (b >= p0 && b <= p1) || (b >= m0 && b <= m1) || (b >= s0 && b <= s1);
    }
};
// A thread's hits of U ids as bits, the wavefront's in one reservation of the list's room.
template <int U>
__device__ __forceinline__ void gather(const float (&y)[U], int first, const Scale& sc, int shift, const Wanted& bins,
                                       u64* list, int room, int& listed) {
    const int lane = threadIdx.x % kWave;
    std::conditional_t<(U > 32), u64, uint32_t> hits = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int whole = sc.whole(y[i]);
        hits |= decltype(hits)(whole < kLive && bins.has((whole >> 1) + shift)) << i;
    }
    int n = U > 32 ? __popcll(hits) : __popc(hits), end = n;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int up = __shfl_up(end, o, kWave);
        if (lane >= o) end += up;
    }
    int base = 0;
    if (lane == kWave - 1 && end) base = atomicAdd(&listed, end);
    int to = __shfl(base, kWave - 1, kWave) + end - n;
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (hits >> i & 1) {
            if (to < room) list[to] = u64(~key_of(y[i])) << 32 | static_cast<uint32_t>(first + i * kThreads);
            ++to;
        }
}

template <int U>
__global__ __launch_bounds__(kThreads, 4) void gather_kernel(ppk::Sample a, Space s, int parts, int size) {
    __shared__ int listed;
    const int row = blockIdx.x / parts, tid = threadIdx.x, v0 = blockIdx.x % parts * size, v1 = min(v0 + size, a.vocab);
    const float* x = a.logits + row * a.ldl;
    float held[U];
    read(x, v0, v1, held);
    const float t = a.temperature ? a.temperature[row] : 1.f;
    const Plan* plan = s.plan + row;
    const double E = plan->E, part_E = s.part[blockIdx.x].E;
    const Wanted bins(plan);
    if (!(t > 0.f)) return;   // (greedy: of the plan nothing is there but E)
    if (!near(E)) {
        if (tid == 0) s.listed[blockIdx.x] = kList + 1;
        return;
    }
    if (tid == 0) listed = 0;
    __syncthreads();
    const int room = room_of(parts);
    u64* list = s.list + int64_t(blockIdx.x) * room;
    if (near(part_E)) {
        const Scale sc(scale_of(t), part_E);
        const int shift = octaves(E, part_E) * kPerOctave;
        for (int v = v0;;) {
            gather(held, v + tid, sc, shift, bins, list, room, listed);
            if ((v += U * kThreads) >= v1) break;
            read(x, v, v1, held);
        }
    }
    __syncthreads();
    if (tid == 0) s.listed[blockIdx.x] = listed;
}

// ------------------------------------------------------------------------------- descent
// Where the list is too long: eight bits of the logit at a time, a histogram of counts and sums, the bin in which the
// bound is passed, then the next eight bits of that bin's ids; equal logits have equal weights, and the id among them is
// counted off.
enum Bound { kCount, kSum };   // what is to exceed the bound
__device__ __forceinline__ bool passes(Bound b, u64 sum, uint32_t count, u64 bound) { return (b == kCount ? count : sum) > bound; }

struct Place {
    int id;
    u64 sum;      // of the ids up to this one
    uint32_t n;   // and how many they are
    float x;
};
struct Descent {
    u64 sum[256];
    uint32_t count[256];
    u64 wave_sum[kPick / kWave];
    uint32_t wave_count[kPick / kWave];
    int digit, found;
    u64 above_sum;
    uint32_t above_count;
};

// The first place, in order, where the running count or sum passes the bound; there is one.
__device__ Place find(const float* x, int vocab, const AnyScale& sc, const Powers& powers, Bound what, u64 bound, Descent& lds) {
    const int tid = threadIdx.x, lane = tid % kWave;
    uint32_t prefix = 0, mask = 0, above_n = 0, equal = 0;   // the last digit's ids: equal logits
    u64 above_s = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) lds.sum[tid] = 0, lds.count[tid] = 0;
        __syncthreads();
        over<4, kPick>(x, 0, vocab, [&](float y, int) {
            const uint32_t k = key_of(y);
            if ((k & mask) != prefix) return;
            const Depth d = sc.depth(y);
            if (!live(d)) return;
            atomicAdd(&lds.sum[(k >> shift) & 255], weight(d, powers));
            atomicAdd(&lds.count[(k >> shift) & 255], 1u);
        });
        __syncthreads();
        const u64 s = tid < 256 ? lds.sum[255 - tid] : 0;   // digits from 255 down
        const uint32_t n = tid < 256 ? lds.count[255 - tid] : 0;
        const u64 es = above_s + block_scan<kPick / kWave>(s, lds.wave_sum);
        const uint32_t en = above_n + block_scan<kPick / kWave>(n, lds.wave_count);
        if (tid < 256 && !passes(what, es - s, en - n, bound) && passes(what, es, en, bound))
            lds.digit = 255 - tid, lds.above_sum = es - s, lds.above_count = en - n;
        __syncthreads();
        above_s = lds.above_sum, above_n = lds.above_count, equal = lds.count[lds.digit];
        prefix |= static_cast<uint32_t>(lds.digit) << shift;
        mask |= 255u << shift;
    }
    const float v = of_key(prefix);
    const u64 w = weight(sc.depth(v), powers);
    uint32_t lo = 1, hi = equal;   // the number of them that passes (the sum of more than there are may pass 64 bits)
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (passes(what, above_s + w * mid, above_n + mid, bound)) hi = mid;
        else lo = mid + 1;
    }
    uint32_t before = 0;
    for (int v0 = 0; v0 < vocab; v0 += kPick) {
        const bool is = v0 + tid < vocab && x[v0 + tid] == v;
        const u64 here = __ballot(is);
        __syncthreads();
        if (lane == 0) lds.wave_count[tid / kWave] = __popcll(here);
        __syncthreads();
        uint32_t mine = before, all = 0;
        for (int i = 0; i < (kPick / kWave); ++i) {
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
    return {id, above_s + w * lo, above_n + lo, v};
}

__device__ Place descend(const float* x, int vocab, const Settings& set, const AnyScale& sc, float top, const Powers& powers,
                         Descent& lds) {
    u64 all = 0, likely = 0;
    uint32_t count = 0, likely_n = 0;
    over<4, kPick>(x, 0, vocab, [&](float y, int) {
        const Depth d = sc.depth(y);
        if (!live(d)) return;
        const u64 w = weight(d, powers);
        all += w, ++count;
        if (share_of(y, top, set) >= set.min_p) likely += w, ++likely_n;
    });
    auto total = [&](auto v, auto* waves) {
        v = block_scan<kPick / kWave>(v, waves);
        __syncthreads();
        if (threadIdx.x == kPick - 1) waves[0] = v;
        __syncthreads();
        v = waves[0];
        __syncthreads();
        return v;
    };
    u64 kept = total(all, lds.wave_sum);
    likely = total(likely, lds.wave_sum);
    count = total(count, lds.wave_count);
    likely_n = total(likely_n, lds.wave_count);
    auto keep = [&](const Place& p) { kept = p.sum, count = p.n; };
    if (set.top_k && static_cast<uint32_t>(set.top_k) < count) keep(find(x, vocab, sc, powers, kCount, set.top_k - 1, lds));
    if (set.top_p < 1.0) keep(find(x, vocab, sc, powers, kSum, share_bound(set.top_p, kept), lds));
    kept = min(kept, likely), count = min(count, likely_n);
    Place p = set.last ? find(x, vocab, sc, powers, kCount, count - 1, lds) : find(x, vocab, sc, powers, kSum, choice_bound(set, kept), lds);
    p.sum = kept;
    return p;
}

// ------------------------------------------------------------------------------- the choice
// An id in a list: ~key, id; in the order of these the likeliest comes first.
__device__ __forceinline__ float logit_of(u64 entry) { return of_key(~static_cast<uint32_t>(entry >> 32)); }
__device__ __forceinline__ u64 better_of(u64 x, u64 y, bool least) { return (x < y) == least ? x : y; }
// Lane i ^ S's x, without LDS, which such exchanges of eight wavefronts would keep busy.
template <int S>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
    const int i = static_cast<int>(x);
    if constexpr (S == 1) {
        return __builtin_amdgcn_update_dpp(0, i, 0xb1, 0xf, 0xf, true);
    } else if constexpr (S == 2) {
        return __builtin_amdgcn_update_dpp(0, i, 0x4e, 0xf, 0xf, true);
    } else if constexpr (S == 4) {   // from four lanes up, then in every other group of four from four lanes down
        const int up = __builtin_amdgcn_update_dpp(0, i, 0x104, 0xf, 0x5, false);
        return __builtin_amdgcn_update_dpp(up, i, 0x114, 0xf, 0xa, false);
    } else if constexpr (S == 8) {
        return __builtin_amdgcn_update_dpp(0, i, 0x128, 0xf, 0xf, true);
    } else if constexpr (S == 16) {
        const auto both = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return threadIdx.x & 16 ? both[0] : both[1];
    } else {
        const auto both = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & 32 ? both[0] : both[1];
    }
}
template <int S>
__device__ __forceinline__ u64 lane_xor(u64 x) {
    return u64(lane_xor<S>(static_cast<uint32_t>(x >> 32))) << 32 | lane_xor<S>(static_cast<uint32_t>(x));
}
// The last steps of a bitonic merge, partners S, S / 2 .. 1 lanes apart.
template <int S>
__device__ __forceinline__ u64 merge_lanes(u64 x, bool up) {
    x = better_of(x, lane_xor<S>(x), ((threadIdx.x & S) == 0) == up);
    if constexpr (S > 1) return merge_lanes<S / 2>(x, up);
    return x;
}
// A wavefront's 64 entries in order, ascending where bit 6 of their number is 0.
template <int SIZE = 2>
__device__ __forceinline__ u64 sort_lanes(u64 x, int i) {
    x = merge_lanes<SIZE / 2>(x, (i & SIZE) == 0);
    if constexpr (SIZE < kWave) return sort_lanes<2 * SIZE>(x, i);
    return x;
}

struct List {
    u64 entry[kList];    // what of the order stands in the id's stead: ~key, id
    u64 run[kList];      // running sums
    uint16_t bins[kList], start[kBins];
    u64 waves[kPick / kWave];
    int first[4];
    u64 likely;
};
// The place among the n > 0 entries of a list, in any order, by kPick threads; a barrier is behind the entries.
template <typename F>
__device__ __forceinline__ void choose(int n, const Settings& set, const AnyScale& sc, float top, const Powers& powers, const Plan* plan, List& lds, F write) {
    const int tid = threadIdx.x;
    u64 *list = lds.entry, *run = lds.run, *waves = lds.waves;
    uint16_t *bins = lds.bins, *start = lds.start;
    int* first = lds.first;
    u64& likely = lds.likely;
    // Bitonic sort of the next power of two in registers, entry tid + kPick j in register j: partners less than 64 apart are
    // lanes, others less than kPick apart come through LDS.
    constexpr int kHeld = kList / kPick;
    int m = kWave;
    while (m < n) m *= 2;
    const int held = (m + kPick - 1) / kPick;
    const bool takes_part = tid / kWave * kWave < m;
    u64 v[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) v[j] = tid + j * kPick < n ? list[tid + j * kPick] : ~0ull;
    if (takes_part) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
            if (j < held) v[j] = sort_lanes(v[j], tid + j * kPick);
    }
    for (int size = 2 * kWave; size <= m; size *= 2) {
        for (int stride = size / 2; stride >= kWave; stride /= 2) {
            if (stride >= kPick) {
#pragma unroll
                for (int s2 = 1; s2 < kHeld; s2 *= 2)
                    if (stride == s2 * kPick) {
#pragma unroll
                        for (int j = 0; j < kHeld; ++j)
                            if (!(j & s2) && j + s2 < kHeld) {
                                const u64 x = v[j], y = v[j + s2];
                                const bool up = ((tid + j * kPick) & size) == 0;
                                v[j] = (x < y) == up ? x : y, v[j + s2] = (x < y) == up ? y : x;
                            }
                    }
                continue;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                if (tid + j * kPick < m) list[tid + j * kPick] = v[j];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                const int i = tid + j * kPick;
                if (i < m) v[j] = better_of(v[j], list[i ^ stride], ((i & stride) == 0) == ((i & size) == 0));
            }
        }
        if (takes_part) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                if (j < held) v[j] = merge_lanes<kWave / 2>(v[j], ((tid + j * kPick) & size) == 0);
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
        if (tid + j * kPick < m) list[tid + j * kPick] = v[j];
    __syncthreads();
    // Sums of the entries up to each, in order; from here on a thread's are neighbours, entry base + j.
    const int base = tid * held;
    int bin[kHeld];
    u64 total[kHeld], before[kHeld], mine = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        bin[j] = kBins;
        if (j >= held) continue;
        const int i = base + j;
        const bool is = i < n;
        v[j] = is ? list[i] : ~0ull;
        const Depth d = sc.depth(logit_of(v[j]));
        bin[j] = is ? min(bin_of(d), kBins - 1) : kBins;
        before[j] = is ? plan->before[bin[j]] : 0;
        if (is) mine += weight(d, powers), bins[i] = static_cast<uint16_t>(bin[j]);
        total[j] = mine;
    }
    const u64 up = block_scan<kPick / kWave>(mine, waves) - mine;
    if (tid < 4) first[tid] = tid < 3 ? n - 1 : n;
    if (tid == 0) likely = plan->before[plan->m0];
#pragma unroll
    for (int j = 0; j < kHeld; ++j)   // (the scan's barriers are behind `bins`)
        if (bin[j] < kBins) {
            run[base + j] = total[j] += up;
            if (base + j == 0 || bins[base + j - 1] != bin[j]) start[bin[j]] = static_cast<uint16_t>(base + j);
        }
    __syncthreads();
    // Of all ids up to each: the bins before its own, and the list's entries of its bin.  `rank`: among these.
    int rank[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        if (j >= held) continue;
        const int lo = bin[j] < kBins ? start[bin[j]] : 0;
        rank[j] = base + j - lo;
        total[j] += before[j] - (lo ? run[lo - 1] : 0);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
        if (bin[j] < kBins) run[base + j] = total[j];
    // The first entry that passes; the last one if a sum of parts and one of ids differ in their last bits just here.
    auto place = [&](int slot, auto passes) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            if (j >= held) break;
            const u64 here = __ballot(bin[j] < kBins && passes(total[j], bin[j], rank[j]));
            if (here && tid % kWave == 0) atomicMin(&first[slot], base + j + __builtin_ctzll(here) * held);
        }
        __syncthreads();
        return first[slot];
    };
    u64 kept = plan->all;
    int end = n - 1;   // the last kept entry
    if (plan->k_bin >= 0) {
        const int last = set.top_k - plan->k_before - 1, of = plan->k_bin;
        kept = run[end = place(0, [&](u64, int b, int r) { return b == of && r == last; })];
    }
    if (set.top_p < 1.0) {
        const u64 bound = share_bound(set.top_p, kept);
        kept = run[end = place(1, [&](u64 sum, int, int) { return sum > bound; })];
    }
    if (set.min_p > 0.0) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
            if (bin[j] < kBins && bin[j] >= plan->m0) {
                if (bin[j] <= plan->m1 && share_of(logit_of(v[j]), top, set) >= set.min_p) atomicMax(&likely, total[j]);
                else atomicMin(&first[3], base + j);
            }
        __syncthreads();
        kept = min(kept, likely), end = min(end, max(first[3] - 1, 0));
    }
    const u64 bound = choice_bound(set, kept);
    const int i = set.last ? end : place(2, [&](u64 sum, int, int) { return sum > bound; });
    if (tid == 0) write(static_cast<int>(static_cast<uint32_t>(list[i])), logit_of(list[i]), kept);
}

// What a row's choice writes.
struct Out {
    const ppk::Sample& a;
    int row;
    __device__ __forceinline__ void none() const {
        if (threadIdx.x) return;
        a.tokens[row] = -1;
        if (a.prob) a.prob[row] = 0.f;
    }
    __device__ __forceinline__ void greedy(int id) const {
        if (threadIdx.x) return;
        a.tokens[row] = id;
        if (a.prob) a.prob[row] = 1.f;
    }
    __device__ __forceinline__ void operator()(int id, double weight, u64 kept) const {   // by one thread
        a.tokens[row] = id;
        if (a.prob) a.prob[row] = static_cast<float>(weight * (static_cast<double>(1ull << kUnitBits) / static_cast<double>(kept)));
    }
};

__global__ __launch_bounds__(kPick) void pick_kernel(ppk::Sample a, Space s, int parts) {
    __shared__ union {
        Descent descent;
        List list;
    } lds;
    __shared__ Powers powers;
    __shared__ int starts[kMaxParts + 1];
    const int row = blockIdx.x, tid = threadIdx.x;
    const Settings set = settings_of(a, row);
    const Out out = {a, row};
    const Whole w = whole_of(s.part + int64_t(row) * parts, parts);
    if (set.greedy && w.id != INT32_MAX) return out.greedy(w.id);
    if (w.E == -INFINITY) return out.none();
    powers.fill();
    const Plan* plan = s.plan + row;
    const AnyScale sc = {scale_of(set.t), plan->E};
    const float top = plan->top;
    // the parts' lists, one behind the other
    if (tid < kWave) {
        const int c = tid < parts ? s.listed[int64_t(row) * parts + tid] : 0;
        int end = c > room_of(parts) ? kList + 1 : c;   // (sixteen of these stay small)
#pragma unroll
        for (int o = 1; o < kMaxParts; o <<= 1) {
            const int up = __shfl_up(end, o, kWave);
            if (tid >= o) end += up;
        }
        if (tid < kMaxParts) starts[tid + 1] = end;
        if (tid == 0) starts[0] = 0;
    }
    __syncthreads();
    const int n = starts[parts];
    auto write = [&](int id, float x, u64 kept) { out(id, power(sc.depth(x), powers), kept); };
    if (n > kList || n == 0) {
        __syncthreads();
        const Place p = descend(a.logits + row * a.ldl, a.vocab, set, sc, top, powers, lds.descent);
        if (tid == 0) write(p.id, p.x, p.sum);
        return;
    }
    for (int p = tid / kWave; p < parts; p += kPick / kWave)   // a wavefront copies a part's
        for (int i = starts[p] + tid % kWave; i < starts[p + 1]; i += kWave)
            lds.list.entry[i] = s.list[(int64_t(row) * parts + p) * room_of(parts) + i - starts[p]];
    __syncthreads();
    choose(n, set, sc, top, powers, plan, lds.list, write);
}

// A row that one workgroup reads at once, from the logits to the token.  512 threads, two wavefronts a SIMD: with 64 logits held
// a thread has 253 registers.
template <int U>
__global__ __launch_bounds__(kThreads) void row_kernel(ppk::Sample a) {
    static_assert(kThreads == kPick, "the same threads to the end");
    __shared__ union {
        struct {
            Bins bins;
            Sums sums;
        } first;
        Descent descent;
        List list;
    } lds;
    __shared__ Powers powers;
    __shared__ Plan plan;
    __shared__ int listed;
    const int row = blockIdx.x, tid = threadIdx.x;
    const float* x = a.logits + row * a.ldl;
    const Settings set = settings_of(a, row);
    const Out out = {a, row};
    float held[U];
    if (tid == 0) listed = 0;
    const Part part = part_of(x, 0, a.vocab, set, lds.first.bins, powers, held);
    if (set.greedy && part.id != INT32_MAX) return out.greedy(part.id);
    if (part.E == -INFINITY) return out.none();
    const AnyScale sc = {scale_of(set.t), part.E};
    auto write = [&](int id, float y, u64 kept) { out(id, power(sc.depth(y), powers), kept); };
    auto by_descent = [&] {
        __syncthreads();
        const Place p = descend(x, a.vocab, set, sc, part.top, powers, lds.descent);
        if (tid == 0) write(p.id, p.x, p.sum);
    };
    if (!near(part.E)) return by_descent();
    for (int b = tid; b < kScan; b += kThreads) {
        lds.first.sums.sum[b] = b < kBins ? lds.first.bins.sum[b] : 0;
        lds.first.sums.count[b] = b < kBins ? lds.first.bins.count[b] : 0;
    }
    plan_of<kThreads>(set, part.E, part.top, lds.first.sums, &plan);
    __syncthreads();
    gather(held, tid, Scale(scale_of(set.t), part.E), 0, Wanted(&plan), lds.list.entry, kList, listed);
    __syncthreads();
    if (U * kThreads > kList && listed > kList) return by_descent();
    choose(listed, set, sc, part.top, powers, &plan, lds.list, write);
}

constexpr int kRowsAtOnce = 1024;   // rows of a set of launches: the workspace's bound

// Parts of a row: about 512 workgroups, of 4096 ids at least.
int parts_of(int rows, int vocab) { return std::max(1, std::min({512 / rows, (vocab + 4095) / 4096, kMaxParts})); }

// Logits that each thread of a row's one workgroup holds, or 0: rows in parts.  In us, four launches and one: one row of 1000
// logits 22 and 12, of 4096 23 and 13, of 8192 24 and 17, of 16,384 24.6 and 23.2, of 32,000 25 and 36; 64 rows 26 and 14, 26 and
// 15, 28 and 18, 28 and 25, 31 and 39; 128 rows of 20,000 and 32,000 43 and 35, 45 and 41; 256 46 and 34, 51 and 42.
int whole_row(int k, int vocab) {
    return vocab <= 8 * kThreads ? 8 : vocab <= 16 * kThreads ? 16 : vocab <= 32 * kThreads ? 32 : vocab <= 64 * kThreads && k >= 128 ? 64 : 0;
}

}  // namespace

namespace ppk {

// (Not less for more rows, so that the largest batch's serves all.)
size_t sample_workspace(int k, int vocab) {
    if (whole_row(1, vocab) || !k) return 0;
    const int rows = min(k, kRowsAtOnce), most = max(min(rows * parts_of(1, vocab), 512), rows);
    return space_bytes(rows, most, rows > 256 ? size_t(rows) * room_of(1) : size_t(most) * room_of(2));
}

void sample(const Sample& all, hipStream_t s) {
    switch (whole_row(all.k, all.vocab)) {
        case 8: row_kernel<8><<<all.k, kThreads, 0, s>>>(all); return;
        case 16: row_kernel<16><<<all.k, kThreads, 0, s>>>(all); return;
        case 32: row_kernel<32><<<all.k, kThreads, 0, s>>>(all); return;
        case 64: row_kernel<64><<<all.k, kThreads, 0, s>>>(all); return;
    }
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
        // (logits that a thread holds; parts of 8016 ids with 32 rather than 16: one row of 128,256 37 us rather than 34)
        auto go = [&](auto held) {
            constexpr int U = decltype(held)::value;
            hist_kernel<U><<<a.k * parts, kThreads, 0, s>>>(a, space, parts, size);
            sum_kernel<<<a.k, kWide, 0, s>>>(a, space, parts);
            gather_kernel<U><<<a.k * parts, kThreads, 0, s>>>(a, space, parts, size);
        };
        if (size <= 8 * kThreads) go(std::integral_constant<int, 8>{});
        else if (size <= 16 * kThreads) go(std::integral_constant<int, 16>{});
        else go(std::integral_constant<int, 32>{});
        pick_kernel<<<a.k, kPick, 0, s>>>(a, space, parts);
    }
}

}  // namespace ppk
