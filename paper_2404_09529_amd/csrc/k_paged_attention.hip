// Attention of one query row per sequence over a paged cache: out = softmax(q k^T / sqrt(D)) v over the
// first lens[i] keys of sequence i, in whatever pages they lie.
//
// Every key and value is read once and used for the G = H / Hkv query heads that share it, so reading them bounds
// the kernel.  The sequences are cut into units of whole 128-key tiles (paged.h); a workgroup has one unit of one
// key/value head, its four wavefronts 32 keys of each tile, each with a softmax of its own (running maximum and
// sum), joined through LDS at the end.  A sequence of one unit is written right away, the units of a longer one leave
// (o, maximum, sum) for join_kernel.
//
// Nothing passes through LDS on the way: keys go from memory into the registers that the 16 x 16 matrix
// instructions take them from.  S^T = K Q^T puts key 8 g + 4 t + r of a wavefront's 32 into row 4 g + r of score tile t,
// so that lane group g (16 lanes) holds the scores of keys 8 g .. 8 g + 7, which is what it has to hold as the operand of
// O^T = V^T P^T; a lane reads the same 16 (or 8, or 4) columns' part of those 8 rows of V, whole rows per 16 lanes.
// The query heads are the instructions' columns; with fewer than 16 the rest are zeros (the matrix cores are idle
// otherwise: a 32-key step of 16 KB takes them 256 cycles of the 6500 that a SIMD's share of the memory needs).
//
// bf16 operands hold what is exact in them: bf16 keys, values and queries, and 8-bit codes, whose scales multiply scores
// and probabilities.  Probabilities (times a value's scale) are two bf16 terms, off by 2^-17, so that the result is as good
// as its one rounding; with float32 queries over 8-bit pages queries and probabilities are three terms, all of float32's bits.
// float32 pages take the float32 matrix instructions.
#include <float.h>

#include <utility>

#include "device.h"
#include "kernels.h"
#include "paged.h"
#include "prepack.h"

namespace {

constexpr int kBlock = 256, kSplitWaves = kBlock / kWave;
constexpr int kStep = 32;   // keys of a wavefront per tile
constexpr int kRows = 16;   // query heads of a workgroup
static_assert(kSplitWaves * kStep == ppk::kPagedTile, "a tile is one step of a workgroup");

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// f(0) .. f(N - 1) with constants for arguments.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
    each_of(f, std::make_integer_sequence<int, N>{});
}

// Lane E's value of every row of 16 lanes.
template <int E>
__device__ __forceinline__ int row_lane(int x) {
    return __builtin_amdgcn_update_dpp(0, x, 0x150 + E, 0xf, 0xf, true);
}
template <int E>
__device__ __forceinline__ float row_lane(float x) {
    return __int_as_float(row_lane<E>(__float_as_int(x)));
}

// Over the four lanes that are 16 apart.
__device__ __forceinline__ float max16(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum16(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// x as N bf16 terms, the largest first.
template <int N>
__device__ __forceinline__ void terms(float x, bf16 (&t)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        t[i] = static_cast<bf16>(x);
        x -= static_cast<float>(t[i]);
    }
}

// Bits of the float32 form of byte B of w, a signed number: one instruction, which takes the byte where it lies.
template <int B>
__device__ __forceinline__ uint32_t byte_value(uint32_t w) {
    uint32_t f;
    if constexpr (B == 0)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(w));
    else if constexpr (B == 1)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(w));
    else if constexpr (B == 2)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(w));
    else
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(w));
    return f;
}

// ------------------------------------------------------------------------------- the split
struct Unit {
    int seq, len, tile0, tile1, units;   // seq < 0: none
};

// Sum over the lanes up to and including this one.
__device__ __forceinline__ int scan_up(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // 1, 2, 4 and 8 lanes up in rows of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row 0's sum to row 1, row 2's to row 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // the first two rows' to the others
    return x;
}
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(scan_up(x), kWave - 1); }

struct Split {
    const int32_t* lens;
    int k, span, target, least;
    __device__ __forceinline__ int len(int i) const { return i < k ? ppk::paged_len(lens[i], span) : 0; }
    // Tiles of a unit, by a wavefront; first: this lane's len(lane).
    __device__ __forceinline__ int unit(int first) const {
        int64_t all = ppk::paged_tiles(first);
        for (int i = (threadIdx.x & 63) + kWave; i < k; i += kWave) all += ppk::paged_tiles(len(i));
        // at most 2^24 tiles a sequence and 2^16 sequences a lane: two sums of 32 bits
        const int64_t lo = wave_total(static_cast<int>(all & 0xffffff)), hi = wave_total(static_cast<int>(all >> 24));
        return ppk::paged_unit((hi << 24) + lo, target, least);
    }
};

// Unit u, by every wavefront for itself.
__device__ __forceinline__ Unit find_unit(const Split& s, int u) {
    const int lane = threadIdx.x & 63;
    int len = s.len(lane);
    const int unit = s.unit(len);
    int base = 0;
    for (int i0 = 0; i0 < s.k; i0 += kWave) {
        if (i0) len = s.len(i0 + lane);
        const int t = ppk::paged_tiles(len), n = i0 + lane < s.k ? ppk::paged_units(t, unit) : 0, end = base + scan_up(n);
        const uint64_t here = __ballot(u < end && u >= end - n);
        if (here) {
            const int l = __builtin_ctzll(here);
            const int first = u - __builtin_amdgcn_readlane(end - n, l), tiles = __builtin_amdgcn_readlane(t, l);
            return {i0 + l, __builtin_amdgcn_readlane(len, l), first * unit, min(first * unit + unit, tiles),
                    __builtin_amdgcn_readlane(n, l)};
        }
        base = __builtin_amdgcn_readlane(end, kWave - 1);
    }
    return {-1, 0, 0, 0, 0};
}

// The first unit of sequence i, and how many it has.
__device__ __forceinline__ int2 units_of(const Split& s, int i) {
    const int lane = threadIdx.x & 63;
    int len = s.len(lane);
    const int unit = s.unit(len);
    int base = 0;
    for (int i0 = 0;; i0 += kWave) {
        if (i0) len = s.len(i0 + lane);
        const int n = i0 + lane < s.k ? ppk::paged_units(ppk::paged_tiles(len), unit) : 0, end = base + scan_up(n);
        if (i < i0 + kWave)
            return make_int2(__builtin_amdgcn_readlane(end - n, i - i0), __builtin_amdgcn_readlane(n, i - i0));
        base = __builtin_amdgcn_readlane(end, kWave - 1);
    }
}

// ------------------------------------------------------------------------------- operands by type
// A wavefront's 32 rows of K and V in registers, and the products with them.  Lane (g, ln) = (lane / 16, lane % 16).
// kcol, vcol: byte offsets of this lane's part of a row of K and V.
template <int D, typename T, typename P>
struct Tile;

// bf16 pages.  K operand of instruction (t, s): dims 32 s + 8 g .. + 7 of key 8 (ln / 4) + 4 t + ln % 4.  V: dims
// 8 ln .. + 7 of the lane group's keys; instruction j takes dim 8 ln + j of all of them.
template <int D>
struct Tile<D, bf16, bf16> {
    static constexpr int KS = D / 32, NJ = D / 16;
    static_assert(D == 128, "a lane's part of a row is 16 bytes");
    u32x4 k[2][KS], v[8];
    struct Query {
        bf16x8 f[KS];
    };

    static __device__ __forceinline__ int kcol(int g) { return 16 * g; }
    static __device__ __forceinline__ int vcol(int ln) { return 16 * ln; }
    static __device__ __forceinline__ int dim(int j, int row) { return 8 * row + j; }
    static __device__ __forceinline__ void query(Query& q, const bf16* x, int g) {
#pragma unroll
        for (int s = 0; s < KS; ++s) q.f[s] = x ? *reinterpret_cast<const bf16x8*>(x + 32 * s + 8 * g) : bf16x8{};
    }
    __device__ __forceinline__ void load_k(int t, const char* p) {
#pragma unroll
        for (int s = 0; s < KS; ++s) k[t][s] = *reinterpret_cast<const u32x4*>(p + 64 * s);
    }
    __device__ __forceinline__ void load_v(int e, const char* p) { v[e] = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ void clear_v(int e) { v[e] = u32x4{}; }
    __device__ __forceinline__ f32x4 scores(int t, const Query& q) const {
        f32x4 s = {};
#pragma unroll
        for (int i = 0; i < KS; ++i)
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][i]), q.f[i], s, 0, 0, 0);
        return s;
    }
    __device__ __forceinline__ void add(const float (&p)[8], f32x4 (&o)[NJ]) const {
        bf16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bf16 t[2];
            terms(p[e], t);
            hi[e] = t[0], lo[e] = t[1];
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            u32x4 f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                f[e] = __builtin_amdgcn_perm(v[2 * e + 1][j / 2], v[2 * e][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
            const bf16x8 a = __builtin_bit_cast(bf16x8, f);
            o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, hi, o[j], 0, 0, 0);
            o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, lo, o[j], 0, 0, 0);
        }
    }
};

// 8-bit pages, without turning codes into numbers one by one.
// Keys: the query as digits of 7 bits (three, for float32 four; value = sum of digit * 128^i * 2^-shift, exact
// down to 2^-20, 2^-27 of the row's largest), products of int8 in int32.  K operand of instruction (t, c): dims 64 c + 16 g
// .. + 15.
// Values: a code is exact in bf16, the upper half of its float32 form.  Lane's part of a row: dims D / 16 ln ..
template <int D, typename T>
struct Tile<D, T, int8_t> {
    static constexpr int NC = D / 64, NJ = D / 16, NV = D / 64, QD = sizeof(T) == 2 ? 3 : 4, PT = sizeof(T) == 2 ? 2 : 3;
    u32x4 k[2][NC];
    uint32_t v[8][NV];
    struct Query {
        i32x4 f[QD][NC];
        int shift;      // of the row
        float poison;   // 0; not a number where the row holds no numbers
    };

    static __device__ __forceinline__ int kcol(int g) { return 16 * g; }
    static __device__ __forceinline__ int vcol(int ln) { return NJ * ln; }
    static __device__ __forceinline__ int dim(int j, int row) { return NJ * row + j; }
    static __device__ __forceinline__ void query(Query& q, const T* x, int g) {
        float y[NC][16] = {};
        uint32_t top = 0;
        if (x) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                load8(x + 64 * c + 16 * g, y[c]);
                load8(x + 64 * c + 16 * g + 8, y[c] + 8);
            }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(y[c][e]) & 0x7fffffffu);
        const bool finite = max16(top < 0x7f800000u ? 0.f : 1.f) == 0.f;
        const float m = max16(__uint_as_float(finite ? top : 0u));
        q.poison = finite ? 0.f : __uint_as_float(0x7fc00000u);
        q.shift = 7 * QD - 1 - __builtin_amdgcn_frexp_expf(m);   // the largest becomes 2^(7 QD - 2) .. 2^(7 QD - 1)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    int n = static_cast<int>(rintf(finite ? ldexpf(y[c][e + b], q.shift) : 0.f));
#pragma unroll
                    for (int i = 0; i < QD; ++i) {
                        const int d = i + 1 < QD ? (n << 25) >> 25 : n;   // -64 .. 63, the last one up to +-65
                        n = (n - d) >> 7;
                        q.f[i][c][e / 4] = (b ? q.f[i][c][e / 4] : 0) | (d & 255) << (8 * b);
                    }
                }
    }
    __device__ __forceinline__ void load_k(int t, const char* p) {
#pragma unroll
        for (int c = 0; c < NC; ++c) k[t][c] = *reinterpret_cast<const u32x4*>(p + 64 * c);
    }
    __device__ __forceinline__ void load_v(int e, const char* p) {
        if constexpr (NV == 2) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(p);
            v[e][0] = x[0], v[e][1] = x[1];
        } else {
            v[e][0] = *reinterpret_cast<const uint32_t*>(p);
        }
    }
    __device__ __forceinline__ void clear_v(int) {}   // codes are numbers whatever they are
    __device__ __forceinline__ f32x4 scores(int t, const Query& q) const {
        i32x4 s[QD];
#pragma unroll
        for (int i = 0; i < QD; ++i) {
            s[i] = i32x4{};
#pragma unroll
            for (int c = 0; c < NC; ++c)
                s[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, k[t][c]), q.f[i][c], s[i], 0, 0, 0);
        }
        f32x4 f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {   // |s| < 2^21
            const float lo = static_cast<float>(s[1][r] * 128 + s[0][r]);
            const float hi = static_cast<float>(QD == 4 ? s[QD - 1][r] * 128 + s[2][r] : s[2][r]);
            f[r] = ldexpf(fmaf(hi, 16384.f, lo), -q.shift) + q.poison;
        }
        return f;
    }
    __device__ __forceinline__ void add(const float (&p)[8], f32x4 (&o)[NJ]) const {
        bf16x8 w[PT];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bf16 t[PT];
            terms(p[e], t);
#pragma unroll
            for (int i = 0; i < PT; ++i) w[i][e] = t[i];
        }
        each<NJ>([&](auto j) {
            u32x4 f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                f[e] = __builtin_amdgcn_perm(byte_value<j % 4>(v[2 * e + 1][j / 4]), byte_value<j % 4>(v[2 * e][j / 4]), 0x07060302u);
#pragma unroll
            for (int i = PT - 1; i >= 0; --i)
                o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), w[i], o[j], 0, 0, 0);
        });
    }
};

// float32 pages.  K operand of instruction (t, 4 c + i): dim 16 c + 4 g + i.  V operand of instruction (4 h + i, e): dim
// 64 h + 4 ln + i of key 8 g + e.
template <int D>
struct Tile<D, float, float> {
    static constexpr int NC = D / 16, NH = D / 64, NJ = D / 16;
    f32x4 k[2][NC], v[8][NH];
    struct Query {
        f32x4 f[NC];
    };

    static __device__ __forceinline__ int kcol(int g) { return 16 * g; }
    static __device__ __forceinline__ int vcol(int ln) { return 16 * ln; }
    static __device__ __forceinline__ int dim(int j, int row) { return 64 * (j / 4) + 4 * row + j % 4; }
    static __device__ __forceinline__ void query(Query& q, const float* x, int g) {
#pragma unroll
        for (int c = 0; c < NC; ++c) q.f[c] = x ? *reinterpret_cast<const f32x4*>(x + 16 * c + 4 * g) : f32x4{};
    }
    __device__ __forceinline__ void load_k(int t, const char* p) {
#pragma unroll
        for (int c = 0; c < NC; ++c) k[t][c] = *reinterpret_cast<const f32x4*>(p + 64 * c);
    }
    __device__ __forceinline__ void load_v(int e, const char* p) {
#pragma unroll
        for (int h = 0; h < NH; ++h) v[e][h] = *reinterpret_cast<const f32x4*>(p + 256 * h);
    }
    __device__ __forceinline__ void clear_v(int e) {
#pragma unroll
        for (int h = 0; h < NH; ++h) v[e][h] = f32x4{};
    }
    __device__ __forceinline__ f32x4 scores(int t, const Query& q) const {
        f32x4 s = {};
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][c][i], q.f[c][i], s, 0, 0, 0);
        return s;
    }
    __device__ __forceinline__ void add(const float (&p)[8], f32x4 (&o)[NJ]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][j / 4][j % 4], p[e], o[j], 0, 0, 0);
    }
};

// ------------------------------------------------------------------------------- the kernel
template <int D>
struct Joined {   // what the wavefronts leave for one another
    float m[kSplitWaves][kRows], l[kSplitWaves][kRows], o[kSplitWaves][kRows][D + 4];
};

// Floats of a unit's result for one query head: o[D], maximum, sum.
template <int D>
constexpr int kPart = D + 4;

template <int D, typename T, typename P>
__global__ __launch_bounds__(kBlock, sizeof(P) == 4 ? 1 : 2) void paged_attention_kernel(
    ppk::PagedCache c, const T* __restrict__ q, int64_t ldq, T* __restrict__ out, float* __restrict__ part, Split split, int groups, float scale_log2) {
    using Tl = Tile<D, T, P>;
    constexpr bool kCodes = sizeof(P) == 1;
    __shared__ Joined<D> lds;
    const ppk::PagedPlace place = ppk::paged_place(blockIdx.x, c.Hkv * groups);
    const Unit u = find_unit(split, place.unit);
    if (u.seq < 0) return;
    const int lane = threadIdx.x & 63, g = lane >> 4, ln = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = c.H / c.Hkv, kvh = place.head / groups, first = place.head % groups * kRows;
    const int heads = min(G - first, kRows), h0 = kvh * G + first;   // this workgroup's query heads

    typename Tl::Query qf;
    Tl::query(qf, ln < heads ? q + u.seq * ldq + int64_t(h0 + ln) * D : nullptr, g);

    const uint32_t row_bytes = c.Hkv * D * sizeof(P);
    const char* kp = static_cast<const char*>(c.kp) + kvh * D * sizeof(P) + Tl::kcol(g);
    const char* vp = static_cast<const char*>(c.vp) + kvh * D * sizeof(P) + Tl::vcol(ln);
    const int32_t* table = c.table + int64_t(u.seq) * c.max_pages;
    // Lane (g, ln) looks after key 8 g + ln % 8 of a step: its page, and (8-bit) the scale of its key or, from ln = 8 on, value.
    const int at = wave * kStep + 8 * g + (ln & 7);
    const float* scales = kCodes ? (ln < 8 ? c.ks : c.vs) + kvh : nullptr;
    auto page = [&](int tile) {
        const int key = tile * ppk::kPagedTile + at;
        return tile < u.tile1 && key < u.len ? table[key >> c.shift] : -1;
    };
    auto row_of = [&](int tile, int pg) { return ppk::paged_row(pg, c.n_pages, tile * ppk::kPagedTile + at, c.shift); };
    struct Buffer {
        Tl t;
        int row;
        float scale;
    };
    // Rows that hold nothing are read from row 0 and left out below.
    auto load = [&](Buffer& b, int row) {
        b.row = row;
        if (!__any(row >= 0)) return;   // past the sequence's end
        const int safe = max(row, 0);
        if constexpr (kCodes) b.scale = scales[int64_t(safe) * c.Hkv];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t r = __shfl(safe, 16 * (ln >> 2) + 4 * t + (ln & 3), kWave);
            b.t.load_k(t, kp + uint64_t(r) * row_bytes);
        }
        each<8>([&](auto e) {
            const uint32_t r = row_lane<e>(safe);
            b.t.load_v(e, vp + uint64_t(r) * row_bytes);
        });
    };

    f32x4 o[Tl::NJ];
#pragma unroll
    for (int j = 0; j < Tl::NJ; ++j) o[j] = f32x4{};
    // m: a reference that no score exceeds by more than 8 in log2 units, so that the accumulators are rescaled on few
    // steps; the same for the four lanes of a query head.  l: this lane's keys alone, until the end.
    float m = -FLT_MAX, l = 0.f;
    const float lazy = 8.0f / scale_log2;
    bool any = false;
    auto step = [&](Buffer& b) {
        if (!__any(b.row >= 0)) return;
        any = true;
        const bool full = __all(b.row >= 0);
        float s[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const f32x4 x = b.t.scores(t, qf);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[4 * t + r] = x[r];
        }
        float scale = 0.f;
        if constexpr (kCodes) {
            scale = b.row >= 0 ? b.scale : 0.f;
            each<8>([&](auto e) { s[e] *= row_lane<e>(scale); });
        }
        if (!full) {
            each<8>([&](auto e) {
                if (row_lane<e>(b.row) < 0) {
                    s[e] = -INFINITY;
                    b.t.clear_v(e);   // what lies there may be no number
                }
            });
        }
        float mx = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[e]);
        mx = max16(mx);
        if (__any(mx > m + lazy)) {
            const float m_new = fmaxf(m, mx);
            const float corr = __builtin_amdgcn_exp2f((m - m_new) * scale_log2);
            l *= corr;
#pragma unroll
            for (int j = 0; j < Tl::NJ; ++j) o[j] *= corr;
            m = m_new;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[e] = __builtin_amdgcn_exp2f((s[e] - m) * scale_log2);
            l += s[e];
        }
        if constexpr (kCodes) {
            each<8>([&](auto e) { s[e] *= row_lane<8 + e>(scale); });
        }
        b.t.add(s, o);
    };

    // Pages two tiles ahead, keys and values one.
    Buffer a, b;
    int pg = page(u.tile0), pg_next = page(u.tile0 + 1);
    load(a, row_of(u.tile0, pg));
    for (int tile = u.tile0; tile < u.tile1; tile += 2) {
        pg = page(tile + 2);
        load(b, row_of(tile + 1, pg_next));
        step(a);
        if (tile + 1 >= u.tile1) break;
        pg_next = page(tile + 3);
        load(a, row_of(tile + 2, pg));
        step(b);
    }

    // Join the wavefronts.  A maximum of -inf stands for no key at all.
    l = sum16(l);
    if (ln < heads) {
        if (g == 0) lds.m[wave][ln] = any ? m : -INFINITY, lds.l[wave][ln] = l;
#pragma unroll
        for (int j = 0; j < Tl::NJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) lds.o[wave][ln][Tl::dim(j, 4 * g + r)] = o[j][r];
    }
    __syncthreads();
    for (int x = threadIdx.x; x < heads * D; x += kBlock) {
        const int h = x / D, d = x % D;
        float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < kSplitWaves; ++w) M = fmaxf(M, lds.m[w][h]);
#pragma unroll
        for (int w = 0; w < kSplitWaves; ++w) {
            const float f = lds.m[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((lds.m[w][h] - M) * scale_log2);
            L += lds.l[w][h] * f;
            O += lds.o[w][h][d] * f;
        }
        if (u.units == 1) {
            out[(int64_t(u.seq) * c.H + h0 + h) * D + d] = static_cast<T>(M == -INFINITY ? 0.f : O / L);
        } else {
            float* p = part + (int64_t(place.unit) * c.H + h0 + h) * kPart<D>;
            p[d] = O;
            if (d == 0) p[D] = M, p[D + 1] = L;
        }
    }
}

// The units of a sequence, in their order: a workgroup takes `per` of its query heads one after another, D / 4
// lanes per unit.
template <int D, typename T>
__global__ __launch_bounds__(kBlock) void join_kernel(const float* __restrict__ part, T* __restrict__ out, Split split, int H,
                                                      int per, float scale_log2) {
    constexpr int LANES = D / 4, AT = kBlock / LANES;   // units at a time
    __shared__ float lm[AT], ll[AT];
    __shared__ f32x4 lo[AT][LANES];
    const int chunks = (H + per - 1) / per, i = blockIdx.x / chunks, h0 = blockIdx.x % chunks * per;
    const int2 u = units_of(split, i);
    if (u.y <= 1) return;
    const int w = threadIdx.x / LANES, d = threadIdx.x % LANES;
    const int64_t ld = int64_t(H) * kPart<D>;
    for (int h = h0; h < min(h0 + per, H); ++h) {
        float m = -INFINITY, l = 0.f;
        f32x4 o = {};
        const float* p = part + (int64_t(u.x) * H + h) * kPart<D>;
#pragma unroll 4
        for (int n = w; n < u.y; n += AT) {
            const float* x = p + n * ld;
            const f32x4 xo = *reinterpret_cast<const f32x4*>(x + 4 * d);
            const float xm = x[D], xl = x[D + 1], M = fmaxf(m, xm);
            const float fa = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - M) * scale_log2);
            const float fb = xm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((xm - M) * scale_log2);
            o = o * fa + xo * fb;
            l = l * fa + xl * fb;
            m = M;
        }
        lo[w][d] = o;
        if (d == 0) lm[w] = m, ll[w] = l;
        __syncthreads();
        if (threadIdx.x < LANES) {
            float M = -INFINITY, L = 0.f;
            f32x4 O = {};
#pragma unroll
            for (int n = 0; n < AT; ++n) M = fmaxf(M, lm[n]);
#pragma unroll
            for (int n = 0; n < AT; ++n) {
                const float f = lm[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((lm[n] - M) * scale_log2);
                L += ll[n] * f;
                O += lo[n][d] * f;
            }
            T* y = out + (int64_t(i) * H + h) * D + 4 * d;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = static_cast<T>(M == -INFINITY ? 0.f : O[e] / L);
        }
        __syncthreads();
    }
}

int groups_of(int H, int Hkv) { return (H / Hkv + kRows - 1) / kRows; }

constexpr int kAlone = 4, kJoinBlocks = 2048;

// Units asked for per head: about 1024 workgroups, four a CU.
int target_of(int H, int Hkv) { return max(1, 1024 / (Hkv * groups_of(H, Hkv))); }

}  // namespace

namespace ppk {

size_t paged_attention_workspace(int k, int H, int Hkv, int D) {
    return k ? (size_t(target_of(H, Hkv)) + k) * H * (D + 4) * sizeof(float) : 0;
}

void paged_attention(int dtype, const PagedCache& c, const int32_t* lens, const void* q, int64_t ldq, void* out,
                     void* part, hipStream_t s) {
    const int groups = groups_of(c.H, c.Hkv), target = target_of(c.H, c.Hkv);
    const unsigned blocks = (target + c.k + 7u) / 8 * 8 * c.Hkv * groups;
    const float scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(c.D));
    // Sequences that a short table bounds are not split: a second launch costs more than their few tiles in a row.
    const int span = paged_span(c.max_pages, c.shift), tiles = paged_tiles(span);
    const Split split{lens, c.k, span, target, tiles <= kAlone ? max(tiles, 1) : 1};
    const int per = (int64_t(c.k) * c.H + kJoinBlocks - 1) / kJoinBlocks, chunks = (c.H + per - 1) / per;
    auto go = [&](auto d, auto t, auto p) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        paged_attention_kernel<D, T, decltype(p)><<<blocks, kBlock, 0, s>>>(
            c, static_cast<const T*>(q), ldq, static_cast<T*>(out), static_cast<float*>(part), split, groups, scale_log2);
        if (tiles > kAlone)
            join_kernel<D, T><<<c.k * chunks, kBlock, 0, s>>>(static_cast<const float*>(part), static_cast<T*>(out), split, c.H,
                                                              per, scale_log2);
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
