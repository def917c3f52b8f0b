// Attention of one query row per sequence over a paged cache: out = softmax(q k^T / sqrt(D)) v over the
// first lens[i] keys of sequence i, in whatever pages they lie.
//
// Every key and value is read once and used for the G = H / Hkv query heads that share it, so reading them bounds
// the kernel.  A wavefront has a range of 32-key steps of one key/value head (paged.h), through as many sequences as it
// spans, with a softmax's running maximum and sum of its own; wavefronts share nothing.  A sequence that lies in one range
// is written right away, the pieces of others leave (o, maximum, sum) for join_kernel.  256 workgroups of eight wavefronts,
// which have neighbouring heads of the same keys, read as fast as anything measured (2 x 415 MB of bf16 rows of 8 heads, reads
// alone: eight heads to a workgroup, 200 of these, 6.4 TB/s; one head to a workgroup of four, 1600 of these, 5.2).
// 64 sequences of 8 to 4096 keys, 32 heads in bf16 (400 MB): 76 us, 5.3 TB/s, and 5.5 for the join; 12 of 6000 to 32,768 keys, 8
// heads in 8 bits (471 MB): 91 us, 5.2 TB/s, and 5.8; 8 of as many keys in float32 (964 MB): 165 us, 5.8 TB/s, and 5.0.  512
// workgroups, steps of 64 keys, two sets of registers for what is on the way, non-temporal loads: the same or slower.
//
// Nothing passes through LDS on the way: keys go from memory into the registers that the 16 x 16 matrix
// instructions take them from.  S^T = K Q^T puts key 8 g + 4 t + r of a step into row 4 g + r of score tile t,
// so that lane group g (16 lanes) holds the scores of keys 8 g .. 8 g + 7, which is what it has to hold as the operand of
// O^T = V^T P^T; a lane reads the same 16 (or 8, or 4) columns' part of those 8 rows of V, whole rows per 16 lanes.
// The query heads are the instructions' columns; with fewer than 16 the rest are zeros (the matrix cores are idle
// otherwise: a step of 16 KB takes them 512 cycles of the 1600 that a CU's share of the memory needs).
//
// bf16 operands hold all bits of what they stand for: bf16 keys, values and queries and 8-bit codes are exact in one, and
// probabilities (times a value's scale) and float32 queries are three terms, off by 2^-25.  Codes are turned into bf16 in registers,
// two for three instructions; their scales multiply scores and probabilities.  (Fewer bits bring no time: probabilities
// of two terms, and 8-bit keys met by the query's 7-bit digits in the int8 instructions, took 80.1 and 96.3 us for the two calls above
// where this takes 80.2 and 96.5, and a query with one loud element lost the others.)
// float32 pages take the float32 matrix instructions.
#include <float.h>

#include <utility>

#include "device.h"
#include "kernels.h"
#include "paged.h"
#include "prepack.h"

namespace {

constexpr int kBlock = ppk::kPagedWaves * kWave;
constexpr int kRows = 16;   // query heads of a wavefront

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

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

struct Split {
    const int32_t* lens;
    int k, span, ranges;
    bool narrow;   // the steps of all sequences, as long as their tables, are below 2^31
};

// The lengths of sequences first .. first + 255 in a wavefront's registers, lane l those of numbers l, 64 + l, 128 + l
// and 192 + l (one wait for memory), and the steps up to and including each.
struct Lens {
    Split s;
    int first;
    int len0, len1, len2, len3;
    int64_t end0, end1, end2, end3;

    __device__ __forceinline__ void load(int i0) {
        first = i0;
        const int i = i0 + (threadIdx.x & 63);
        const int n0 = s.lens[min(i, s.k - 1)], n1 = s.lens[min(i + kWave, s.k - 1)],
                  n2 = s.lens[min(i + 2 * kWave, s.k - 1)], n3 = s.lens[min(i + 3 * kWave, s.k - 1)];
        len0 = i < s.k ? ppk::paged_len(n0, s.span) : 0;
        len1 = i + kWave < s.k ? ppk::paged_len(n1, s.span) : 0;
        len2 = i + 2 * kWave < s.k ? ppk::paged_len(n2, s.span) : 0;
        len3 = i + 3 * kWave < s.k ? ppk::paged_len(n3, s.span) : 0;
    }
    __device__ __forceinline__ int64_t scan(int len) const {
        const int n = ppk::paged_steps(len);
        if (s.narrow) return scan_up(n);
        const int lo = scan_up(n & 0xffff), hi = scan_up(n >> 16);   // at most 2^26 steps, 64 times
        return (int64_t(hi) << 16) + lo;
    }
    static __device__ __forceinline__ int64_t of_lane(int64_t x, int l) {
        return int64_t(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), l))) |
               int64_t(__builtin_amdgcn_readlane(static_cast<int>(x >> 32), l)) << 32;
    }
    // The block from sequence i0 on, `base` steps before it; the steps up to its end.
    __device__ __forceinline__ int64_t block(int i0, int64_t base) {
        load(i0);
        const int n = s.k - i0;
        end0 = base + scan(len0);
        base = of_lane(end0, 63);
        end1 = end2 = end3 = base;
        if (n > kWave) end1 = base + scan(len1), base = of_lane(end1, 63), end2 = end3 = base;
        if (n > 2 * kWave) end2 = base + scan(len2), base = of_lane(end2, 63), end3 = base;
        if (n > 3 * kWave) end3 = base + scan(len3), base = of_lane(end3, 63);
        return base;
    }
    // Steps of all sequences; the first block stays.
    __device__ __forceinline__ int64_t total() {
        if (s.k <= 4 * kWave) return block(0, 0);
        int64_t all = 0;
        for (int i0 = 4 * kWave; i0 < s.k; i0 += 4 * kWave) all = block(i0, all);
        return all + block(0, 0);
    }
    // Sequence i >= first, the same in all lanes: its length; its last step's number plus one (within the block).
    __device__ __forceinline__ int length(int i) {
        if (i >= first + 4 * kWave) load(i);
        const int c = (i - first) / kWave, l = (i - first) % kWave;
        const int a = __builtin_amdgcn_readlane(len0, l), b = __builtin_amdgcn_readlane(len1, l),
                  d = __builtin_amdgcn_readlane(len2, l), e = __builtin_amdgcn_readlane(len3, l);
        return c == 0 ? a : c == 1 ? b : c == 2 ? d : e;
    }
    __device__ __forceinline__ int64_t end(int i) const {
        const int c = (i - first) / kWave, l = (i - first) % kWave;
        const int64_t a = of_lane(end0, l), b = of_lane(end1, l), d = of_lane(end2, l), e = of_lane(end3, l);
        return c == 0 ? a : c == 1 ? b : c == 2 ? d : e;
    }
    // The sequence of step s0 < total(); its block stays.
    __device__ __forceinline__ int holding(int64_t s0) {
        int64_t base = of_lane(end3, 63);
        for (int i0 = first; base <= s0; base = block(i0, base)) i0 += 4 * kWave;
        const uint64_t a = __ballot(end0 > s0), b = __ballot(end1 > s0), c = __ballot(end2 > s0), d = __ballot(end3 > s0);
        return first + (a ? __builtin_ctzll(a) : b ? kWave + __builtin_ctzll(b) : c ? 2 * kWave + __builtin_ctzll(c) : 3 * kWave + __builtin_ctzll(d));
    }
};

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
    // f(j), j < NJ, are the values of `row` of the products; Y: float, or the type of the result.
    template <typename Y, typename F>
    static __device__ __forceinline__ void put(Y* y, int row, F f) {
        const float v[8] = {f(0), f(1), f(2), f(3), f(4), f(5), f(6), f(7)};
        store8(y + 8 * row, v);
    }
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
        bf16x8 w[3];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bf16 t[3];
            terms(p[e], t);
            w[0][e] = t[0], w[1][e] = t[1], w[2][e] = t[2];
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            u32x4 f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                f[e] = __builtin_amdgcn_perm(v[2 * e + 1][j / 2], v[2 * e][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
            const bf16x8 a = __builtin_bit_cast(bf16x8, f);
#pragma unroll
            for (int i = 2; i >= 0; --i) o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[i], o[j], 0, 0, 0);
        }
    }
};

// 8-bit pages.  A code is exact in bf16, the upper half of its float32 form.
// Keys: the query, brought into -1 .. 1 by a power of two, as one bf16 term (bf16) or three.  K operand of instruction (t, c, h):
// dims 64 c + 16 g + 8 h .. + 7.
// Values: lane's part of a row: dims D / 16 ln ..
template <int D, typename T>
struct Tile<D, T, int8_t> {
    static constexpr int NC = D / 64, NJ = D / 16, NV = D / 64, QT = sizeof(T) == 2 ? 1 : 3, PT = 3;
    u32x4 k[2][NC];
    uint32_t v[8][NV];
    struct Query {
        bf16x8 f[QT][NC][2];
        int shift;      // of the row: the terms' sum is q * 2^shift
        float poison;   // 0; not a number where the row holds no numbers
    };

    static __device__ __forceinline__ int kcol(int g) { return 16 * g; }
    static __device__ __forceinline__ int vcol(int ln) { return NJ * ln; }
    template <typename Y, typename F>
    static __device__ __forceinline__ void put(Y* y, int row, F f) {
        if constexpr (NJ == 8) {
            const float v[8] = {f(0), f(1), f(2), f(3), f(4), f(5), f(6), f(7)};
            store8(y + 8 * row, v);
        } else {
#pragma unroll
            for (int j = 0; j < NJ; ++j) y[NJ * row + j] = static_cast<Y>(f(j));
        }
    }
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
        q.shift = -__builtin_amdgcn_frexp_expf(m);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                bf16 t[QT];
                terms(finite ? ldexpf(y[c][e], q.shift) : 0.f, t);
#pragma unroll
                for (int i = 0; i < QT; ++i) q.f[i][c][e / 8][e % 8] = t[i];
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
        f32x4 s = {};
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 f;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t x = k[t][c][2 * h + w];
                    f[2 * w] = __builtin_amdgcn_perm(byte_value<1>(x), byte_value<0>(x), 0x07060302u);
                    f[2 * w + 1] = __builtin_amdgcn_perm(byte_value<3>(x), byte_value<2>(x), 0x07060302u);
                }
#pragma unroll
                for (int i = QT - 1; i >= 0; --i)
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), q.f[i][c][h], s, 0, 0, 0);
            }
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = ldexpf(s[r], -q.shift) + q.poison;
        return s;
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
    template <typename Y, typename F>
    static __device__ __forceinline__ void put(Y* y, int row, F f) {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const f32x4 v = {f(4 * h), f(4 * h + 1), f(4 * h + 2), f(4 * h + 3)};
            *reinterpret_cast<f32x4*>(y + 64 * h + 4 * row) = v;
        }
    }
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
struct Joined {   // what the wavefronts of a workgroup that has one sequence leave for one another
    float m[ppk::kPagedWaves][kRows], l[ppk::kPagedWaves][kRows], o[ppk::kPagedWaves][kRows][D + 4];
};

// Floats of a piece's result for one query head: o[D], maximum (-inf: no key), sum.  A range leaves at most two pieces:
// number 0 starts with the range, number 1 does not.
template <int D>
constexpr int kPart = D + 4;
template <int D>
__device__ __forceinline__ int64_t part_at(int range, int piece, int H, int h) {
    return ((int64_t(range) * 2 + piece) * H + h) * kPart<D>;
}

// What a range leaves for the joining workgroup of its number: the sequence that it continues, of `pieces` pieces, is
// joined by pieces - 1 workgroups, and this one is number `turn`.  Piece x is in range `first` + x, but with fewer steps
// than ranges (steps > 0: their number) a step is a piece, and `first` the first one.  The first piece is number p0 there.
struct Join {
    int seq, pieces, turn, first, p0, steps;   // seq < 0: nothing to join
};
constexpr size_t kJoinBytes = 32;
static_assert(sizeof(Join) <= kJoinBytes, "room in the workspace");

// WHOLE: a workgroup has one sequence for one head, its wavefronts every eighth step, joined through LDS.
template <int D, typename T, typename P, bool WHOLE>
__global__ __launch_bounds__(kBlock, 2) void paged_attention_kernel(ppk::PagedCache c, const T* __restrict__ q,
                                                                    int64_t ldq, T* __restrict__ out,
                                                                    float* __restrict__ part, char* __restrict__ joins,
                                                                    Split split, int groups,
                                                                    float scale_log2) {
    using Tl = Tile<D, T, P>;
    constexpr bool kCodes = sizeof(P) == 1;
    const int lane = threadIdx.x & 63, g = lane >> 4, ln = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // Where this wavefront is: step `st` of sequence `seq`, which has `steps`; `left` steps to go after it.
    struct Where {
        int seq, st, len, steps;
    };
    Lens lens = {split};
    Where at = {};
    int64_t left;
    const int all_heads = c.Hkv * groups;
    const ppk::PagedPlace place = WHOLE ? ppk::PagedPlace{0, static_cast<int32_t>(blockIdx.x % all_heads)}
                                        : ppk::paged_place(blockIdx.x, gridDim.x, wave, all_heads);
    const int head = place.head, range = place.range;
    if (!WHOLE && range >= split.ranges) return;
    const int G = c.H / c.Hkv, kvh = head / groups, first = head % groups * kRows;
    const int heads = min(G - first, kRows), h0 = kvh * G + first;   // this wavefront's query heads
    auto zero = [&](int seq) {
        if (ln >= heads) return;
        T* y = out + (int64_t(seq) * c.H + h0 + ln) * D;
#pragma unroll
        for (int r = 0; r < 4; ++r) Tl::put(y, 4 * g + r, [](int) { return 0.f; });
    };
    bool begins = true;      // the piece starts with its sequence
    int piece = 0;
    if constexpr (WHOLE) {
        at.seq = blockIdx.x / all_heads;
        at.st = wave;
        at.len = ppk::paged_len(split.lens[at.seq], split.span);
        at.steps = ppk::paged_steps(at.len);
        left = (at.steps - wave + ppk::kPagedWaves - 1) / ppk::kPagedWaves;
    } else {
        const int64_t all = lens.total(), s0 = ppk::paged_start(range, all, split.ranges);
        left = ppk::paged_start(range + 1, all, split.ranges) - s0;
        Join join = {-1, 0, 0, 0, 0, 0};
        if (left > 0) {
            at.seq = lens.holding(s0);
            at.len = lens.length(at.seq);
            at.steps = ppk::paged_steps(at.len);
            at.st = at.steps - static_cast<int>(lens.end(at.seq) - s0);
            if (at.st > 0) {
                const int64_t begin = s0 - at.st;
                const int r0 = ppk::paged_range(begin, all, split.ranges);
                if (all < split.ranges)
                    join = {at.seq, at.steps, at.st - 1, static_cast<int>(begin), 0, static_cast<int>(all)};
                else
                    join = {at.seq, ppk::paged_range(begin + at.steps - 1, all, split.ranges) - r0 + 1, range - r0 - 1, r0,
                            ppk::paged_start(r0, all, split.ranges) == begin ? 0 : 1, 0};
            }
        }
        if (head == 0 && lane == 0) *reinterpret_cast<Join*>(joins + range * kJoinBytes) = join;
        if (range == 0) {   // sequences without keys: those before the first step here, the others behind the sequence before them
            const int n = all > 0 ? lens.holding(0) : split.k;   // (this range may be empty itself)
            for (int i = 0; i < n; ++i) zero(i);
        }
        if (left <= 0) return;
        begins = at.st == 0;
    }

    const uint32_t row_bytes = c.Hkv * D * sizeof(P);
    const char* kp = static_cast<const char*>(c.kp) + kvh * D * sizeof(P) + Tl::kcol(g);
    const char* vp = static_cast<const char*>(c.vp) + kvh * D * sizeof(P) + Tl::vcol(ln);
    // Lane (g, ln) looks after key 8 g + ln % 8 of a step: its page, and (8-bit) the scale of its key or, from ln = 8 on, value.
    const int mine = 8 * g + (ln & 7);
    const float* scales = kCodes ? (ln < 8 ? c.ks : c.vs) + kvh : nullptr;
    // (No load of the loop below is behind a branch: the compiler would wait for all of them where the ways join.)
    auto page = [&](const Where& w) {
        const int key = max(min(w.st * ppk::kPagedStep + mine, w.len - 1), 0);
        return c.table[int64_t(w.seq) * c.max_pages + (key >> c.shift)];
    };
    auto row_of = [&](const Where& w, int pg) {
        const int key = w.st * ppk::kPagedStep + mine;
        return key < w.len ? ppk::paged_row(pg, c.n_pages, key, c.shift) : -1;
    };
    auto advance = [&](Where& w) {
        if constexpr (WHOLE) {
            w.st += ppk::kPagedWaves;
        } else if (++w.st >= w.steps) {
            int n = w.seq + 1, len = 0;
            while (n < split.k && (len = lens.length(n)) == 0) ++n;
            if (n < split.k) w = {n, 0, len, ppk::paged_steps(len)};   // (else past the last range's end)
        }
    };
    // Rows that hold nothing are read from row 0 and left out below.
    Tl t;
    auto load_k = [&](int row) {
        const int safe = max(row, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t r = __shfl(safe, 16 * (ln >> 2) + 4 * i + (ln & 3), kWave);
            t.load_k(i, kp + uint64_t(r) * row_bytes);
        }
        return kCodes ? scales[int64_t(safe) * c.Hkv] : 0.f;
    };
    auto load_v = [&](int row) {
        const int safe = max(row, 0);
        each<8>([&](auto e) {
            const uint32_t r = row_lane<e>(safe);
            t.load_v(e, vp + uint64_t(r) * row_bytes);
        });
    };
    typename Tl::Query qf;
    auto load_q = [&](int seq) { Tl::query(qf, ln < heads ? q + seq * ldq + int64_t(h0 + ln) * D : nullptr, g); };

    f32x4 o[Tl::NJ];
    // m: a reference that no score exceeds by more than 8 in log2 units, so that the accumulators are rescaled on few
    // steps; the same for the four lanes of a query head.  l: this lane's keys alone, until the end.
    float m, l;
    bool any;
    auto clear = [&] {
#pragma unroll
        for (int j = 0; j < Tl::NJ; ++j) o[j] = f32x4{};
        m = -FLT_MAX, l = 0.f, any = false;
    };
    clear();
    const float lazy = 8.0f / scale_log2;

    // Write what ends here: a whole sequence, or a piece.
    auto flush = [&](int seq, bool complete) {
        const float L = sum16(l);
        if (ln >= heads) return;
        if (complete) {
            T* y = out + (int64_t(seq) * c.H + h0 + ln) * D;
            const float inv = any ? 1.0f / L : 0.f;   // 0 / 0: scores of -inf alone
#pragma unroll
            for (int r = 0; r < 4; ++r) Tl::put(y, 4 * g + r, [&](int j) { return any ? o[j][r] * inv : 0.f; });
        } else {
            float* y = part + part_at<D>(range, piece, c.H, h0 + ln);
#pragma unroll
            for (int r = 0; r < 4; ++r) Tl::put(y, 4 * g + r, [&](int j) { return o[j][r]; });
            if (g == 0) y[D] = any ? m : -INFINITY, y[D + 1] = L;
        }
    };

    if (left > 0) {
        Where next = at;
        advance(next);
        int row = row_of(at, page(at)), page_next = page(next);
        load_q(at.seq);
        float scale = load_k(row);
        load_v(row);
        // The registers of a step's keys take the next step's as soon as the scores are formed, those of the values after the
        // second product, and the other wavefronts fill the wait; a page number is read two steps ahead.
        auto step = [&](auto more) {
            int row_next = -1;
            Where then = next;
            if constexpr (more) {
                advance(then);
                row_next = row_of(next, page_next);
                page_next = page(then);
            }
            float s[8], scale_next = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const f32x4 x = t.scores(i, qf);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[4 * i + r] = x[r];
            }
            // (Loads are kept from moving up, where they would need registers of their own.)
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (more) {
                if (!WHOLE && next.seq != at.seq) load_q(next.seq);
                scale_next = load_k(row_next);
            }
            __builtin_amdgcn_sched_barrier(0);
            any |= __any(row >= 0);
            if constexpr (kCodes) {
                scale = row >= 0 ? scale : 0.f;
                each<8>([&](auto e) { s[e] *= row_lane<e>(scale); });
            }
            if (!__all(row >= 0)) {
                each<8>([&](auto e) {
                    if (row_lane<e>(row) < 0) {
                        s[e] = -INFINITY;
                        t.clear_v(e);   // what lies there may be no number
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
            if constexpr (kCodes) each<8>([&](auto e) { s[e] *= row_lane<8 + e>(scale); });
            t.add(s, o);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (more) load_v(row_next);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (!WHOLE) {
                const bool ends = at.st + 1 == at.steps;
                if (!more || ends) {
                    flush(at.seq, begins && ends);
                    if (ends) {   // (`next` stays in this sequence if it is the last one with keys)
                        const int end = next.seq > at.seq ? next.seq : split.k;
                        for (int i = at.seq + 1; i < end; ++i) zero(i);
                    }
                    clear();
                    begins = true, piece = 1;
                }
            }
            at = next, next = then, row = row_next, scale = scale_next;
        };
#pragma unroll 1
        for (; left > 1; --left) step(std::true_type{});
        step(std::false_type{});
    }

    if constexpr (WHOLE) {
        __shared__ Joined<D> lds;
        const float L = sum16(l);
        if (ln < heads) {
            if (g == 0) lds.m[wave][ln] = any ? m : -INFINITY, lds.l[wave][ln] = L;
#pragma unroll
            for (int r = 0; r < 4; ++r) Tl::put(lds.o[wave][ln], 4 * g + r, [&](int j) { return o[j][r]; });
        }
        __syncthreads();
        const int seq = blockIdx.x / all_heads;
        for (int x = threadIdx.x; x < heads * D; x += kBlock) {
            const int h = x / D, d = x % D;
            float M = -INFINITY, S = 0.f, O = 0.f;
#pragma unroll
            for (int w = 0; w < ppk::kPagedWaves; ++w) M = fmaxf(M, lds.m[w][h]);
#pragma unroll
            for (int w = 0; w < ppk::kPagedWaves; ++w) {
                const float f = lds.m[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((lds.m[w][h] - M) * scale_log2);
                S += lds.l[w][h] * f;
                O += lds.o[w][h][d] * f;
            }
            out[(int64_t(seq) * c.H + h0 + h) * D + d] = static_cast<T>(M == -INFINITY ? 0.f : O / S);
        }
    }
}

// The pieces of sequences that span ranges, in their order.  Workgroup r joins heads of the sequence that range r
// continues, every (pieces - 1)th of them, so that all workgroups have about as much to read.
constexpr int kJoin = 512;
template <int D, typename T>
__global__ __launch_bounds__(kJoin) void join_kernel(const float* __restrict__ part, const char* __restrict__ joins,
                                                     T* __restrict__ out, int ranges, int H, float scale_log2) {
    constexpr int LANES = D / 4, AT = kJoin / LANES, PER = kWave / LANES;   // lanes of a piece; pieces at a time
    __shared__ float lm[AT], ll[AT];
    __shared__ f32x4 lo[AT][LANES];
    const Join j = *reinterpret_cast<const Join*>(joins + blockIdx.x * kJoinBytes);
    if (j.seq < 0 || j.turn >= H) return;
    const int d = threadIdx.x % LANES;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {};
    // pieces from x0 on, every `step`th, of head h into m, l and o
    auto gather = [&](int h, int x0, int step) {
        m = -INFINITY, l = 0.f, o = f32x4{};
#pragma unroll 4
        for (int x = x0; x < j.pieces; x += step) {
            const int r = j.steps ? ppk::paged_range(j.first + x, j.steps, ranges) : j.first + x;
            const float* p = part + part_at<D>(r, x ? 0 : j.p0, H, h);
            const f32x4 xo = *reinterpret_cast<const f32x4*>(p + 4 * d);
            const float xm = p[D], xl = p[D + 1], M = fmaxf(m, xm);
            const float fa = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - M) * scale_log2);
            const float fb = xm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((xm - M) * scale_log2);
            o = o * fa + xo * fb;
            l = l * fa + xl * fb;
            m = M;
        }
    };
    auto write = [&](int h, float M, float L, const f32x4& O) {
        T* y = out + (int64_t(j.seq) * H + h) * D + 4 * d;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = static_cast<T>(M == -INFINITY ? 0.f : O[e] / L);
    };
    if (j.pieces <= 8 * PER) {   // a wavefront joins a head's few pieces by itself
        const int w = threadIdx.x % kWave / LANES;
        for (int h = j.turn + threadIdx.x / kWave * (j.pieces - 1); h < H; h += kJoin / kWave * (j.pieces - 1)) {
            gather(h, w, PER);
#pragma unroll
            for (int s = LANES; s < kWave; s *= 2) {
                const float M = fmaxf(m, __shfl_xor(m, s, kWave));
                const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - M) * scale_log2);
                o *= f, l *= f, m = M;
                l += __shfl_xor(l, s, kWave);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], s, kWave);
            }
            if (w == 0) write(h, m, l, o);
        }
        return;
    }
    const int w = threadIdx.x / LANES;
    for (int h = j.turn; h < H; h += j.pieces - 1) {
        gather(h, w, AT);
        lo[w][d] = o;
        if (d == 0) lm[w] = m, ll[w] = l;
        __syncthreads();
        if (threadIdx.x < LANES) {
            float M = -INFINITY, L = 0.f;
            f32x4 O = {};
#pragma unroll
            for (int x = 0; x < AT; ++x) M = fmaxf(M, lm[x]);
#pragma unroll
            for (int x = 0; x < AT; ++x) {
                const float f = lm[x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((lm[x] - M) * scale_log2);
                L += ll[x] * f;
                O += lo[x][d] * f;
            }
            write(h, M, L, O);
        }
        __syncthreads();
    }
}

int heads_of(int H, int Hkv) { return Hkv * ((H / Hkv + kRows - 1) / kRows); }

// Sequences that a short table bounds are a workgroup's each, in one launch, if the workgroups find room at once.  Ranges
// and their join, and this, in us: one sequence of 500 keys, 8 heads in bf16 10.5 and 8.1, of 1000 12.4 and 12.5, of 2000
// 12.5 and 20.8; 8 bits, 1000: 12.5 and 11.7; eight sequences of up to 485 keys, 2 heads of 64 in float32, 9.5 and 9.4, of up
// to 895 9.9 and 13.4.  (The lengths are the device's: a short sequence with a long table is split, 285 keys 10.6 rather than 6.6.)
constexpr int kWhole = 1024, kWholeF32 = 512, kWholeBlocks = 256;

}  // namespace

namespace ppk {

size_t paged_attention_workspace(int k, int H, int Hkv, int D) {
    return k ? size_t(paged_ranges(heads_of(H, Hkv))) * (2 * H * (D + 4) * sizeof(float) + kJoinBytes) : 0;
}

void paged_attention(int dtype, const PagedCache& c, const int32_t* lens, const void* q, int64_t ldq, void* out,
                     void* part, hipStream_t s) {
    const int heads = heads_of(c.H, c.Hkv), groups = heads / c.Hkv, span = paged_span(c.max_pages, c.shift);
    const float scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(c.D));
    const Split split{lens, c.k, span, paged_ranges(heads), int64_t(c.k) * paged_steps(span) <= INT32_MAX};
    const bool whole = span <= (c.kv_type == PP_KV_F32 ? kWholeF32 : kWhole) && int64_t(c.k) * heads <= kWholeBlocks;
    char* joins = static_cast<char*>(part) + split.ranges * (2 * c.H * (c.D + 4) * sizeof(float));
    auto go = [&](auto d, auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr int D = decltype(d)::value;
        const T* x = static_cast<const T*>(q);
        T* y = static_cast<T*>(out);
        float* f = static_cast<float*>(part);
        if (whole) {
            paged_attention_kernel<D, T, P, true><<<c.k * heads, kBlock, 0, s>>>(c, x, ldq, y, f, joins, split, groups, scale_log2);
            return;
        }
        paged_attention_kernel<D, T, P, false><<<paged_groups(heads), kBlock, 0, s>>>(c, x, ldq, y, f, joins, split, groups, scale_log2);
        if (split.ranges > 1) join_kernel<D, T><<<split.ranges, kJoin, 0, s>>>(f, joins, y, split.ranges, c.H, scale_log2);
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
