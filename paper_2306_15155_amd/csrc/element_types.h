// Elements of the operators that take fp32, bf16 and fp16 matrices: 16-byte pieces at any element's alignment, arithmetic in fp32, one rounding
// (to nearest, ties to even) where a result is stored.  And the counter-based generator behind every dropped element.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace sensei {

struct Bf16 { unsigned short u; };
struct F16 { unsigned short u; };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(Bf16 x) { return __uint_as_float((unsigned)x.u << 16); }
__device__ __forceinline__ float to_f32(F16 x) { return (float)__builtin_bit_cast(_Float16, x.u); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ Bf16 from_f32<Bf16>(float x) { return {__builtin_bit_cast(unsigned short, (__bf16)x)}; }
template <> __device__ __forceinline__ F16 from_f32<F16>(float x) { return {__builtin_bit_cast(unsigned short, (_Float16)x)}; }

// N elements side by side.  The hardware takes wide global accesses at any address, so an odd leading dimension or head width costs no
// other path; the vector types say what alignment there is.
typedef unsigned U32x4 __attribute__((ext_vector_type(4)));
template <int BYTES, int ALIGN> struct RawOf;
template <> struct RawOf<16, 4> { typedef U32x4 type __attribute__((aligned(4))); };
template <> struct RawOf<16, 2> { typedef U32x4 type __attribute__((aligned(2))); };

template <class T, int N> struct Piece {
    typedef typename RawOf<N * (int)sizeof(T), (int)sizeof(T)>::type Raw;
    T x[N];
    __device__ __forceinline__ static Piece load(const T *p) { return __builtin_bit_cast(Piece, *reinterpret_cast<const Raw *>(p)); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<Raw *>(p) = __builtin_bit_cast(Raw, *this); }
};
template <class T> constexpr int kPerPiece = 16 / (int)sizeof(T);

constexpr float kLog2E = 1.44269502162933349609375f;        // log2(e) rounded to fp32 ...
constexpr float kLog2ELow = 1.92596303380834e-8f;           // ... and what the rounding left
constexpr float kLn2 = 0.69314718055994530942f;

// exp(x) by one product and one instruction: off by |x| 2^-24 of itself for the product's rounding, beside the instruction's unit in the last place.  For a
// softmax, whose sums weigh that with exp(x): 2^-24 / e of the largest at most.  0 for -inf, NaN stays NaN.
__device__ __forceinline__ float exp_weight(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// exp(x) for x <= 0 (a little above is fine): 2^(x log2 e) with the product's rounding put back to first order, so that the error stays at the
// exponential instruction's own unit in the last place however large |x| is.  Below -104 the result is under the smallest fp32 number
// of any kind: zero.  NaN stays NaN.
__device__ __forceinline__ float exp_neg(float x) {
    const float y = x * kLog2E;
    const float r = fmaf(x, kLog2ELow, fmaf(x, kLog2E, -y));
    const float e = __builtin_amdgcn_exp2f(y);
    return x < -104.f ? 0.f : fmaf(e * kLn2, r, e);
}

// ---- moves between lanes
template <int CTRL> __device__ __forceinline__ float dpp(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true)); }
template <int CTRL> __device__ __forceinline__ int dpp(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true); }
__device__ __forceinline__ float from_16_away(float x) { return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401F)); }

// x joined over L neighbouring lanes (1 to 64, all active) by an operation whose order does not matter but for rounding, in all of them: the
// neighbour in a pair, the other pair of a quad, lanes mirrored within eight and within sixteen, the other sixteen, the other half
template <int L, class Op> __device__ __forceinline__ float over_lanes(float x, Op op) {
    if (L >= 2) x = op(x, dpp<0xB1>(x));
    if (L >= 4) x = op(x, dpp<0x4E>(x));
    if (L >= 8) x = op(x, dpp<0x141>(x));
    if (L >= 16) x = op(x, dpp<0x140>(x));
    if (L >= 32) x = op(x, from_16_away(x));
    if (L >= 64) x = op(x, __shfl_xor(x, 32, 64));
    return x;
}
template <int L> __device__ __forceinline__ float sum_over(float x) { return over_lanes<L>(x, [](float a, float b) { return a + b; }); }
template <int L> __device__ __forceinline__ float max_over(float x) { return over_lanes<L>(x, [](float a, float b) { return fmaxf(a, b); }); }

// ---- Philox4x32 with seven rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011): four words of 32 bits from a
// 128-bit counter and a 64-bit key, nothing kept between calls, so a mask is formed again wherever it is needed.  Seven rounds are the
// fewest that the authors report to pass every test of BigCrush; ten, their default, would make the dropping of 16-bit elements bound by
// the integer multiplier (a quarter of the vector rate) and not by memory.
struct DropKey {
    unsigned k0, k1;            // the seed
    unsigned offset;            // fourth counter word, before what *offset_dev adds
    const unsigned *offset_dev; // null, or a device word that is read when the kernel runs: a replayed graph gets another mask
    unsigned threshold;         // an element is dropped when its word is below
    float keep_scale;           // 1 / (1 - p)
};
struct Words { unsigned w[4]; };

__host__ __device__ __forceinline__ Words philox(unsigned c0, unsigned c1, unsigned c2, unsigned c3, unsigned k0, unsigned k1) {
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(b >> 32) ^ c1 ^ k0;
        c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ k1;
        c3 = (unsigned)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// Division of numbers below 2^31 by a fixed one: floor(n / d) = (n * m) >> s with m = floor(2^s / d) + 1, s = 31 + ceil(log2 d): what m has too
// much is at most d <= 2^(s - 31), so n times it stays below 2^s.
struct FastDiv {
    unsigned d, m;
    int s;
    __host__ static FastDiv of(unsigned d) {
        int log = 0;
        while ((1ull << log) < d) ++log;
        return {d, (unsigned)((1ull << (31 + log)) / d + 1), 31 + log};
    }
    __host__ __device__ __forceinline__ unsigned div(unsigned n) const { return (unsigned)(((unsigned long long)n * m) >> s); }
};

}  // namespace sensei
