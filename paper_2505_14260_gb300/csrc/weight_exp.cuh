// Weights of tokens in fixed point: rint(2^44 * exp((logit - max) / T)) as 64-bit integers.
//
// A token is drawn where the cumulative weight passes a uniform, and top-p cuts where it passes
// a share, so what two evaluations of a weight differ by is the chance that they pick different
// tokens, once for each of up to 400,000 borders. With fp32 exponentials that is per cents over a
// flat row; at 2^-44 of the largest weight it is below 1e-7. Integers also add up to the same sum
// in any order, so nothing depends on how a row is spread over threads and CTAs.
//
// fp64 has no rate on this machine that would do (a few values per SM and cycle), so the exponent
// is a pair of fp32 values, exact to about 2^-42 where the weight counts:
//   y = (max - x) log2(e) / T = j / 1024 + g, |g| <= 2^-11;  2^-y = 2^-(j / 1024) * 2^-g
// with 2^-(j % 1024 / 1024) as a pair from a table and 2^-g = 1 - g ln 2 + (g ln 2)^2 / 2 - ..., of
// which only the first term needs more than fp32: the second is below 2^-24. About 40 fp32
// operations a weight. The table and the three terms follow from the definition of exp alone.
#pragma once

#include "common.cuh"

namespace msd {

constexpr int EXP_STEPS = 1024;
constexpr int WEIGHT_BITS = 44;             // 393216 weights of 2^44 stay below 2^63

struct alignas(16) ExpTable {
    float pair[2 * EXP_STEPS];              // 2^(-j / 1024): the fp32 value, and what it leaves
    constexpr ExpTable() : pair() {
        for (int j = 0; j < EXP_STEPS; ++j) {
            const double a = -0.69314718055994530942 * j / EXP_STEPS;
            double term = 1.0, sum = 0.0;
            for (int n = 1; n < 26; ++n) {
                sum += term;
                term *= a / n;
            }
            pair[2 * j] = (float)sum;
            pair[2 * j + 1] = (float)(sum - (double)(float)sum);
        }
    }
};

// The scale log2(e) / T of a row as a pair, and the row's largest logit (finite).
struct RowScale {
    float top, c_hi, c_lo;
};

// y = (top - x) * c as an unnormalised pair; y.x is not below 46 (or NaN) where the weight is 0.
__device__ __forceinline__ float2 exponent_of(float x, const RowScale &r) {
    const float s = r.top - x;
    const float b = s - r.top;
    const float e = (r.top - (s - b)) + (-x - b);       // s + e = top - x exactly
    const float p = __fmul_rn(s, r.c_hi);               // _rn: not to be fused with what follows
    return make_float2(p, fmaf(s, r.c_lo, fmaf(e, r.c_hi, fmaf(s, r.c_hi, -p))));
}

// 2^44 * 2^-(y.x + y.y), to a unit or two; 0 where y.x >= 46. table: in shared memory.
__device__ __forceinline__ unsigned long long weight_of(float2 y, const float2 *table) {
    constexpr float MAGIC = 12582912.f;                 // 1.5 * 2^23 = 0x4B400000: adding it rounds to an integer
    constexpr unsigned BIAS = 0x4B400000u;
    constexpr float L = -0.693147180559945309f, L_LO = (float)(-0.69314718055994530942 - (double)-0.693147180559945309f);
    const float t = fmaf(y.x, (float)EXP_STEPS, MAGIC);
    const unsigned j = __float_as_uint(t);              // BIAS + j; BIAS's low 10 bits, and the 9 above bit 13, are 0
    const float g = fmaf(t - MAGIC, -1.f / EXP_STEPS, y.x);        // exact
    const float a = __fmul_rn(g, L);
    const float a_lo = fmaf(y.y, L, fmaf(g, L_LO, fmaf(g, L, -a)));
    const float m = fmaf(a, fmaf(a, fmaf(a, 1.f / 6.f, 0.5f), a_lo), a_lo);      // e^(a + a_lo) = 1 + a + m
    const float2 w = table[j & (EXP_STEPS - 1)];
    const float h = fmaf(w.x, a, w.x);                  // h + l = (w.x + w.y) (1 + a + m)
    const float l = fmaf(w.y, a, fmaf(w.x, m, fmaf(w.x, a, w.x - h))) + w.y;
    // (h + l) * 2^(44 - n), n = j >> 10, as an integer: its part above 2^22, and what is left of it (at most 3/4 * 2^22,
    // so that MAGIC still rounds it to an integer)
    const float scale = __uint_as_float((127u + WEIGHT_BITS - 22 - (j >> 10)) << 23);
    const float v = __fmul_rn(h, scale);
    const float tv = v + MAGIC;
    const float rest = fmaf(fmaf(l, scale, v - (tv - MAGIC)), 4194304.f, MAGIC);
    const unsigned long long sum = (unsigned long long)__float_as_uint(tv) * 4194304u + __float_as_uint(rest) -
                                   ((unsigned long long)BIAS * 4194304u + BIAS);
    return y.x < 46.f ? sum : 0;
}

// Orders finite and infinite logits as unsigned numbers (-0 as 0).
__device__ __forceinline__ unsigned key_of(float x) {
    const unsigned b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float logit_of(unsigned key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

}  // namespace msd
