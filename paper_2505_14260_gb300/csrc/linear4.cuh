// Weights in 4 bits: what the kernels of their products share.
#pragma once

#include "common.cuh"
#include "msd.h"

namespace msd {

struct Weight {
    uint8_t *codes;
    bf16 *scales;
    uint8_t *zeros;
    int o, k, group, groups;
};

// Codes i and i + 4 of a word (i < 4, the word shifted by 4 i) less the zero, as a bf16 pair. off: 128 + zero, twice.
__device__ __forceinline__ uint32_t pair_of(uint32_t shifted, __nv_bfloat162 off) {
    uint32_t v;
    asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(v) : "r"(shifted));      // (a & b) | c
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<__nv_bfloat162 *>(&v), off);
    return *reinterpret_cast<const uint32_t *>(&d);
}

// 8 values of x as the pairs (0, 4), (1, 5), (2, 6), (3, 7); fp32 as three bf16 planes that add up to them.
template <typename T> struct Octet;
template <> struct Octet<bf16> {
    static constexpr int PLANES = 1;
    uint4 v;
    __device__ __forceinline__ void load(const bf16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void pairs(uint32_t (&b)[1][4]) const {
        b[0][0] = __byte_perm(v.x, v.z, 0x5410);
        b[0][1] = __byte_perm(v.x, v.z, 0x7632);
        b[0][2] = __byte_perm(v.y, v.w, 0x5410);
        b[0][3] = __byte_perm(v.y, v.w, 0x7632);
    }
};
template <> struct Octet<float> {
    static constexpr int PLANES = 3;
    float4 lo, hi;
    __device__ __forceinline__ void load(const float *p) {
        lo = *reinterpret_cast<const float4 *>(p);
        hi = *reinterpret_cast<const float4 *>(p + 4);
    }
    __device__ __forceinline__ void clear() { lo = hi = make_float4(0.f, 0.f, 0.f, 0.f); }
    // A value's upper 16 bits, those of what is left, and the 8 bits left then: truncations, so the three parts add
    // up to it (but for what lies below 2^-133) and none overflows. What is not finite leaves NaN in the later parts.
    static __device__ __forceinline__ void part(float a, float c, uint32_t (&b)[3][4], int i) {
        const auto upper = [](float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); };
        const float ra = a - upper(a), rc = c - upper(c), la = ra - upper(ra), lc = rc - upper(rc);
        b[0][i] = __byte_perm(__float_as_uint(a), __float_as_uint(c), 0x7632);
        b[1][i] = __byte_perm(__float_as_uint(ra), __float_as_uint(rc), 0x7632);
        b[2][i] = __byte_perm(__float_as_uint(la), __float_as_uint(lc), 0x7632);
    }
    __device__ __forceinline__ void pairs(uint32_t (&b)[3][4]) const {
        part(lo.x, hi.x, b, 0);
        part(lo.y, hi.y, b, 1);
        part(lo.z, hi.z, b, 2);
        part(lo.w, hi.w, b, 3);
    }
};

// Products on the 5th-generation tensor cores (linear4_tc.cu). stall: chunks of 128 elements of K from this one on never get
// their codes, so that the waits for them run out (a test).
constexpr int NO_STALL = 0x7FFFFFFF;
template <typename T>
cudaError_t launch_linear4_tc(const T *x, long ldx, int m, const Weight &w, float *y, long ldy, int accumulate, cudaStream_t s,
                              int stall = NO_STALL);

// How they are launched: rows and outputs to a CTA, parts of K, whether scales and zeros are staged (`slice` groups of them) and codes
// read without tensor copies.
struct Linear4Shape {
    int rows, outputs, split;
    bool staged, direct;
    int slice;
    size_t smem;
};
template <typename T> Linear4Shape linear4_tc_shape(int m, const Weight &w);

// About how long up to 16 rows take there.
template <typename T> float linear4_tc_us(const Weight &w);

}  // namespace msd
