// Products with weights in 4 bits (msd_linear4) and the codes, scales and zeros of such a weight
// (msd_quantize4). Formats in include/msd.h.
#include <algorithm>

#include "common.cuh"
#include "msd.h"

namespace msd {

struct Weight {
    uint8_t *codes;
    bf16 *scales;
    uint8_t *zeros;
    int o, k, group, groups;
};

// y[i][j] = sum over groups of scale * sum x (code - zero): a warp per output and 8 rows of x.
template <typename T>
__global__ void __launch_bounds__(256)
linear4_kernel(const T *__restrict__ x, long ldx, int m, Weight w, float *__restrict__ y, long ldy, int accumulate) {
    wait_prior();
    allow_dependents();
    const int lane = threadIdx.x & 31, j = blockIdx.x * 8 + (threadIdx.x >> 5), i0 = blockIdx.y * 8;
    if (j >= w.o) return;
    const uint32_t *codes = reinterpret_cast<const uint32_t *>(w.codes + (long)j * (w.k / 2));
    float acc[8] = {};
    for (int c = lane; c < w.k / 8; c += 32) {
        const uint32_t q = codes[c];
        const long g = (long)j * w.groups + c * 8 / w.group;
        const float s = __bfloat162float(w.scales[g]);
        const int z = w.zeros ? w.zeros[g] : 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i0 + i >= m) break;
            const float4 a = Vec4<T>::load(x + (long)(i0 + i) * ldx + c * 8), b = Vec4<T>::load(x + (long)(i0 + i) * ldx + c * 8 + 4);
            const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) t = fmaf(v[e], (float)((int)(q >> (4 * e) & 15) - z), t);
            acc[i] = fmaf(s, t, acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i0 + i >= m) break;
        const float t = warp_sum(acc[i]);
        if (lane == 0) {
            float *at = y + (long)(i0 + i) * ldy + j;
            *at = accumulate ? *at + t : t;
        }
    }
}

// The bf16 nearest to span / n (ties to even), span = hi + lo exactly, n = 7 or 15, span >= 0. The
// fp32 quotient may sit on the other side of the midpoint of two bf16 values than the true one;
// n times the midpoint is exact, so the comparison is made there.
__device__ __forceinline__ float scale_of(float hi, float lo, float n) {
    const float q = hi / n;
    const unsigned below = __float_as_uint(q) & 0xFFFF0000u;
    const float mid = __uint_as_float(below | 0x8000u);
    const float over = fmaf(-n, mid, hi) + lo;
    const float s = __uint_as_float(below + (over > 0.f || (over == 0.f && (below & 0x10000u)) ? 0x10000u : 0u));
    return s >= 0x1p-126f ? s : 0.f;                    // 1 / s is finite
}

// w / s to the nearest integer, ties to even, |w / s| < 2^8. The residual w - q s is exact.
__device__ __forceinline__ float nearest(float w, float s, float inv) {
    float q = rintf(w * inv);
    const float r = fmaf(-q, s, w);
    const float twice = r + r;
    const bool odd = (int)q & 1;
    if (twice > s || (twice == s && odd)) q += 1.f;
    else if (twice < -s || (twice == -s && odd)) q -= 1.f;
    return q;
}

__device__ __forceinline__ float clean(float w) { return w == w ? w : 0.f; }

// One thread per group (simple form).
template <typename T>
__global__ void __launch_bounds__(128)
quantize4_kernel(const T *__restrict__ x, long ldw, Weight w, T *__restrict__ values, long ldv) {
    wait_prior();
    allow_dependents();
    const long at = (long)blockIdx.x * 128 + threadIdx.x;
    if (at >= (long)w.o * w.groups) return;
    const int j = (int)(at / w.groups), g = (int)(at % w.groups);
    const int k0 = g * w.group, k1 = min(k0 + w.group, w.k);
    const T *row = x + (long)j * ldw;
    float lo = 0.f, hi = 0.f;
    for (int k = k0; k < k1; ++k) {
        const float v = clean((float)row[k]);
        lo = fminf(lo, v);
        hi = fmaxf(hi, v);
    }
    float s, z = 8.f;
    if (w.zeros) {
        const float d = hi - lo, b = d - hi;
        s = scale_of(d, (hi - (d - b)) + (-lo - b), 15.f);
        z = s > 0.f ? fminf(fmaxf(nearest(-lo, s, 1.f / s), 0.f), 15.f) : 0.f;
        w.zeros[at] = (uint8_t)z;
    } else {
        s = scale_of(fmaxf(hi, -lo), 0.f, 7.f);
    }
    w.scales[at] = __float2bfloat16(s);
    const float inv = s > 0.f ? 1.f / s : 0.f;
    for (int k = k0; k < k1; k += 2) {
        unsigned byte = 0;
        for (int e = 0; e < 2; ++e) {
            const float v = fminf(fmaxf(clean((float)row[k + e]), -16.f * s), 16.f * s);
            const float q = s > 0.f ? fminf(fmaxf(nearest(v, s, inv) + z, 0.f), 15.f) : z;
            byte |= (unsigned)q << (4 * e);
            if (values) values[(long)j * ldv + k + e] = (T)(s * (q - z));
        }
        w.codes[(long)j * (w.k / 2) + k / 2] = (uint8_t)byte;
    }
}

static bool take_weight(const msd_weight4 *w, Weight *out) {
    if (!w || !w->codes || !w->scales || w->o < 1 || w->k < 8 || w->k % 8 || reinterpret_cast<uintptr_t>(w->codes) % 4 ||
        reinterpret_cast<uintptr_t>(w->scales) % 2 || (w->group != 32 && w->group != 64 && w->group != 128))
        return false;
    *out = Weight{w->codes, static_cast<bf16 *>(w->scales), w->zeros, w->o, w->k, w->group, (w->k + w->group - 1) / w->group};
    return true;
}

static bool bad_rows(const void *p, long ld, int dtype, int width) {
    const int size = dtype == MSD_F32 ? 4 : 2;
    return !p || ld < width || reinterpret_cast<uintptr_t>(p) % 16 || ld * size % 16;
}

}  // namespace msd

using namespace msd;

extern "C" {

msd_status msd_linear4(const void *x, int64_t ldx, int32_t x_dtype, int32_t m, const msd_weight4 *weight, float *y,
                       int64_t ldy, int32_t accumulate, void *stream) {
    Weight w;
    if (m < 0 || !take_weight(weight, &w) || (x_dtype != MSD_F32 && x_dtype != MSD_BF16)) return MSD_ERR_INVALID;
    if (m == 0) return MSD_OK;
    if (bad_rows(x, ldx, x_dtype, w.k) || !y || ldy < w.o || reinterpret_cast<uintptr_t>(y) % 4) return MSD_ERR_INVALID;
    if (m > 65535 * 8) return MSD_ERR_INVALID;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid((w.o + 7) / 8, (m + 7) / 8);
    const cudaError_t e =
        x_dtype == MSD_F32
            ? launch_chain(linear4_kernel<float>, grid, 256, 0, s, static_cast<const float *>(x), (long)ldx, m, w, y, (long)ldy, accumulate)
            : launch_chain(linear4_kernel<bf16>, grid, 256, 0, s, static_cast<const bf16 *>(x), (long)ldx, m, w, y, (long)ldy, accumulate);
    if (e != cudaSuccess) return MSD_ERR_CUDA;
    note_launch();
    return MSD_OK;
}

msd_status msd_quantize4(const void *x, int64_t ldw, int32_t dtype, const msd_weight4 *out, void *values, int64_t ldv,
                         void *stream) {
    Weight w;
    if (!take_weight(out, &w) || (dtype != MSD_F32 && dtype != MSD_BF16) || bad_rows(x, ldw, dtype, w.k) ||
        (values && bad_rows(values, ldv, dtype, w.k)))
        return MSD_ERR_INVALID;
    const long ctas = ((long)w.o * w.groups + 127) / 128;
    if (ctas > 0x7FFFFFFF) return MSD_ERR_INVALID;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e =
        dtype == MSD_F32 ? launch_chain(quantize4_kernel<float>, (unsigned)ctas, 128, 0, s, static_cast<const float *>(x), (long)ldw, w, static_cast<float *>(values), (long)ldv)
                         : launch_chain(quantize4_kernel<bf16>, (unsigned)ctas, 128, 0, s, static_cast<const bf16 *>(x), (long)ldw, w, static_cast<bf16 *>(values), (long)ldv);
    if (e != cudaSuccess) return MSD_ERR_CUDA;
    note_launch();
    return MSD_OK;
}

}  // extern "C"
