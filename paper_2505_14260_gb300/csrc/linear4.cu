// Products with weights in 4 bits (msd_linear4) and the codes, scales and zeros of such a weight
// (msd_quantize4). Formats in include/msd.h.
#include <algorithm>
#include <type_traits>

#include "linear4.cuh"

namespace msd {

// ---------------------------------------------------------------------------
// A few rows of x (m <= 16): mma.sync m16n8k16, weights as A (16 outputs), rows of x as B.
//
// The codes are what has to be read, and at the rate of memory 50 of them arrive per SM and
// cycle, so what counts is instructions per code. A word of 8 codes becomes 4 bf16 pairs with
// three shifts, four selections (code | 0x4300 is the bf16 128 + code) and four subtractions of
// 128 + zero (exact), 11 for 8 codes of a lane; the products' order within a word is free, so
// pairs are (0, 4), (1, 5), (2, 6), (3, 7) of it and x is permuted alike. Each mma takes codes of
// one group, and a group's sum is scaled on the way into the total, so no weight is rounded. (A tensor core cuts a sum's last
// bits at each product added: fp32's later planes have sums of their own, which cost nothing. Groups of 128: errors of 8e-8, not 4.4e-7.)
//
// A warp has 32 outputs and every 8th run of groups; the 8 warps' totals meet in shared memory in
// a fixed order. Weights go from memory to registers, DEPTH chunks of 128 elements ahead; x is
// read from the caches (16 bytes a lane and word).
// ---------------------------------------------------------------------------
constexpr int FEW_WARPS = 8, FEW_OUT = 32, FEW_DEPTH = 3;
constexpr size_t FEW_BESIDE = 64 * 1024;        // room for scales and zeros

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// GROUP elements share a scale; lane t % 4 has GROUP / 4 consecutive ones of each group of its rows. NT: tiles of 8
// rows of x. WIDE: the codes of a lane and group are aligned to their size.
template <typename T, int GROUP, int NT, bool WIDE>
__global__ void __launch_bounds__(FEW_WARPS * 32)
linear4_few_kernel(const T *__restrict__ x, long ldx, int m, Weight w, float *__restrict__ y, long ldy, int accumulate) {
    constexpr int WORDS = GROUP / 32;           // words of a lane, row and group
    constexpr int PER = 128 / GROUP;            // groups of a chunk
    constexpr int P = Octet<T>::PLANES;
    wait_prior();
    allow_dependents();
    extern __shared__ __align__(16) uint8_t smem[];
    float *part = reinterpret_cast<float *>(smem);                                  // [warps][FEW_OUT][NT * 8]
    bf16 *scales = reinterpret_cast<bf16 *>(smem + FEW_WARPS * FEW_OUT * NT * 8 * 4);   // [FEW_OUT][groups]
    uint8_t *zeros = reinterpret_cast<uint8_t *>(scales + FEW_OUT * w.groups);          // [FEW_OUT][groups]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int j0 = blockIdx.x * FEW_OUT, outs = min(FEW_OUT, w.o - j0);
    const int chunks = (w.groups + PER - 1) / PER, c0 = chunks * warp / FEW_WARPS, c1 = chunks * (warp + 1) / FEW_WARPS;
    const int words_row = w.k / 8;
    const uint32_t *codes = reinterpret_cast<const uint32_t *>(w.codes);
    const uint32_t *row[4];                     // outputs g, g + 8, g + 16, g + 24; the last one's codes stand in for those past it
#pragma unroll
    for (int r = 0; r < 4; ++r) row[r] = codes + (long)(j0 + min(g + 8 * r, outs - 1)) * words_row;

    uint32_t q[FEW_DEPTH][4][4];                // [chunk][row][word]
    auto fetch = [&](int c, uint32_t (&to)[4][4]) {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int at = (c * PER + e) * (GROUP / 8) + t * WORDS;       // first word
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t *d = to[r] + e * WORDS;
                if (WIDE && at + WORDS <= words_row) {
                    if constexpr (WORDS == 4) {
                        const uint4 v = __ldcs(reinterpret_cast<const uint4 *>(row[r] + at));
                        d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
                    } else if constexpr (WORDS == 2) {
                        const uint2 v = __ldcs(reinterpret_cast<const uint2 *>(row[r] + at));
                        d[0] = v.x; d[1] = v.y;
                    } else {
                        d[0] = __ldcs(row[r] + at);
                    }
                } else {
#pragma unroll
                    for (int v = 0; v < WORDS; ++v) d[v] = at + v < words_row ? __ldcs(row[r] + at + v) : 0;
                }
            }
        }
    };
#pragma unroll
    for (int d = 0; d < FEW_DEPTH; ++d)
        if (c0 + d < c1) fetch(c0 + d, q[d]);

    {   // scales and zeros of the tile: one run of each, in 16-byte pieces where they lie so
        const auto copy = [&](uint8_t *to, const uint8_t *from, int bytes) {
            constexpr int T = FEW_WARPS * 32, U = 4;
            int done = 0;
            if (reinterpret_cast<uintptr_t>(from) % 16 == 0) {
                const int n = bytes / 16;
                for (int i0 = tid; i0 < n; i0 += U * T) {
                    uint4 v[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) v[u] = reinterpret_cast<const uint4 *>(from)[min(i0 + u * T, n - 1)];
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (i0 + u * T < n) reinterpret_cast<uint4 *>(to)[i0 + u * T] = v[u];
                }
                done = n * 16;
            }
            for (int i = done + tid; i < bytes; i += T) to[i] = from[i];
        };
        copy(reinterpret_cast<uint8_t *>(scales), reinterpret_cast<const uint8_t *>(w.scales + (long)j0 * w.groups), outs * w.groups * 2);
        if (w.zeros) copy(zeros, w.zeros + (long)j0 * w.groups, outs * w.groups);
    }
    __syncthreads();

    float total[2][NT][4] = {};
    const T *xr[NT];
    bool on[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        on[n] = 8 * n + g < m;
        xr[n] = x + (long)(on[n] ? 8 * n + g : 0) * ldx;
    }
    auto chunk = [&](int c, const uint32_t (&from)[4][4]) {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int group = c * PER + e;
            if (PER > 1 && group >= w.groups) break;
            float acc[P > 1 ? 2 : 1][2][NT][4] = {};                                // fp32: the first planes, the later ones
            __nv_bfloat162 off[4];
            float sc[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = min(g + 8 * r, outs - 1) * w.groups + group;
                const unsigned o = 0x4300u + (w.zeros ? zeros[at] : 8u);             // 128 + zero
                const uint32_t both = o | o << 16;
                off[r] = *reinterpret_cast<const __nv_bfloat162 *>(&both);
                sc[r] = __bfloat162float(scales[at]);
            }
#pragma unroll
            for (int v = 0; v < WORDS; ++v) {
                const int at = (group * (GROUP / 8) + t * WORDS + v) * 8;           // first element of the word
                Octet<T> o[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (on[n] && at < w.k) o[n].load(xr[n] + at); else o[n].clear();
                }
                uint32_t a[4][4];
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[r][i] = pair_of(from[r][e * WORDS + v] >> (4 * i), off[r]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint32_t b[P][4];
                    o[n].pairs(b);
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            mma_16816(acc[p > 0][h][n], a[2 * h][0], a[2 * h + 1][0], a[2 * h][1], a[2 * h + 1][1], b[p][0], b[p][1]);
                            mma_16816(acc[p > 0][h][n], a[2 * h][2], a[2 * h + 1][2], a[2 * h][3], a[2 * h + 1][3], b[p][2], b[p][3]);
                        }
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float sum = P > 1 ? acc[0][h][n][i] + acc[P > 1][h][n][i] : acc[0][h][n][i];
                        total[h][n][i] = fmaf(sc[2 * h + (i >> 1)], sum, total[h][n][i]);
                    }
        }
    };
    for (int c = c0; c < c1; c += FEW_DEPTH) {
#pragma unroll
        for (int d = 0; d < FEW_DEPTH; ++d) {
            if (c + d < c1) {
                chunk(c + d, q[d]);
                if (c + d + FEW_DEPTH < c1) fetch(c + d + FEW_DEPTH, q[d]);
            }
        }
    }

    // totals of the warps, added in their order
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                part[(warp * NT * 8 + n * 8 + 2 * t + (i & 1)) * FEW_OUT + 16 * h + 8 * (i >> 1) + g] = total[h][n][i];
    __syncthreads();
    for (int i = tid; i < NT * 8 * FEW_OUT; i += FEW_WARPS * 32) {
        const int j = i % FEW_OUT, r = i / FEW_OUT;
        if (j >= outs || r >= m) continue;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < FEW_WARPS; ++k) v += part[(k * NT * 8 + r) * FEW_OUT + j];
        float *to = y + (long)r * ldy + j0 + j;
        *to = accumulate ? *to + v : v;
    }
}

template <typename T>
using FewKernel = void (*)(const T *, long, int, Weight, float *, long, int);

template <typename T, int GROUP>
static FewKernel<T> few_kernel(bool two, bool wide) {
    if constexpr (sizeof(T) == 2)               // (fp32: 8 rows at most)
        if (two) return wide ? linear4_few_kernel<T, GROUP, 2, true> : linear4_few_kernel<T, GROUP, 2, false>;
    return wide ? linear4_few_kernel<T, GROUP, 1, true> : linear4_few_kernel<T, GROUP, 1, false>;
}

static size_t few_beside(const Weight &w) { return (size_t)FEW_OUT * w.groups * 3; }

static Linear4Shape few_shape(int m, const Weight &w) {
    const int align = w.group / 8;              // bytes of a lane's codes of a group
    const bool wide = reinterpret_cast<uintptr_t>(w.codes) % align == 0 && w.k / 2 % align == 0;
    const int step = m > 8 ? 16 : 8;            // m <= 16
    return Linear4Shape{step, FEW_OUT, 1, true, !wide, w.groups, (size_t)FEW_WARPS * FEW_OUT * step * 4 + few_beside(w)};
}

template <typename T>
static cudaError_t launch_few(const T *x, long ldx, int m, const Weight &w, float *y, long ldy, int accumulate, cudaStream_t s) {
    const Linear4Shape c = few_shape(m, w);
    const bool wide = !c.direct;
    const FewKernel<T> f = w.group == 128 ? few_kernel<T, 128>(m > 8, wide) : w.group == 64 ? few_kernel<T, 64>(m > 8, wide) : few_kernel<T, 32>(m > 8, wide);
    const size_t smem = c.smem;
    constexpr size_t most = (size_t)FEW_WARPS * FEW_OUT * 16 * 4 + FEW_BESIDE;
    cudaError_t e = cudaSuccess;
    // (one value, whatever the call: another thread may be between this and its launch)
    if (smem > 48 * 1024) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e == cudaSuccess) {
        e = launch_chain(f, (w.o + FEW_OUT - 1) / FEW_OUT, FEW_WARPS * 32, smem, s, x, ldx, m, w, y, ldy, accumulate);
        note_launch();
    }
    return e;
}

// Whether these kernels take less time than the ones on tcgen05: a CTA of 32 outputs takes 2.5 us and a time for each element of a row
// (1, 8 and 16 rows, k 1024 to 11008, groups of 32, 64 and 128), and 152 of them run at a time; two on an SM, as those of up to 8 bf16
// rows do, take about as long as one after the other. (One row, groups of 128: k and o 4096 6.3 us here, 9.7 there; k 11008 12.3 and
// 15.2; o 32000 25.5 and 25.0. Groups of 32: k 1024 4.5 and 7.6, o 11008 31 and 19. 16 rows, o 11008, groups of 128: 21 and 13.5.)
// Rows whose scales would not fit beside the sums (k past 21824, 43648 and 87296) take less time there in any case.
template <typename T>
static bool few_rows(int m, const Weight &w) {
    constexpr bool f32 = sizeof(T) == 4;
    if (m > (f32 ? 8 : 16) || few_beside(w) > FEW_BESIDE) return false;
    constexpr float us[3][3] = {{2.4e-3f, 1.3e-3f, 0.9e-3f}, {2.6e-3f, 1.6e-3f, 1.2e-3f}, {2.8e-3f, 1.7e-3f, 1.5e-3f}};
    const float each = us[f32 ? 2 : m > 8][w.group == 32 ? 0 : w.group == 64 ? 1 : 2];
    const float waves = !f32 && m <= 8 ? std::max(1.f, 1.1f / (FEW_OUT * 152) * w.o) : (float)((w.o + FEW_OUT * 152 - 1) / (FEW_OUT * 152));
    return 2.5f + each * w.k * waves < linear4_tc_us<T>(w);
}

// The bf16 nearest to span / n (ties to even), span = hi + lo exactly, n = 7 or 15, span >= 0. The fp32 product may sit on the
// other side of a bf16 value or of the midpoint of two than the quotient; n times the midpoint above the lower one is exact, so the
// comparison is made there, and either neighbour leads to the right one.
__device__ __forceinline__ float scale_of(float hi, float lo, float n) {
    const float q = hi * (n == 7.f ? 1.f / 7.f : 1.f / 15.f);
    const unsigned below = __float_as_uint(q) & 0xFFFF0000u;
    const float mid = __uint_as_float(below | 0x8000u);
    const float over = fmaf(-n, mid, hi) + lo;
    const float s = __uint_as_float(below + (over > 0.f || (over == 0.f && (below & 0x10000u)) ? 0x10000u : 0u));
    return s >= 0x1p-126f ? s : 0.f;                    // 1 / s is finite
}

// 1 / s to an ulp, s normal and below 2^126.
__device__ __forceinline__ float reciprocal(float s) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    return r;
}

// w / s to the nearest integer, ties to even, |w / s| <= 16, inv about 1 / s, half = s / 2 (0, infinity: 0 for every w). The
// residual w - q s is exact, so it shows where the rounded product w (1 / s) fell on the wrong side of a border. Adding 1.5 * 2^23
// rounds to an integer whose lowest bit is the sum's.
__device__ __forceinline__ float nearest(float w, float s, float inv, float half) {
    constexpr float MAGIC = 12582912.f;
    const float t = fmaf(w, inv, MAGIC), q = t - MAGIC;
    const float r = fmaf(-q, s, w);
    const bool off = fabsf(r) > half || (fabsf(r) == half && (__float_as_uint(t) & 1u));
    return off ? q + copysignf(1.f, r) : q;
}

// The same for a w of bf16 (and s always is): 2 w and an odd multiple of s are whole multiples of a power of two, so w / s is
// half an integer or at least 2^-11 away from it, and rounding w (1 / s) to multiples of 2^-11 first tells which.
__device__ __forceinline__ float nearest_bf16(float w, float inv) {
    constexpr float MAGIC = 12582912.f, FINE = 6144.f;          // 1.5 * 2^23, 1.5 * 2^12
    return (fmaf(w, inv, FINE) - FINE) + MAGIC - MAGIC;
}

__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
    const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p + 4));
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16 *p, float (&v)[8]) {
    const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p));
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<float4 *>(p + 4), make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void store8(bf16 *p, const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    __stcs(reinterpret_cast<uint4 *>(p), make_uint4(u[0], u[1], u[2], u[3]));
}

// Codes of a matrix: 8 consecutive elements a lane, 4, 8 or 16 lanes a group, so a warp has runs of 256 elements of a
// row and reads, and writes codes and values, in whole lines. Each value is read once; what bounds it is memory: 32000 x 5120 fp32 with
// zeros and values take 205 us, 6.9 TB/s; 4096 x 4096 bf16 15.7 us, of them 13 the kernel's (issue slots 75% busy).
constexpr int Q_THREADS = 256, Q_RUN = 256;
template <typename T, int GROUP, bool ZEROS>
__global__ void __launch_bounds__(Q_THREADS)
quantize4_kernel(const T *__restrict__ x, long ldw, Weight w, T *__restrict__ values, long ldv, int runs) {
    constexpr int LANES = GROUP / 8, U = sizeof(T) == 2 ? 4 : 2;            // U runs in flight a warp
    wait_prior();
    allow_dependents();
    const int lane = threadIdx.x & 31;
    const unsigned t = blockIdx.x * (Q_THREADS / 32) + (threadIdx.x >> 5);
    const int j = (int)(t / (unsigned)runs), k0 = (int)(t - (unsigned)j * (unsigned)runs) * (U * Q_RUN) + lane * 8;
    if (j >= w.o) return;
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (k0 + u * Q_RUN < w.k) {
            load8(x + (long)j * ldw + k0 + u * Q_RUN, v[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float lo = 0.f, hi = 0.f;                           // (fminf and fmaxf leave NaN out)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (ZEROS) {
                lo = fminf(lo, v[u][i]);
                hi = fmaxf(hi, v[u][i]);
            } else {
                hi = fmaxf(hi, fabsf(v[u][i]));
            }
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) {
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            if (ZEROS) lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        }
        float s, z = 8.f;
        if (ZEROS) {
            const float d = hi - lo, b = d - hi;            // d + its rounding error = hi - lo
            s = scale_of(d, (hi - (d - b)) + (-lo - b), 15.f);
            z = s > 0.f ? fminf(fmaxf(nearest(-lo, s, reciprocal(s), 0.5f * s), 0.f), 15.f) : 0.f;
        } else {
            s = scale_of(hi, 0.f, 7.f);
        }
        const int k = k0 + u * Q_RUN;
        if (k >= w.k) continue;
        const long g = (long)j * w.groups + k / GROUP;
        if ((lane & (LANES - 1)) == 0) {
            w.scales[g] = __float2bfloat16(s);
            if (ZEROS) w.zeros[g] = (uint8_t)z;
        }
        const float inv = s > 0.f ? reciprocal(s) : 0.f, half = s > 0.f ? 0.5f * s : INFINITY;
        uint32_t word = 0;
        float back[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = v[u][i] == v[u][i] ? v[u][i] : 0.f;
            float q = (sizeof(T) == 2 ? nearest_bf16(c, inv) : nearest(c, s, inv, half)) + z;
            if (ZEROS) q = fminf(q, 15.f);                  // (7.03 steps at most without zeros, none below the zero with them)
            word |= (__float_as_uint(q + 12582912.f) & 15u) << (4 * i);
            back[i] = s * (q - z);
        }
        reinterpret_cast<uint32_t *>(w.codes)[(long)j * (w.k / 8) + k / 8] = word;
        if (values) store8(values + (long)j * ldv + k, back);
    }
}

template <typename T, int GROUP>
static cudaError_t launch_quantize(const T *x, long ldw, const Weight &w, T *values, long ldv, cudaStream_t s) {
    constexpr int U = sizeof(T) == 2 ? 4 : 2;
    const int runs = (w.k + U * Q_RUN - 1) / (U * Q_RUN);
    const long ctas = ((long)w.o * runs + Q_THREADS / 32 - 1) / (Q_THREADS / 32);
    if (ctas * (Q_THREADS / 32) > 0x7FFFFFFF) return cudaErrorInvalidValue;
    const cudaError_t e = w.zeros ? launch_chain(quantize4_kernel<T, GROUP, true>, (unsigned)ctas, Q_THREADS, 0, s, x, ldw, w, values, ldv, runs)
                                  : launch_chain(quantize4_kernel<T, GROUP, false>, (unsigned)ctas, Q_THREADS, 0, s, x, ldw, w, values, ldv, runs);
    note_launch();
    return e;
}

constexpr int MOST_ROWS = 65535 * 32;           // a grid's height in tiles of 32
constexpr int MOST_SIZE = 1 << 30;              // of o and k: they are rounded up to groups, chunks and tiles in 32 bits

static bool take_weight(const msd_weight4 *w, Weight *out) {
    if (!w || !w->codes || !w->scales || w->o < 1 || w->o > MOST_SIZE || w->k < 8 || w->k > MOST_SIZE || w->k % 8 ||
        reinterpret_cast<uintptr_t>(w->codes) % 4 || reinterpret_cast<uintptr_t>(w->scales) % 2 || (w->group != 32 && w->group != 64 && w->group != 128))
        return false;
    *out = Weight{w->codes, static_cast<bf16 *>(w->scales), w->zeros, w->o, w->k, w->group, (w->k + w->group - 1) / w->group};
    return true;
}

static bool bad_rows(const void *p, long ld, int dtype, int width) {
    const int size = dtype == MSD_F32 ? 4 : 2;
    return !p || ld < width || reinterpret_cast<uintptr_t>(p) % 16 || ld * size % 16;
}

static msd_status linear4(const void *x, long ldx, int x_dtype, int m, const msd_weight4 *weight, float *y, long ldy, int accumulate,
                          void *stream, int stall) {
    Weight w;
    if (m < 0 || m > MOST_ROWS || !take_weight(weight, &w) || (x_dtype != MSD_F32 && x_dtype != MSD_BF16)) return MSD_ERR_INVALID;
    if (m == 0) return MSD_OK;
    if (bad_rows(x, ldx, x_dtype, w.k) || !y || ldy < w.o || reinterpret_cast<uintptr_t>(y) % 4) return MSD_ERR_INVALID;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const auto run = [&](auto *p) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(p)>>;
        if (stall == NO_STALL && few_rows<T>(m, w)) return launch_few(p, ldx, m, w, y, ldy, accumulate, s);
        return launch_linear4_tc(p, ldx, m, w, y, ldy, accumulate, s, stall);
    };
    const cudaError_t e = x_dtype == MSD_F32 ? run(static_cast<const float *>(x)) : run(static_cast<const bf16 *>(x));
    return e == cudaSuccess ? MSD_OK : MSD_ERR_CUDA;
}

}  // namespace msd

using namespace msd;

extern "C" {

msd_status msd_linear4(const void *x, int64_t ldx, int32_t x_dtype, int32_t m, const msd_weight4 *weight, float *y,
                       int64_t ldy, int32_t accumulate, void *stream) {
    return linear4(x, ldx, x_dtype, m, weight, y, ldy, accumulate, stream, NO_STALL);
}

msd_status msd_test_linear4_timeout(const void *x, int64_t ldx, int32_t x_dtype, int32_t m, const msd_weight4 *weight, float *y,
                                    int64_t ldy, int32_t chunk, void *stream) {
    if (chunk < 0 || chunk == NO_STALL || !weight || reinterpret_cast<uintptr_t>(weight->codes) % 16 || weight->k % 32) return MSD_ERR_INVALID;
    return linear4(x, ldx, x_dtype, m, weight, y, ldy, 0, stream, chunk);
}

msd_status msd_test_linear4_shape(int32_t x_dtype, int32_t m, const msd_weight4 *weight, msd_linear4_shape *out) {
    Weight w;
    if (m < 1 || m > MOST_ROWS || !take_weight(weight, &w) || (x_dtype != MSD_F32 && x_dtype != MSD_BF16) || !out) return MSD_ERR_INVALID;
    const auto shape = [&](auto v) {
        using T = decltype(v);
        const bool few = few_rows<T>(m, w);
        const Linear4Shape c = few ? few_shape(m, w) : linear4_tc_shape<T>(m, w);
        *out = msd_linear4_shape{few, c.rows, c.outputs, c.split, c.staged, c.direct, (int32_t)c.smem};
    };
    x_dtype == MSD_F32 ? shape(float()) : shape(bf16());
    return MSD_OK;
}

msd_status msd_quantize4(const void *x, int64_t ldw, int32_t dtype, const msd_weight4 *out, void *values, int64_t ldv,
                         void *stream) {
    Weight w;
    if (!take_weight(out, &w) || (dtype != MSD_F32 && dtype != MSD_BF16) || bad_rows(x, ldw, dtype, w.k) ||
        (values && bad_rows(values, ldv, dtype, w.k)))
        return MSD_ERR_INVALID;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const auto run = [&](auto *from, auto *to) {
        return w.group == 128  ? launch_quantize<std::remove_pointer_t<decltype(to)>, 128>(from, (long)ldw, w, to, (long)ldv, s)
               : w.group == 64 ? launch_quantize<std::remove_pointer_t<decltype(to)>, 64>(from, (long)ldw, w, to, (long)ldv, s)
                               : launch_quantize<std::remove_pointer_t<decltype(to)>, 32>(from, (long)ldw, w, to, (long)ldv, s);
    };
    const cudaError_t e = dtype == MSD_F32 ? run(static_cast<const float *>(x), static_cast<float *>(values))
                                           : run(static_cast<const bf16 *>(x), static_cast<bf16 *>(values));
    return e == cudaSuccess ? MSD_OK : MSD_ERR_CUDA;
}

}  // extern "C"
