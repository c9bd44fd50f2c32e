// Products with weights in 4 bits on the 5th-generation tensor cores.
//
// y = x W^T with W's rows as the M side: codes come by tensor copies (128 rows of 64 bytes), a
// thread turns its row's codes into bf16 differences code - zero (exact) and puts them into tensor
// memory as the A operand; x is the B operand, staged in shared memory once for 256 outputs. An
// accumulator takes one group's products, and a group's sum is scaled on its way from tensor
// memory into the thread's fp32 totals, so no weight is rounded: what is done per code is 11
// integer and bf16 operations for 8 codes, one fused multiply per row of x for each group, and
// nothing in the tensor cores that another form would save.
//
// A CTA (448 threads, one an SM: it holds all of the tensor memory) has 256 outputs, two groups of
// four warps with 128 each, and up to N rows of x; K is cut between the CTAs of a cluster where
// there are fewer tiles than SMs, and their totals meet through distributed shared memory in rank
// order. Roles:
//   warps 0-7    a row of W a thread: codes -> tensor memory, and the chunk before: sums -> totals
//   warps 8-11   x of a chunk of 128 elements, swizzled as the MMA reads it, a chunk a warp
//   warp 12      MMAs       warp 13      copies of codes
// The codes of a word go in as the pairs (0, 4), (1, 5), (2, 6), (3, 7), so x's octets are ordered
// alike. A wait that runs out (2 s) leaves NaN in the CTA's part of y.
#include <algorithm>
#include <cstring>

#include <cudaTypedefs.h>

#include "linear4.cuh"
#include "tcgen05.cuh"

namespace msd {
namespace {

constexpr int THREADS = 448, TILE = 128, CHUNK = 128, OUT = 256, X_WARPS = 4;
constexpr uint32_t WBOX = TILE * CHUNK / 2, WSTAGE = 2 * WBOX;
constexpr uint32_t SMEM_MOST = 227 * 1024 - 2048;               // less static shared memory

template <typename T, int GROUP, int N>
struct Lay {
    static constexpr int P = Octet<T>::PLANES, PER = CHUNK / GROUP;
    static constexpr uint32_t XBOX = N * 128, XPLANE = 2 * XBOX, XSTAGE = P * XPLANE;
    static constexpr int XS = XSTAGE > 24 * 1024 ? 2 : 4;
    static constexpr int WS = XSTAGE > 24 * 1024 ? 5 : 6;
    static constexpr int DS = 128 / N;                          // accumulators of a group of warps
    static constexpr uint32_t X = 0, W = XS * XSTAGE, SCALES = W + WS * WSTAGE;
    static constexpr uint32_t ROOM = SMEM_MOST - 1024 - SCALES; // for scales and zeros
    static constexpr uint32_t T_A = 0, T_D = 128, T_HALF = 256; // columns of a group of warps
    static_assert(N * OUT * 4 <= SCALES, "totals of a CTA fit where the stages were");
    static_assert(SCALES + 1024 <= SMEM_MOST, "");
};

struct Args {
    Weight w;
    const void *x;
    long ldx, ldy;
    float *y;
    int m, accumulate, split, staged, slice;                    // slice: groups of a CTA that are staged
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float peer_value(uint32_t local, int rank) {
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts16(uint32_t a, const uint32_t *v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}

template <typename T, int GROUP, int N>
__global__ void __launch_bounds__(THREADS, 1)
linear4_tc_kernel(const __grid_constant__ CUtensorMap map, const Args a) {
    using L = Lay<T, GROUP, N>;
    constexpr int PER = L::PER, P = L::P, XS = L::XS, WS = L::WS, DS = L::DS;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * WS + 2 * XS + 8 + 4 * DS];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    const uint32_t base = (su32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const smem = smem_raw + (base - su32(smem_raw));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t w_full = su32(bars), w_empty = w_full + 8 * WS, x_full = w_empty + 8 * WS, x_empty = x_full + 8 * XS,
                   a_full = x_empty + 8 * XS, a_empty = a_full + 32, d_full = a_empty + 32, d_empty = d_full + 16 * DS;
    const int rank = (int)(blockIdx.x % a.split), tile = (int)(blockIdx.x / a.split);
    const int j0 = tile * OUT, i0 = (int)blockIdx.y * N, rows = min(N, a.m - i0);
    const int chunks = (a.w.k + CHUNK - 1) / CHUNK;
    const int c0 = (int)((long)chunks * rank / a.split), nc = (int)((long)chunks * (rank + 1) / a.split) - c0;
    if (tid == 0) {
        for (int i = 0; i < WS; ++i) {
            bar_init(w_full + 8 * i, 1);
            bar_init(w_empty + 8 * i, 8);
        }
        for (int i = 0; i < XS; ++i) {
            bar_init(x_full + 8 * i, 1);
            bar_init(x_empty + 8 * i, 1);
        }
        for (int i = 0; i < 4; ++i) {
            bar_init(a_full + 8 * i, 128);
            bar_init(a_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2 * DS; ++i) {
            bar_init(d_full + 8 * i, 1);
            bar_init(d_empty + 8 * i, 128);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_abort = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(&s_tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = s_tmem;
    wait_prior();
    allow_dependents();

    float total[N];
    if (warp < 8) {
        // ---- codes to tensor memory, sums to totals --------------------------------------------
#pragma unroll
        for (int i = 0; i < N; ++i) total[i] = 0.f;
        const int half = warp >> 2, row = (warp & 3) * 32 + lane, out = half * TILE + row;
        const int spitch = OUT + 2, zpitch = OUT + 4;
        bf16 *const s_scales = reinterpret_cast<bf16 *>(smem + L::SCALES);
        uint8_t *const s_zeros = smem + L::SCALES + (size_t)a.slice * spitch * 2;
        const int g0 = c0 * PER, gs = min(nc * PER, a.w.groups - g0), outs = min(OUT, a.w.o - j0);
        if (a.staged) {
            const unsigned magic = 0xFFFFFFFFu / (unsigned)gs + 1;          // i / gs for i * gs < 2^32; gs 1: 0
            for (int i = tid; i < outs * gs; i += 256) {
                const int r = gs > 1 ? (int)__umulhi((unsigned)i, magic) : i, g = i - r * gs;
                const long at = (long)(j0 + r) * a.w.groups + g0 + g;
                s_scales[g * spitch + r] = a.w.scales[at];
                if (a.w.zeros) s_zeros[g * zpitch + r] = a.w.zeros[at];
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
        }
        const long wide_at = (long)(j0 + min(out, outs - 1)) * a.w.groups + g0;
        auto scale_at = [&](int g) {
            if (g >= gs || out >= outs) return 0.f;
            return __bfloat162float(a.staged ? s_scales[g * spitch + out] : a.w.scales[wide_at + g]);
        };
        auto zero_at = [&](int g) {
            if (!a.w.zeros || g >= gs || out >= outs) return 8u;
            return (unsigned)(a.staged ? s_zeros[g * zpitch + out] : a.w.zeros[wide_at + g]);
        };
        const uint32_t t_a = tmem + ((uint32_t)(warp & 3) << 21) + half * L::T_HALF + L::T_A;
        const uint32_t t_d = tmem + ((uint32_t)(warp & 3) << 21) + half * L::T_HALF + L::T_D;
        const uint32_t code_row = base + L::W + half * WBOX + row * 64;
        const uint32_t swz = (uint32_t)(row >> 1 & 3) << 4;
        bool ok = true;
        auto promote = [&](int ci) {
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const int gi = ci * PER + e, ds = gi % DS;
                const float s = scale_at(gi);
                ok = w_wait(d_full + 8 * (half * DS + ds), (uint32_t)(gi / DS) & 1u, &s_abort, nullptr);
                if (!ok) return;
                fence_after();
                constexpr int STEP = N < 32 ? N : 32;
                uint32_t d[N];
#pragma unroll
                for (int i = 0; i < N; i += STEP) {
                    if constexpr (STEP == 16) tmem_ld16(t_d + ds * N + i, d + i);
                    else tmem_ld32(t_d + ds * N + i, d + i);
                }
                fence_before();
                bar_arrive(d_empty + 8 * (half * DS + ds));
#pragma unroll
                for (int i = 0; i < N; ++i) total[i] = fmaf(s, __uint_as_float(d[i]), total[i]);
            }
        };
        for (int ci = 0; ci < nc && ok; ++ci) {
            const int ws = ci % WS, slot = ci & 1;
            ok = w_wait(w_full + 8 * ws, (uint32_t)(ci / WS) & 1u, &s_abort, nullptr);
            if (!ok) break;
            uint4 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = lds16(code_row + ws * WSTAGE + ((i << 4) ^ swz));
            __syncwarp();
            if (lane == 0) bar_arrive(w_empty + 8 * ws);
            ok = w_wait(a_empty + 8 * (half * 2 + slot), ((uint32_t)(ci >> 1) & 1u) ^ 1u, &s_abort, nullptr);
            if (!ok) break;
            fence_after();
#pragma unroll
            for (int h = 0; h < 2; ++h) {                       // 64 elements: 32 columns
                uint32_t p[32];
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const int word = 8 * h + v;
                    const unsigned z = 0x4300u + zero_at(ci * PER + word * 8 / GROUP);
                    const uint32_t both = z | z << 16;
                    const uint4 &f = q[word >> 2];
                    const uint32_t c = (word & 3) == 0 ? f.x : (word & 3) == 1 ? f.y : (word & 3) == 2 ? f.z : f.w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[4 * v + i] = pair_of(c >> (4 * i), *reinterpret_cast<const __nv_bfloat162 *>(&both));
                }
                tmem_st32(t_a + slot * 64 + 32 * h, p);
            }
            fence_before();
            bar_arrive(a_full + 8 * (half * 2 + slot));
            if (ci > 0) promote(ci - 1);
        }
        if (ok) promote(nc - 1);
        if (!ok || s_abort)
#pragma unroll
            for (int i = 0; i < N; ++i) total[i] = NAN;
    } else if (warp < 8 + X_WARPS) {
        // ---- rows of x --------------------------------------------------------------------------
        const T *const x = static_cast<const T *>(a.x) + (long)i0 * a.ldx;
        for (int ci = warp - 8; ci < nc && warp - 8 < XS; ci += XS) {
            const int slot = ci % XS;
            if (!w_wait(x_empty + 8 * slot, ((uint32_t)(ci / XS) & 1u) ^ 1u, &s_abort, nullptr)) break;
            const uint32_t to = base + L::X + slot * L::XSTAGE;
            const int k0 = (c0 + ci) * CHUNK;
            constexpr int BATCH = N / 2 < 8 ? N / 2 : 8;
            for (int b = 0; b < N / 2; b += BATCH) {
                Octet<T> o[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int n = ((b + i) * 32 + lane) >> 4, at = k0 + (lane & 15) * 8;
                    if (n < rows && at < a.w.k) o[i].load(x + (long)n * a.ldx + at); else o[i].clear();
                }
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int n = ((b + i) * 32 + lane) >> 4, c = lane & 15;
                    uint32_t v[P][4];
                    o[i].pairs(v);
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        sts16(to + p * L::XPLANE + (c >> 3) * L::XBOX + n * 128 + (((c & 7) ^ (n & 7)) << 4), v[p]);
                }
            }
            fence_proxy();
            __syncwarp();
            if (lane == 0) bar_arrive(x_full + 8 * slot);
        }
    } else if (warp == 12) {
        // ---- MMAs ---------------------------------------------------------------------------------
        const uint32_t on = elect_one(), id = idesc(TILE, N, 0);
        bool ok = true;
        for (int ci = 0; ci < nc && ok; ++ci) {
            const int xs = ci % XS, slot = ci & 1;
            ok = w_wait(x_full + 8 * xs, (uint32_t)(ci / XS) & 1u, &s_abort, nullptr);
            const uint64_t d_x = sdesc(base + L::X + xs * L::XSTAGE, 16, 1024);
            for (int half = 0; half < 2 && ok; ++half) {
                ok = w_wait(a_full + 8 * (half * 2 + slot), (uint32_t)(ci >> 1) & 1u, &s_abort, nullptr);
                const uint32_t t = tmem + half * L::T_HALF;
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    const int gi = ci * PER + e, ds = gi % DS;
                    if (ok) ok = w_wait(d_empty + 8 * (half * DS + ds), ((uint32_t)(gi / DS) & 1u) ^ 1u, &s_abort, nullptr);
                    if (!ok) break;
                    fence_after();
#pragma unroll
                    for (int kk = 0; kk < GROUP / 16; ++kk) {
                        const int k16 = e * (GROUP / 16) + kk;
#pragma unroll
                        for (int p = 0; p < P; ++p)
                            w_mma_ts(on, t + L::T_D + ds * N, t + L::T_A + slot * 64 + k16 * 8,
                                     d_x + ((p * L::XPLANE + (k16 >> 2) * L::XBOX + (k16 & 3) * 32) >> 4), id, kk > 0 || p > 0);
                    }
                    w_commit(on, d_full + 8 * (half * DS + ds));
                }
                if (ok) w_commit(on, a_empty + 8 * (half * 2 + slot));
            }
            if (ok) w_commit(on, x_empty + 8 * xs);
        }
        __syncwarp();
    } else {
        // ---- copies of codes ---------------------------------------------------------------------
        const uint32_t on = elect_one();
        int filled = 0;
        for (; filled < nc; ++filled) {
            const int ws = filled % WS;
            if (!w_wait(w_empty + 8 * ws, ((uint32_t)(filled / WS) & 1u) ^ 1u, &s_abort, nullptr)) break;
            const uint32_t to = base + L::W + ws * WSTAGE;
            w_expect_tx(on, w_full + 8 * ws, WSTAGE);
            w_tma2d(on, to, &map, (c0 + filled) * (CHUNK / 2), j0, w_full + 8 * ws);
            w_tma2d(on, to + WBOX, &map, (c0 + filled) * (CHUNK / 2), j0 + TILE, w_full + 8 * ws);
        }
        if (s_abort) {                                          // copies in flight land before the CTA goes on
            volatile int never = 0;
            for (int i = max(filled - WS, 0); i < filled; ++i) bar_wait_slow(w_full + 8 * (i % WS), (uint32_t)(i / WS) & 1u, &never, nullptr);
        }
        __syncwarp();
    }
    fence_before();
    __syncthreads();
    if (warp == 12) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }

    float *const y = a.y + (long)i0 * a.ldy;
    if (a.split == 1) {
        const int j = j0 + warp * 32 + lane;
        if (warp < 8 && j < a.w.o) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i < rows) {
                    float *at = y + (long)i * a.ldy + j;
                    *at = a.accumulate ? *at + total[i] : total[i];
                }
            }
        }
        return;
    }
    float *const buf = reinterpret_cast<float *>(smem);         // [N][OUT]
    if (warp < 8)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[i * OUT + tid] = total[i];
    cluster_sync();
    if (warp < 8) {
        const int j = j0 + tid;
        for (int i = rank; i < rows; i += a.split) {
            float v = 0.f;
            for (int r = 0; r < a.split; ++r) v += peer_value(base + (i * OUT + tid) * 4, r);
            if (j < a.w.o) {
                float *at = y + (long)i * a.ldy + j;
                *at = a.accumulate ? *at + v : v;
            }
        }
    }
    cluster_sync();
}

bool code_map(const Weight &w, CUtensorMap *map) {
    static PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
        cudaDriverEntryPointQueryResult q;
        void *fn = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            fn = nullptr;
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }();
    if (!encode) return false;
    memset(map, 0, sizeof *map);
    const cuuint64_t dims[2] = {(cuuint64_t)w.k / 2, (cuuint64_t)w.o};
    const cuuint64_t strides[1] = {(cuuint64_t)w.k / 2};
    const cuuint32_t box[2] = {CHUNK / 2, TILE};
    const cuuint32_t estr[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, w.codes, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int GROUP, int N>
cudaError_t launch(const CUtensorMap &map, Args a, cudaStream_t s) {
    using L = Lay<T, GROUP, N>;
    const int chunks = (a.w.k + CHUNK - 1) / CHUNK, tiles = (a.w.o + OUT - 1) / OUT, cols = (a.m + N - 1) / N;
    a.split = std::max(1, std::min({8, chunks, 152 / std::max(1, tiles * cols)}));
    const int slice = (chunks + a.split - 1) / a.split * L::PER;
    const size_t beside = (size_t)slice * ((OUT + 2) * 2 + (a.w.zeros ? OUT + 4 : 0));
    a.staged = beside <= L::ROOM;
    a.slice = a.staged ? slice : 0;
    const size_t smem = std::max<size_t>(L::SCALES + 1024 + (a.staged ? beside : 0), tmem_smem_floor(512));
    cudaError_t e = cudaFuncSetAttribute(linear4_tc_kernel<T, GROUP, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_MOST);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(tiles * a.split, cols);
    lc.blockDim = THREADS;
    lc.dynamicSmemBytes = smem;
    lc.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = a.split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = programmatic(s) ? 2 : 1;
    e = cudaLaunchKernelEx(&lc, linear4_tc_kernel<T, GROUP, N>, map, a);
    note_launch();
    return e;
}

template <typename T, int GROUP>
cudaError_t launch_n(const CUtensorMap &map, const Args &a, cudaStream_t s) {
    return a.m <= 16 ? launch<T, GROUP, 16>(map, a, s) : a.m <= 32 ? launch<T, GROUP, 32>(map, a, s) : launch<T, GROUP, 64>(map, a, s);
}

}  // namespace

template <typename T>
cudaError_t launch_linear4_tc(const T *x, long ldx, int m, const Weight &w, float *y, long ldy, int accumulate, cudaStream_t s) {
    CUtensorMap map;
    if (!code_map(w, &map)) return cudaErrorUnknown;
    const Args a{w, x, ldx, ldy, y, m, accumulate, 1, 0, 0};
    return w.group == 128 ? launch_n<T, 128>(map, a, s) : w.group == 64 ? launch_n<T, 64>(map, a, s) : launch_n<T, 32>(map, a, s);
}

template cudaError_t launch_linear4_tc<float>(const float *, long, int, const Weight &, float *, long, int, cudaStream_t);
template cudaError_t launch_linear4_tc<bf16>(const bf16 *, long, int, const Weight &, float *, long, int, cudaStream_t);

}  // namespace msd
