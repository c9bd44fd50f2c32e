// Products with weights in 4 bits on the 5th-generation tensor cores.
//
// y = x W^T with W's rows as the M side: codes come by tensor copies (128 rows of 64 bytes), a
// thread turns its row's codes into bf16 differences code - zero (exact) and puts them into tensor
// memory as the A operand; x is the B operand, staged in shared memory. An accumulator takes one
// group's products, and a group's sum is scaled on its way from tensor memory into the thread's
// fp32 totals, so no weight is rounded.
//
// A CTA (one an SM: it holds all of the tensor memory) has 256 outputs, two halves of 128, and up to 64 rows of x, or 128
// outputs and up to 128 rows; K is cut between the CTAs of a cluster where there are fewer tiles than SMs, and their totals meet
// through distributed shared memory in rank order. Chunks are 128 elements of K. Roles:
//   warps 0-3    MMAs, of the even or the odd chunks (of a half; first, since a scheduler prefers them: as the last warps, an
//                MMA's issue took them 100 cycles)
//   warps 4-7    x: copies of bf16, put into order where need be; fp32 as three bf16 planes that add up to it, swizzled as the MMA
//                reads them
//   warps 8-15   a row of W a thread: a group's sum from tensor memory, scaled, into fp32 totals (of half the rows of x, with 128
//                outputs)
//   warps 16-31  a row of W a thread: codes -> tensor memory; four warps for the even chunks of a half and four for the odd ones, or
//                four for every fourth chunk; the first of the four also issue the copies of codes, four chunks ahead
// For 8 codes, in the order of a word's shifts ((0, 4), (1, 5), (2, 6), (3, 7), x ordered alike), the integer pipe, half a warp a
// cycle, takes 3 shifts, 4 selections and 4 subtractions: 704 cycles for a chunk of 256 outputs, against 512 of the MMAs of 64 rows and
// 330 of a copy at the rate of memory. With 128 rows to a CTA x stays as copied (ordering 128 rows took the four copying warps
// longer than a chunk) and codes come out in their own order, for 2 more operations of 8 codes.
//
// What bounds it (clocks around the roles' waits in a scratch build, which itself takes 5 to 10% longer): no pipe alone, the integer one
// is busy 37 to 54% and issue 50 to 65% of the time.
//   groups of 128   60 rows, 256 outputs: 1350 cycles a chunk, the code warps busy 84% of them, MMAs waiting for x 28, codes 25 and
//                   accumulators 19%. 128 rows and outputs: 900, 512 of them MMAs; the code warps wait 40% for their buffer, the sum warps
//                   51% for sums. 16 rows, 128 outputs: 720; a code warp waits 27% for its buffer, the sum warps 65%
//   groups of 64, 32   MMAs wait for accumulators that the sum warps have not read: 66 and 78% of the time with 128 rows (1550 and 2300
//                   cycles a chunk of 128 outputs), 75% with 64 (groups of 32)
//   fp32, 32 rows   MMAs wait for x 64% of the time (groups of 128, 2600 cycles for 256 outputs): the copying warps split it in planes
// To start and to end a CTA takes about 4 us, to join 2 to 3.5. One group of warps a half doing everything in turn took 1800 cycles
// a chunk. Measured, us (groups of 128, other weights for each call): k 4096, o 11008: 16 rows 13.5, 60 rows 16.7, 128 rows 22, 645
// rows 84 (690 TFLOP/s); k 11008, o 4096, 60 rows 18.2. A wait that runs out (2 s) leaves NaN in the CTA's part of y.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include <cudaTypedefs.h>

#include "linear4.cuh"
#include "tcgen05.cuh"

namespace msd {
namespace {

constexpr int TILE = 128, CHUNK = 128;
constexpr uint32_t WBOX = TILE * CHUNK / 2;
constexpr uint32_t SMEM_MOST = 227 * 1024 - 2048;               // less static shared memory
constexpr int CODE_WARPS = 16, SUM_WARPS = 8, THREADS = 1024;
constexpr int AHEAD = 4;                                        // chunks (a multiple of a cycle, and less than a ring has stages)
constexpr int COPY_0 = 4, SUM_0 = 8, CODE_0 = SUM_0 + SUM_WARPS;                   // first warps of the roles

template <typename T, int GROUP, int N, int OUTPUTS>
struct Lay {
    static constexpr bool SPLIT = sizeof(T) == 4;               // x in planes
    // 256 outputs, two halves; or HALF of that: the four groups of code warps take every fourth chunk, the two of sum warps half of the
    // rows of x
    static constexpr bool HALF = OUTPUTS == TILE;
    static constexpr int OUT = OUTPUTS, CYCLE = HALF ? 4 : 2, TOK = HALF ? N / 2 : N;
    static constexpr uint32_t WSTAGE = OUT / TILE * WBOX;
    static constexpr bool IN_ORDER = N > 64;                     // x as copied; else in the order of a word's shifts
    static constexpr int P = Octet<T>::PLANES, PER = CHUNK / GROUP;
    // registers by role: over the eight groups of four warps they are the launch's 64 a thread
    static constexpr int R_CODE = 56, R_SUM = SPLIT ? 96 : 104, R_ISSUE = 40, R_COPY = SPLIT ? 56 : 40;
    static_assert(4 * R_CODE + 2 * R_SUM + R_ISSUE + R_COPY <= 64 * 8, "");
    static constexpr uint32_t XBOX = N * 128, XPLANE = 2 * XBOX, XSTAGE = P * XPLANE;
    static constexpr int XS = SPLIT && N > 16 ? 2 : 4;          // even: a stage's chunks are all even or all odd ones
    static constexpr int X_PARTS = SPLIT ? 4 / XS : 1;          // warps that fill a stage of x
    static constexpr int WS = HALF ? 8 : 6;
    static constexpr int DS = (HALF ? 256 : 128) / N, HS = DS / 2;          // accumulators (of a half), of even or odd chunks
    static constexpr uint32_t X = 0, W = XS * XSTAGE, SCALES = W + WS * WSTAGE;
    static constexpr uint32_t ROOM = SMEM_MOST - 1024 - SCALES; // for scales and zeros
    static constexpr uint32_t T_A = 0, T_D = 128, T_HALF = 256; // columns of a half
    static_assert(N * OUT * 4 <= SCALES, "totals of a CTA fit where the stages were");
    static_assert(SCALES + 1024 <= SMEM_MOST, "");
};

struct Args {
    Weight w;
    const void *x;
    long ldx, ldy;
    float *y;
    int m, accumulate, split, staged, slice;                    // slice: groups of a CTA that are staged
    int direct;                                                 // codes at addresses that tensor copies do not take
    int stall;                                                  // chunks of K from this one on get no codes (a test's waits run out)
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

// Codes 2 i and 2 i + 1 of a word (byte i) less the zero, as a bf16 pair. The even one is put below 128, the odd one, from
// the word shifted by one bit, at the third bit below 16; off: 128 + zero and 16 + zero.
__device__ __forceinline__ uint32_t pair_in_order(uint32_t word, int i, __nv_bfloat162 off) {
    uint32_t v = __byte_perm(word, word >> 1, 0x0400 | i | i << 8);
    asm("lop3.b32 %0, %0, 0x0078000F, 0x41804300, 0xEA;" : "+r"(v));                     // (a & b) | c
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<__nv_bfloat162 *>(&v), off);
    return *reinterpret_cast<const uint32_t *>(&d);
}

// A warp waits for the barrier's use-th completion (in laps of `lap` uses). It sleeps in the barrier for up to 20 us at a time: what
// polls takes issue slots, and they are what the kernel runs out of.
__device__ __forceinline__ bool use_wait_slow(uint32_t bar, uint32_t parity, volatile int *abort) {
    const unsigned long long t0 = gtime();
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.b32 %0, 1, 0, p;\n}"
            : "=r"(ok)
            : "r"(bar), "r"(parity), "r"(20000u)
            : "memory");
        if (__all_sync(0xffffffffu, ok)) return true;
        if (__any_sync(0xffffffffu, *abort)) return false;
        if (__any_sync(0xffffffffu, gtime() - t0 > TIMEOUT_NS)) {
            *abort = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool use_wait(uint32_t bar, int use, int lap, volatile int *abort) {
    const uint32_t parity = (uint32_t)(use / lap) & 1u;
    return __all_sync(0xffffffffu, bar_try(bar, parity)) || use_wait_slow(bar, parity, abort);
}

template <typename T, int GROUP, int N, int OUTPUTS>
__global__ void __launch_bounds__(THREADS, 1)
linear4_tc_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap x_map, const Args a) {
    using L = Lay<T, GROUP, N, OUTPUTS>;
    constexpr int PER = L::PER, P = L::P, XS = L::XS, WS = L::WS, DS = L::DS, HS = L::HS, OUT = L::OUT, CYCLE = L::CYCLE;
    constexpr bool HALF = L::HALF;
    constexpr uint32_t WSTAGE = L::WSTAGE;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * WS + 3 * XS + 16 + 4 * DS + 4];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    const uint32_t base = (su32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const smem = smem_raw + (base - su32(smem_raw));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t w_full = su32(bars), w_empty = w_full + 8 * WS, x_full = w_empty + 8 * WS, x_empty = x_full + 8 * XS,
                   a_full = x_empty + 8 * XS, a_empty = a_full + 64, d_full = a_empty + 64, d_empty = d_full + 16 * DS, x_raw = d_empty + 16 * DS,
                   drained = x_raw + 8 * XS;
    const int rank = (int)(blockIdx.x % a.split), tile = (int)(blockIdx.x / a.split);
    const int j0 = tile * OUT, i0 = (int)blockIdx.y * N, rows = min(N, a.m - i0);
    const int chunks = (a.w.k + CHUNK - 1) / CHUNK;
    const int c0 = (int)((long)chunks * rank / a.split), nc = (int)((long)chunks * (rank + 1) / a.split) - c0;
    if (tid == 0) {
        for (int i = 0; i < WS; ++i) {
            bar_init(w_full + 8 * i, 1);
            bar_init(w_empty + 8 * i, HALF ? 4 : 8);
        }
        for (int i = 0; i < XS; ++i) {
            bar_init(x_full + 8 * i, L::X_PARTS);
            bar_init(x_empty + 8 * i, HALF ? 1 : 2);
            bar_init(x_raw + 8 * i, 1);
        }
        for (int i = 0; i < 8; ++i) {
            bar_init(a_full + 8 * i, 4);
            bar_init(a_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2 * DS; ++i) {
            bar_init(d_full + 8 * i, 1);
            bar_init(d_empty + 8 * i, HALF ? 8 : 4);
        }
        for (int i = 0; i < 4; ++i) bar_init(drained + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_abort = 0;
        if (!a.direct) asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
        if constexpr (!L::SPLIT) asm volatile("prefetch.tensormap [%0];" ::"l"(&x_map) : "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(&s_tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = s_tmem;
    wait_prior();
    allow_dependents();

    // scales and zeros [group][output], a run of outputs beside one another
    constexpr int SPITCH = OUT + 2, ZPITCH = OUT + 4;
    bf16 *const s_scales = reinterpret_cast<bf16 *>(smem + L::SCALES);
    uint8_t *const s_zeros = smem + L::SCALES + (size_t)a.slice * SPITCH * 2;
    const int g0 = c0 * PER, gs = min(nc * PER, a.w.groups - g0), outs = min(OUT, a.w.o - j0);
    const auto stage = [&](auto *to, const auto *from, int pitch, int t, int threads) {
        const unsigned magic = 0xFFFFFFFFu / (unsigned)gs + 1;          // i / gs for i * gs < 2^32; gs 1: 0
        constexpr int U = 8;                                            // loads in flight a thread
        for (int b = t; b < outs * gs; b += U * threads) {
            std::remove_reference_t<decltype(*to)> v[U];
            int at[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = min(b + u * threads, outs * gs - 1);
                const int r = gs > 1 ? (int)__umulhi((unsigned)i, magic) : i, g = i - r * gs;
                v[u] = from[(long)(j0 + r) * a.w.groups + g0 + g];
                at[u] = g * pitch + r;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) to[at[u]] = v[u];
        }
    };

    // every role ends here: stages, accumulators and codes are done with
    const auto done = [] { fence_before(); asm volatile("bar.sync 3, %0;" ::"n"(THREADS) : "memory"); };
    if (warp >= CODE_0) {
        // ---- codes to tensor memory ---------------------------------------------------------------
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::R_CODE));
        const int g = (warp - CODE_0) >> 2, half = HALF ? 0 : g >> 1, slot = g % CYCLE, row = (warp & 3) * 32 + lane, out = half * TILE + row;
        const uint32_t t_a = tmem + ((uint32_t)(warp & 3) << 21) + (g >> 1) * L::T_HALF + L::T_A + (g & 1) * 64;
        const uint32_t code_row = base + L::W + half * WBOX + row * 64, swz = (uint32_t)(row >> 1 & 3) << 4;
        const uint8_t *const z_at = a.staged ? s_zeros + out : a.w.zeros + (long)(j0 + min(out, outs - 1)) * a.w.groups + g0;
        const int z_step = a.staged ? ZPITCH : 1;
        const bool copies = !a.direct && (warp & 3) == 0 && g < CYCLE;                 // (a warp for each place in the cycle)
        const uint32_t on = elect_one();
        int copied = slot;                                      // chunks copied: slot, slot + CYCLE, ... below this
        const auto copy = [&](int ci) {
            const int ws = ci % WS;
            if (c0 + ci >= a.stall || !use_wait(w_empty + 8 * ws, ci + WS, WS, &s_abort)) return;
            const uint32_t to = base + L::W + ws * WSTAGE, bar = w_full + 8 * ws;
            w_expect_tx(on, bar, WSTAGE);
            w_tma2d(on, to, &map, (c0 + ci) * (CHUNK / 2), j0, bar);
            if constexpr (!HALF) w_tma2d(on, to + WBOX, &map, (c0 + ci) * (CHUNK / 2), j0 + TILE, bar);
            copied = ci + CYCLE;
        };
        if (copies)
            for (int ci = slot; ci < min(nc, AHEAD); ci += CYCLE) copy(ci);
        if (a.staged && a.w.zeros) {
            stage(s_zeros, a.w.zeros, ZPITCH, tid - CODE_0 * 32, CODE_WARPS * 32);
            asm volatile("bar.sync 1, 512;" ::: "memory");
        }
        bool ok = true;
        for (int ci = slot; ci < nc && ok; ci += CYCLE) {
            const int ws = ci % WS;
            if (copies && ci + AHEAD < nc) copy(ci + AHEAD);
            uint32_t from = code_row + ws * WSTAGE;
            if (a.direct) {                                     // the warp's 32 rows, two at a time, by words to where a copy would put them
                from = code_row + slot * WSTAGE;
                const int words = a.w.k / 8, at = (c0 + ci) * (CHUNK / 8) + (lane & 15), r0 = half * TILE + (warp & 3) * 32 + (lane >> 4);
                const uint32_t *const codes = reinterpret_cast<const uint32_t *>(a.w.codes) + at;
                __syncwarp();                                   // (the last chunk's have been read)
#pragma unroll 1
                for (int b = 0; b < 32; b += 16) {
                    uint32_t v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = at < words ? __ldcs(codes + (long)(j0 + min(r0 + b + 2 * i, outs - 1)) * words) : 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = (warp & 3) * 32 + (lane >> 4) + b + 2 * i;
                        const uint32_t to = base + L::W + slot * WSTAGE + half * WBOX + r * 64 + (((lane & 12) << 2) ^ ((r >> 1 & 3) << 4)) + (lane & 3) * 4;
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"(v[i]) : "memory");
                    }
                }
                __syncwarp();
            } else {
                ok = use_wait(w_full + 8 * ws, ci, WS, &s_abort);
                if (!ok) break;
            }
            uint4 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = lds16(from + ((i << 4) ^ swz));
            unsigned z[PER];
#pragma unroll
            for (int e = 0; e < PER; ++e) z[e] = a.w.zeros && ci * PER + e < gs ? z_at[(long)(ci * PER + e) * z_step] : 8u;
            __syncwarp();
            if (lane == 0 && !a.direct) bar_arrive(w_empty + 8 * ws);
            // 64 elements at a time, so that the MMAs of the first are done when the next chunk's come
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                const uint32_t bar = 8 * (g * 2 + sub);
                ok = ok && use_wait(a_empty + bar, ci + CYCLE, CYCLE, &s_abort);
                if (!ok) break;
                fence_after();
#pragma unroll
                for (int i = 2 * sub; i < 2 * sub + 2; ++i) {   // 32 elements: 16 columns
                    const uint32_t zero = z[i * 32 / GROUP], both = L::IN_ORDER ? 0x41804300u + zero * 0x00080001u : 0x43004300u + zero * 0x10001u;
                    const __nv_bfloat162 off = *reinterpret_cast<const __nv_bfloat162 *>(&both);
                    const uint32_t f[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
                    uint32_t p[16];
#pragma unroll
                    for (int c = 0; c < 16; ++c) p[c] = L::IN_ORDER ? pair_in_order(f[c >> 2], c & 3, off) : pair_of(f[c >> 2] >> (4 * (c & 3)), off);
                    tmem_st16(t_a + 16 * i, p);
                }
                tmem_st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(a_full + bar);
            }
        }
        if (copies && s_abort) {                                // copies in flight land before the CTA goes on
            volatile int never = 0;
            for (int ci = slot; ci < copied; ci += CYCLE)
                if (ci + WS >= copied) bar_wait_slow(w_full + 8 * (ci % WS), (uint32_t)(ci / WS) & 1u, &never, nullptr);
            __syncwarp();
        }
        done();
    } else if (warp >= SUM_0) {
        // ---- sums to totals -------------------------------------------------------------------------
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::R_SUM));
        const int half = (warp - SUM_0) >> 2, out = (tid - SUM_0 * 32) % OUT, tok0 = HALF ? half * L::TOK : 0;
        if (a.staged) {
            stage(s_scales, a.w.scales, SPITCH, tid - SUM_0 * 32, SUM_WARPS * 32);
            asm volatile("bar.sync 2, 256;" ::: "memory");
        }
        const bf16 *const s_at = a.staged ? s_scales + out : a.w.scales + (long)(j0 + min(out, outs - 1)) * a.w.groups + g0;
        const int s_step = a.staged ? SPITCH : 1;
        const uint32_t t_d = tmem + ((uint32_t)(warp & 3) << 21) + L::T_D + (HALF ? 0 : half * L::T_HALF);
        constexpr int TOK = L::TOK;
        float total[TOK];
#pragma unroll
        for (int i = 0; i < TOK; ++i) total[i] = 0.f;
        bool ok = true;
        for (int gi = 0; gi < nc * PER; ++gi) {
            const int ci = gi / PER, li = (ci >> 1) * PER + gi % PER, ds = (ci & 1) * HS + li % HS;
            const float s = gi < gs && out < outs ? __bfloat162float(s_at[(long)gi * s_step]) : 0.f;
            const uint32_t bar = 8 * (HALF ? ds : half * DS + ds), from = t_d + (HALF ? ds / HS * L::T_HALF + ds % HS * N + tok0 : ds * N);
            ok = use_wait(d_full + bar, li, HS, &s_abort);
            if (!ok) break;
            fence_after();
            constexpr int STEP = TOK < 16 ? TOK : 16;
#pragma unroll
            for (int i0 = 0; i0 < TOK; i0 += STEP) {
                uint32_t d[STEP];
                if constexpr (STEP == 16) tmem_ld16(from + i0, d); else tmem_ld8(from + i0, d);
                if (i0 + STEP == TOK) {
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(d_empty + bar);
                }
#pragma unroll
                for (int i = 0; i < STEP; ++i) total[i0 + i] = fmaf(s, __uint_as_float(d[i]), total[i0 + i]);
            }
        }
        if (!ok || s_abort)
#pragma unroll
            for (int i = 0; i < TOK; ++i) total[i] = NAN;
        done();
        const int j = j0 + out;
        if (a.split > 1) {
#pragma unroll
            for (int i = 0; i < TOK; ++i) reinterpret_cast<float *>(smem)[(tok0 + i) * OUT + out] = total[i];
        } else if (j < a.w.o) {
#pragma unroll
            for (int i = 0; i < TOK; ++i) {
                if (tok0 + i < rows) {
                    float *at = a.y + (long)(i0 + tok0 + i) * a.ldy + j;
                    *at = a.accumulate ? *at + total[i] : total[i];
                }
            }
        }
    } else if (warp < COPY_0) {
        // ---- MMAs ---------------------------------------------------------------------------------
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::R_ISSUE));
        const uint32_t on = elect_one();                        // (whole warps: addresses stay in uniform registers)
        // (HALF: warps 0 and 1, of the even and the odd chunks)
        const int half = HALF ? 0 : warp >> 1, slot = warp & 1;
        const uint32_t id = idesc(TILE, N, 0);
        bool ok = !HALF || warp < 2;
        for (int ci = slot; ci < nc && ok; ci += 2) {
            const int g = HALF ? ci & 3 : half * 2 + slot;
            const uint32_t t_a = tmem + (g >> 1) * L::T_HALF + L::T_A + (g & 1) * 64;
            const int xs = ci % XS;
            ok = use_wait(x_full + 8 * xs, ci, XS, &s_abort);
            const uint64_t d_x = sdesc(base + L::X + xs * L::XSTAGE, 16, 1024);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const int li = (ci >> 1) * PER + e, ds = slot * HS + li % HS;      // (no accumulator is shared by two warps' waits)
                const uint32_t d_bar = 8 * (HALF ? ds : half * DS + ds);
                const uint32_t t_d = tmem + L::T_D + (HALF ? ds / HS * L::T_HALF + ds % HS * N : half * L::T_HALF + ds * N);
                ok = ok && use_wait(d_empty + d_bar, li + HS, HS, &s_abort);
                if (!ok) break;
                fence_after();
                // (fp32's later planes first: a tensor core cuts a sum's last bits at each product added, and they are smaller. At groups
                // of 128 that makes errors 8e-8 of 4.4e-7, in 4% more time; at 32 they are 1.5e-7 plane after plane)
                constexpr bool LATER_FIRST = P > 1 && GROUP > 32;
#pragma unroll
                for (int part = LATER_FIRST ? 0 : 1; part < 2 && ok; ++part) {
#pragma unroll
                    for (int kk = 0; kk < GROUP / 16; ++kk) {
                        const int k16 = e * (GROUP / 16) + kk;
                        const uint32_t bar = 8 * (g * 2 + (k16 >> 2));
                        if ((!LATER_FIRST || part == 0) && k16 % 4 == 0) {
                            ok = ok && use_wait(a_full + bar, ci, CYCLE, &s_abort);
                            if (!ok) break;
                            fence_after();
                        }
#pragma unroll
                        for (int p = LATER_FIRST && part == 1 ? 0 : P - 1; p >= (part == 0 ? 1 : 0); --p)
                            w_mma_ts(on, t_d, t_a + k16 * 8, d_x + ((p * L::XPLANE + (k16 >> 2) * L::XBOX + (k16 & 3) * 32) >> 4), id,
                                     kk > 0 || p < (LATER_FIRST && part == 1 ? P : P - 1));
                        if (part == 1 && k16 % 4 == 3) w_commit(on, a_empty + bar);
                    }
                }
                if (!ok) break;
                w_commit(on, d_full + d_bar);
            }
            if (ok) w_commit(on, x_empty + 8 * xs);
        }
        if (__any_sync(0xffffffffu, s_abort)) {                 // MMAs in flight end before their operands and tensor memory go
            volatile int never = 0;
            w_commit(on, drained + 8 * warp);
            bar_wait_slow(drained + 8 * warp, 0, &never, nullptr);
        }
        __syncwarp();
        done();
    } else {
        // ---- x ----------------------------------------------------------------
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::R_COPY));
        const int w = warp - COPY_0;
        if constexpr (L::IN_ORDER) {
            if (w == 0) {
                const uint32_t on = elect_one();
                int ci = 0;
                for (; ci < nc; ++ci) {
                    const int xs = ci % XS;
                    if (!use_wait(x_empty + 8 * xs, ci + XS, XS, &s_abort)) break;
                    const uint32_t to = base + L::X + xs * L::XSTAGE, bar = x_full + 8 * xs;
                    w_expect_tx(on, bar, L::XSTAGE);
                    w_tma2d(on, to, &x_map, (c0 + ci) * CHUNK, i0, bar);
                    w_tma2d(on, to + L::XBOX, &x_map, (c0 + ci) * CHUNK + 64, i0, bar);
                }
                if (s_abort) {                                  // copies in flight land before the CTA goes on
                    volatile int never = 0;
                    for (int c = max(0, ci - XS); c < ci; ++c) bar_wait_slow(x_full + 8 * (c % XS), (uint32_t)(c / XS) & 1u, &never, nullptr);
                }
                __syncwarp();
            }
        } else if constexpr (!L::SPLIT) {
            // a stage a warp: copied, then each 8 values put into the order of the codes' pairs where they lie
            static_assert(XS == 4, "");
            const uint32_t on = elect_one(), at = base + L::X + w * L::XSTAGE;
            int copied = -1;
            for (int filled = w; filled < nc; filled += XS) {
                if (!use_wait(x_empty + 8 * w, filled + XS, XS, &s_abort)) break;
                copied = filled;
                w_expect_tx(on, x_raw + 8 * w, L::XSTAGE);
                w_tma2d(on, at, &x_map, (c0 + filled) * CHUNK, i0, x_raw + 8 * w);
                w_tma2d(on, at + L::XBOX, &x_map, (c0 + filled) * CHUNK + 64, i0, x_raw + 8 * w);
                if (!use_wait(x_raw + 8 * w, filled, XS, &s_abort)) break;
#pragma unroll 1
                for (int b = 0; b < N / 2; b += 4) {
                    Octet<T> o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i].v = lds16(at + ((b + i) * 32 + lane) * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t v[1][4];
                        o[i].pairs(v);
                        sts16(at + ((b + i) * 32 + lane) * 16, v[0]);
                    }
                }
                fence_proxy();
                __syncwarp();
                if (lane == 0) bar_arrive(x_full + 8 * w);
            }
            if (s_abort && copied >= 0) {                       // a copy in flight lands before the CTA goes on
                volatile int never = 0;
                bar_wait_slow(x_raw + 8 * w, (uint32_t)(copied / XS) & 1u, &never, nullptr);
            }
            __syncwarp();
        } else {
            const T *const x = static_cast<const T *>(a.x) + (long)i0 * a.ldx;
            for (int ci = w % XS; ci < nc; ci += XS) {
                const int slot = ci % XS;
                if (!use_wait(x_empty + 8 * slot, ci + XS, XS, &s_abort)) break;
                const uint32_t to = base + L::X + slot * L::XSTAGE;
                const int k0 = (c0 + ci) * CHUNK;
                constexpr int BATCH = 4;
                for (int b = w / XS * (N / 2 / L::X_PARTS); b < (w / XS + 1) * (N / 2 / L::X_PARTS); b += BATCH) {
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
        }
        done();
    }
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }

    if (a.split == 1) return;
    float *const y = a.y + (long)i0 * a.ldy;
    cluster_sync();                                             // totals [N][OUT] of every CTA
    // a part of the rows of x for each CTA, a row for each eight warps
    for (int i = rank + a.split * (tid / OUT); i < rows; i += a.split * (THREADS / OUT)) {
        const int o = tid % OUT;
        if (tid >= THREADS / OUT * OUT) break;
        float v = 0.f;
        for (int r = 0; r < a.split; ++r) v += peer_value(base + (i * OUT + o) * 4, r);
        if (j0 + o < a.w.o) {
            float *at = y + (long)i * a.ldy + j0 + o;
            *at = a.accumulate ? *at + v : v;
        }
    }
    cluster_sync();
}

// A matrix of rows x width elements of `size` bytes, `pitch` elements apart (a multiple of 16 bytes), in boxes of height x inner.
bool make_map(CUtensorMap *map, CUtensorMapDataType type, int size, const void *p, long width, long rows, long pitch, int inner, int height,
              CUtensorMapSwizzle swizzle) {
    static PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
        cudaDriverEntryPointQueryResult q;
        void *fn = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            fn = nullptr;
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)pitch * size};
    const cuuint32_t box[2] = {(cuuint32_t)inner, (cuuint32_t)height};
    const cuuint32_t estr[2] = {1, 1};
    return encode(map, type, 2, const_cast<void *>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Into how many parts K is cut, and about how long a call takes then. A part is a CTA that has an SM to itself, so what counts is how
// many clusters of that size fit the GPU at once (GPCs have 16 to 20 SMs: 152, 76, 46, 36, 28, 23, 15 and 15 were counted), a
// chunk's time, and what a CTA does beside its chunks: 3.8 us to start and to end, and to join 2.2 with 128 outputs or 16 rows, 3.5
// with 256 and 64 rows.
struct Cut {
    int split;
    float us;
};
Cut best_cut(long tiles, int chunks, float chunk_us, float join_us) {
    constexpr int fit[8] = {152, 76, 46, 36, 28, 23, 15, 15};
    Cut best{1, 0.f};
    for (int s = 1; s <= 8 && s <= chunks; ++s) {
        const float us = (tiles + fit[s - 1] - 1) / fit[s - 1] * (chunk_us * ((chunks + s - 1) / s) + 3.8f + (s > 1 ? join_us : 0.f));
        if (s == 1 || us < best.us) best = {s, us};
    }
    return best;
}
template <typename T, int GROUP, int N, int OUTPUTS>
Cut cut_of(int m, const Weight &w) {
    using L = Lay<T, GROUP, N, OUTPUTS>;
    // a chunk's time with groups of 32, 64 and 128: fp32, 16 and 32 rows; bf16, 16, 32, 64 and 128
    constexpr float us[2][6][3] = {{{1.30f, 1.04f, 0.87f}, {1.90f, 1.70f, 1.45f}, {1.20f, 0.80f, 0.67f}, {1.53f, 0.93f, 0.77f}, {2.05f, 1.18f, 0.84f}, {}},
                                   {{0.87f, 0.70f, 0.61f}, {1.30f, 1.20f, 1.13f}, {0.79f, 0.50f, 0.40f}, {0.85f, 0.56f, 0.44f}, {1.10f, 0.65f, 0.56f},
                                    {1.74f, 0.90f, 0.57f}}};
    constexpr int row = (L::SPLIT ? 0 : 2) + (N > 64 ? 3 : N > 32 ? 2 : N > 16 ? 1 : 0);
    return best_cut((long)((w.o + L::OUT - 1) / L::OUT) * ((m + N - 1) / N), (w.k + CHUNK - 1) / CHUNK,
                    us[L::HALF][row][GROUP == 32 ? 0 : GROUP == 64 ? 1 : 2], L::HALF ? 2.2f : 1.6f + 0.03f * N);
}

// How a call is launched with blocks of N rows and OUTPUTS outputs: the parts of K, and what of scales and zeros a CTA stages.
template <typename T, int GROUP, int N, int OUTPUTS>
Linear4Shape shape_of(int m, const Weight &w) {
    using L = Lay<T, GROUP, N, OUTPUTS>;
    const int chunks = (w.k + CHUNK - 1) / CHUNK, split = cut_of<T, GROUP, N, OUTPUTS>(m, w).split;
    const int slice = (chunks + split - 1) / split * L::PER;
    const size_t beside = (size_t)slice * ((L::OUT + 2) * 2 + (w.zeros ? L::OUT + 4 : 0));
    const bool staged = beside <= L::ROOM, direct = reinterpret_cast<uintptr_t>(w.codes) % 16 != 0 || w.k % 32 != 0;
    const size_t smem = std::max<size_t>(L::SCALES + 1024 + (staged ? beside : 0), tmem_smem_floor(512));
    return Linear4Shape{N, OUTPUTS, split, staged, direct, staged ? slice : 0, smem};
}

template <typename T, int GROUP, int N, int OUTPUTS>
cudaError_t launch(Args a, cudaStream_t s) {
    using L = Lay<T, GROUP, N, OUTPUTS>;
    const Linear4Shape c = shape_of<T, GROUP, N, OUTPUTS>(a.m, a.w);
    CUtensorMap map, x_map;
    memset(&x_map, 0, sizeof x_map);
    a.direct = c.direct;
    memset(&map, 0, sizeof map);
    if ((!a.direct && !make_map(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.w.codes, a.w.k / 2, a.w.o, a.w.k / 2, CHUNK / 2, TILE, CU_TENSOR_MAP_SWIZZLE_64B)) ||
        (!L::SPLIT && !make_map(&x_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, a.x, a.w.k, a.m, a.ldx, 64, N, CU_TENSOR_MAP_SWIZZLE_128B)))
        return cudaErrorUnknown;
    const int tiles = (a.w.o + L::OUT - 1) / L::OUT, cols = (a.m + N - 1) / N;
    a.split = c.split;
    a.staged = c.staged;
    a.slice = c.slice;
    cudaError_t e = cudaFuncSetAttribute(linear4_tc_kernel<T, GROUP, N, OUTPUTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_MOST);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(tiles * a.split, cols);
    lc.blockDim = THREADS;
    lc.dynamicSmemBytes = c.smem;
    lc.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = a.split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = programmatic(s) ? 2 : 1;
    e = cudaLaunchKernelEx(&lc, linear4_tc_kernel<T, GROUP, N, OUTPUTS>, map, x_map, a);
    note_launch();
    return e;
}

template <int N> using Rows = std::integral_constant<int, N>;
template <int N> using Outs = std::integral_constant<int, N>;

// f of the rows and outputs that a CTA of this call has.
//
// 128 outputs to a CTA where that fills the GPU better: 60 rows, k and o 4096, groups of 128 10.7 us, with 256 12.9; o 11008 21.6 and
// 16.6; 16 fp32 rows, k 8192, o 1024 10.5 and 12.2.
template <typename T, int GROUP, int N>
float best_us(int m, const Weight &w) {
    return std::min(cut_of<T, GROUP, N, 128>(m, w).us, cut_of<T, GROUP, N, 256>(m, w).us);
}
template <typename T, int GROUP, int N, typename F>
auto with_outputs(int m, const Weight &w, F f) {
    if (cut_of<T, GROUP, N, 128>(m, w).us < cut_of<T, GROUP, N, 256>(m, w).us) return f(Rows<N>(), Outs<128>());
    return f(Rows<N>(), Outs<256>());
}
template <typename T, int GROUP, typename F>
auto with_blocks(int m, const Weight &w, F f) {
    if (m <= 16) return with_outputs<T, GROUP, 16>(m, w, f);
    // (fp32: 32 rows at most. With 256 outputs the 64 totals of 64 rows would leave the copying warps too few registers; with 128
    // outputs two stages of x and the codes' ring would fit: not built)
    if constexpr (sizeof(T) == 2) {
        // 128 rows of x with 128 outputs: chunks that take less than those of 64 rows and 256 outputs. (645 rows, k 4096, 11008
        // outputs: 82 us instead of 112.) Rows just past a multiple of 128 can leave the first with more waves: 130 rows of the
        // same 41 us instead of 30.
        if (m > 64 && cut_of<T, GROUP, 128, 128>(m, w).us < best_us<T, GROUP, 64>(m, w)) return f(Rows<128>(), Outs<128>());
        if (m > 32) return with_outputs<T, GROUP, 64>(m, w, f);
    }
    return with_outputs<T, GROUP, 32>(m, w, f);
}
template <typename F>
auto with_group(const Weight &w, F f) {
    return w.group == 128 ? f(std::integral_constant<int, 128>()) : w.group == 64 ? f(std::integral_constant<int, 64>()) : f(std::integral_constant<int, 32>());
}

}  // namespace

template <typename T>
cudaError_t launch_linear4_tc(const T *x, long ldx, int m, const Weight &w, float *y, long ldy, int accumulate, cudaStream_t s, int stall) {
    const Args a{w, x, ldx, ldy, y, m, accumulate, 1, 0, 0, 0, stall};
    return with_group(w, [&](auto group) {
        return with_blocks<T, decltype(group)::value>(
            m, w, [&](auto rows, auto outs) { return launch<T, decltype(group)::value, decltype(rows)::value, decltype(outs)::value>(a, s); });
    });
}

template <typename T>
Linear4Shape linear4_tc_shape(int m, const Weight &w) {
    return with_group(w, [&](auto group) {
        return with_blocks<T, decltype(group)::value>(
            m, w, [&](auto rows, auto outs) { return shape_of<T, decltype(group)::value, decltype(rows)::value, decltype(outs)::value>(m, w); });
    });
}

template <typename T>
float linear4_tc_us(const Weight &w) {
    return with_group(w, [&](auto group) { return best_us<T, decltype(group)::value, 16>(1, w); });
}

template float linear4_tc_us<float>(const Weight &);
template float linear4_tc_us<bf16>(const Weight &);
template Linear4Shape linear4_tc_shape<float>(int, const Weight &);
template Linear4Shape linear4_tc_shape<bf16>(int, const Weight &);
template cudaError_t launch_linear4_tc<float>(const float *, long, int, const Weight &, float *, long, int, cudaStream_t, int);
template cudaError_t launch_linear4_tc<bf16>(const bf16 *, long, int, const Weight &, float *, long, int, cudaStream_t, int);

}  // namespace msd
