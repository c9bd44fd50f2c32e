// Attention over pages on CUDA cores (fp32 pools), and the launch that joins partial results.
//
// A CTA takes 64 packed rows (pages_attn.cuh; 16 where sequences have few) against key tiles of 64: scores as register
// tiles of packed fp32 FMAs over even and odd elements, an online softmax in base 2 over the 16 threads that share a row,
// the weights as pairs (p, p) in shared memory, O in registers as packed columns. K and V have one buffer each: the next
// tile's K is copied (cp.async) while the weights meet V, and its V while the next scores are made. What bounds it: the
// shared-memory loads that feed the FMAs, and at few tiles the chain of round trips (schedule, table, K). Measured with
// the join: 16 heads of 64, two chunks of up to 333 rows 34 us; a tree of 16 rows behind 96 tokens 11 us.
// A key that a row does not see has the weight -0, and in a tile whose V holds a NaN or an infinity such keys are
// skipped (looked for only where a row does not see the whole tile); slots past the sequence's end are not read, and
// those of a table entry that is no page count as zeros.
#include <type_traits>

#include "pages_attn.cuh"

namespace msd {
namespace {

constexpr int KT = 64, THREADS = 256;
constexpr float HIDDEN = -0.f;
constexpr int JOIN_WARPS = 8;

template <int HD, int ROWS>
struct Lay {
    static constexpr int LD = HD + 4;                 // padded: the rows a warp reads together sit in different banks
    static constexpr int PLD = KT + 2;                // in pairs
    static constexpr int Q = 0, K = Q + ROWS * LD, V = K + KT * LD, P = V + KT * LD;
    static constexpr int SCHED = P + 2 * ROWS * PLD;  // floats before the schedule
    static constexpr int SMEM = SCHED * 4 + (int)sizeof(AttnSched);
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long pair(float x, float y) {
    unsigned long long d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
    return d;
}
__device__ __forceinline__ float lo(unsigned long long v) { return __uint_as_float((unsigned)v); }
__device__ __forceinline__ float hi(unsigned long long v) { return __uint_as_float((unsigned)(v >> 32)); }
// 16 bytes into shared memory, zeros where `live` is false
__device__ __forceinline__ void copy16(float *dst, const float *src, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(src),
                 "r"(live ? 16 : 0)
                 : "memory");
}
template <int N>
__device__ __forceinline__ void copies_wait() {          // all but the last N groups
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

template <int HD, int ROWS>
__global__ void __launch_bounds__(THREADS) pages_attn_simt_kernel(const PagesAttn a) {
    using L = Lay<HD, ROWS>;
    constexpr int R = ROWS / 16, C = HD / 64;            // rows of a thread; groups of 4 columns of O
    extern __shared__ __align__(16) float sm[];
    __shared__ int s_lost;                               // an entry of the table is no page
    if (threadIdx.x == 0) s_lost = 0;
    float *sQ = sm + L::Q, *sK = sm + L::K, *sV = sm + L::V;
    unsigned long long *sP = reinterpret_cast<unsigned long long *>(sm + L::P);
    AttnSched &sched = *reinterpret_cast<AttnSched *>(sm + L::SCHED);
    wait_prior();
    allow_dependents();
    attn_schedule<ROWS, KT, THREADS>(a, sched, blockIdx.x, gridDim.x);
    const PagesView &v = a.pv;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, G = a.group;
    if (tid == 0) name_parts<ROWS, KT>(a, sched, blockIdx.x);
    if (a.mask && a.window) check_depths<ROWS, KT>(a, sched, tid, THREADS);
    const float *kv = static_cast<const float *>(v.kv) + (long)a.layer * v.n_pages * v.page_elems();
    AttnWalk<ROWS, KT> walk(a, sched);
    Segment g;
    while (walk.next(g)) {
        const int len = sched.len[g.i], rows = sched.rows[g.i], start = a.b.row_start[g.i], base = len - rows;
        const int m0 = g.tile * ROWS, nm = min(rows * G - m0, ROWS);
        const int live_rows = a.mask && a.n_nodes ? min(rows, a.n_nodes[g.i]) : rows;
        const int *table = v.table + (long)a.b.seqs[g.i] * v.max_pages;
        auto key_of = [&](int j) { return (j < g.range.sink_tiles ? j : g.range.lo + j - g.range.sink_tiles) * KT; };
        // K (what 0) or V (1) of a tile
        auto load = [&](float *dst, int what, int key0) {
#pragma unroll
            for (int e = tid; e < KT * (HD / 4); e += THREADS) {
                const int k = e / (HD / 4), c = (e - k * (HD / 4)) * 4, slot = key0 + k;
                int id = slot < len ? table[slot >> v.page_shift] : -1;
                const bool live = (unsigned)id < (unsigned)v.n_pages;         // (else zeros)
                if (!live && slot < len) s_lost = 1;
                copy16(dst + k * L::LD + c,
                       live ? kv + id * v.page_elems() + ((long)(what * v.kv_heads + g.h) * v.page + (slot & (v.page - 1))) * HD + c : kv,
                       live);
            }
            copies_commit();
        };
        __syncthreads();                                 // the segment before has been read
        for (int e = tid; e < ROWS * (HD / 4); e += THREADS) {
            const int m = e / (HD / 4), c = (e - m * (HD / 4)) * 4, r = group_div(a, m0 + m);
            const float *src = static_cast<const float *>(a.q);
            if (m < nm) src += (start + r) * a.ldq + (long)(g.h * G + m0 + m - r * G) * HD + c;
            copy16(sQ + m * L::LD + c, src, m < nm);
        }
        load(sK, 0, key_of(g.j0));
        load(sV, 1, key_of(g.j0));
        // this thread's rows
        int qrow[R], place[R];
        const uint64_t *mrow[R];
#pragma unroll
        for (int x = 0; x < R; ++x) {
            const int m = m0 + R * ty + x, r = group_div(a, m);
            const bool in = R * ty + x < nm && r < live_rows;
            qrow[x] = in ? r : -1;
            const long at = (long)g.i * a.nodes + r;
            mrow[x] = in && a.mask ? a.mask + at * a.words : nullptr;
            place[x] = base + (a.mask ? (in && a.window ? node_depth(a, g.i, r) : 0) : r);
        }
        // all rows that are there see a whole tile that ends and starts within these
        const bool blind = group_div(a, m0 + nm - 1) >= live_rows;
        const int full_end = blind ? 0 : base + (a.mask ? 0 : group_div(a, m0) + 1);
        const int full_start = !a.window ? 0 : base + (a.mask ? a.nodes : group_div(a, m0 + nm - 1)) - a.window + 1;
        unsigned long long acc[R][2 * C];
        float mx[R], sum[R];
#pragma unroll
        for (int x = 0; x < R; ++x) {
            mx[x] = -INFINITY;
            sum[x] = 0.f;
#pragma unroll
            for (int c = 0; c < 2 * C; ++c) acc[x][c] = 0;
        }
        for (int j = g.j0; j < g.j1; ++j) {
            const int key0 = key_of(j);
            const bool full = key0 + KT <= full_end && (key0 >= full_start || key0 + KT <= a.sinks);
            copies_wait<1>();                            // K (and Q)
            __syncthreads();
            unsigned long long s2[R][4];
#pragma unroll
            for (int x = 0; x < R; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) s2[x][y] = 0;
#pragma unroll 4
            for (int d = 0; d < HD; d += 4) {
                ulonglong2 q[R], k[4];
#pragma unroll
                for (int x = 0; x < R; ++x) q[x] = *reinterpret_cast<const ulonglong2 *>(sQ + (R * ty + x) * L::LD + d);
#pragma unroll
                for (int y = 0; y < 4; ++y) k[y] = *reinterpret_cast<const ulonglong2 *>(sK + (tx + 16 * y) * L::LD + d);
#pragma unroll
                for (int x = 0; x < R; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) s2[x][y] = fma2(q[x].y, k[y].y, fma2(q[x].x, k[y].x, s2[x][y]));
            }
#pragma unroll
            for (int x = 0; x < R; ++x) {
                float s[4], top = -INFINITY;
                bool see[4] = {true, true, true, true};
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    s[y] = lo(s2[x][y]) + hi(s2[x][y]);
                    if (!full) {
                        const int slot = key0 + tx + 16 * y, node = slot - base;
                        bool ok = qrow[x] >= 0 && slot < len;
                        int at = slot;
                        if (ok && node >= 0) {
                            if (a.mask) {
                                ok = mrow[x][node >> 6] >> (node & 63) & 1;
                                if (a.window) at = base + node_depth(a, g.i, node);
                            } else {
                                ok = node <= qrow[x];
                            }
                        }
                        if (a.window) ok = ok && (place[x] - at < a.window || at < a.sinks);
                        see[y] = ok;
                    }
                    if (see[y]) top = fmaxf(top, s[y]);
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o, 16));
                const float now = fmaxf(mx[x], top * a.scale_log2);
                const float use = now == -INFINITY ? 0.f : now;
                const float f = exp2_fast(mx[x] - use);
                mx[x] = now;
                float part = 0.f;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float p = see[y] ? exp2_fast(fmaf(s[y], a.scale_log2, -use)) : HIDDEN;
                    part += p;
                    sP[(R * ty + x) * L::PLD + tx + 16 * y] = pair(p, p);
                }
                sum[x] = sum[x] * f + part;
                const unsigned long long f2 = pair(f, f);
#pragma unroll
                for (int c = 0; c < 2 * C; ++c) acc[x][c] = fma2(acc[x][c], f2, 0);
            }
            copies_wait<0>();                            // V
            bool odd = false;
            if (!full) {
#pragma unroll
                for (int e = tid; e < KT * (HD / 4); e += THREADS) {
                    const int k = e / (HD / 4), c = (e - k * (HD / 4)) * 4;
                    const float4 y = *reinterpret_cast<const float4 *>(sV + k * L::LD + c);
                    odd |= !(isfinite(y.x) && isfinite(y.y) && isfinite(y.z) && isfinite(y.w));
                }
            }
            odd = __syncthreads_or(odd);                 // (and everybody's P and V are there, and K has been read)
            if (j + 1 < g.j1) load(sK, 0, key_of(j + 1));
            auto add = [&](auto skip) {
#pragma unroll 2
                for (int k = 0; k < KT; k += 2) {
                    ulonglong2 p[R];
#pragma unroll
                    for (int x = 0; x < R; ++x) p[x] = *reinterpret_cast<const ulonglong2 *>(sP + (R * ty + x) * L::PLD + k);
#pragma unroll
                    for (int c = 0; c < C; ++c)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const ulonglong2 w = *reinterpret_cast<const ulonglong2 *>(sV + (k + u) * L::LD + 64 * c + 4 * tx);
#pragma unroll
                            for (int x = 0; x < R; ++x) {
                                const unsigned long long q = u ? p[x].y : p[x].x;
                                if (decltype(skip)::value && (unsigned)q == 0x80000000u) continue;
                                acc[x][2 * c] = fma2(q, w.x, acc[x][2 * c]);
                                acc[x][2 * c + 1] = fma2(q, w.y, acc[x][2 * c + 1]);
                            }
                        }
                }
            };
            if (odd) add(std::true_type());
            else add(std::false_type());
            if (j + 1 < g.j1) {
                __syncthreads();                         // V and P have been read
                load(sV, 1, key_of(j + 1));
            }
        }
        const bool whole = segment_whole(g);
        const long slot = part_slot(g, blockIdx.x) * ROWS;
#pragma unroll
        for (int x = 0; x < R; ++x) {
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sum[x] += __shfl_xor_sync(0xffffffffu, sum[x], o, 16);
            const int m = R * ty + x;
            if (m >= nm) continue;
            const int q = group_div(a, m0 + m), r = start + q, head = g.h * G + m0 + m - q * G;
            // (a sum that is not a number is kept; only an empty row divides by nothing)
            const float inv = !whole ? 1.f : sum[x] == 0.f ? 0.f : 1.f / sum[x];
            float *out = whole ? static_cast<float *>(a.out) + r * a.ldo + (long)head * HD : a.part_o + (slot + m) * HD;
#pragma unroll
            for (int c = 0; c < C; ++c)
                *reinterpret_cast<float4 *>(out + 64 * c + 4 * tx) =
                    make_float4(lo(acc[x][2 * c]) * inv, hi(acc[x][2 * c]) * inv, lo(acc[x][2 * c + 1]) * inv, hi(acc[x][2 * c + 1]) * inv);
            if (tx == 0) {
                if (!whole) *reinterpret_cast<float2 *>(a.part_ml + 2 * (slot + m)) = make_float2(mx[x], sum[x]);
                else if (a.lse)
                    a.lse[(long)r * v.heads + head] = sum[x] == 0.f ? -INFINITY : (mx[x] + log2f(sum[x])) * 0.6931471805599453f;
            }
        }
    }
    __syncthreads();
    if (tid == 0 && s_lost) set_status(v.status, ST_RANGE);
}

// Joins the partial results of items that several CTAs worked on: block (CTA that ended an item, rows), a warp
// RW rows. A lane holds the weight of a part (32 at a time); the parts' O are added in the order of the keys, PRE
// requested at once, the first ones before the weights are known. Long contexts have few rows and many parts (RW 1,
// PRE 8), prompts many rows and mostly two parts (RW 2, PRE 2; joined by the last CTA to be done instead, inside
// the main kernel, ragged chunks took 340 us, not 303, and a tree 47, not 23). Cold: 6 to 7 us after single tokens, 14 to 15 us after
// prompts of 4096 and 8192 rows.
template <typename T, int HD, int RW, int PRE>
__global__ void __launch_bounds__(32 * JOIN_WARPS) pages_attn_join_kernel(const PagesAttn a, int tile_rows) {
    wait_prior();
    allow_dependents();
    const PartItem item = a.part_item[blockIdx.x];
    const int lane = threadIdx.x & 31, m0 = (blockIdx.y * JOIN_WARPS + (threadIdx.x >> 5)) * RW;
    if (m0 >= item.rows) return;
    constexpr int E = HD / 32;
    const int c0 = item.cta, parts = (int)blockIdx.x - c0 + 1;
    auto at = [&](int k, int m) { return (2l * (c0 + k) + (k == 0 ? 1 : 0)) * tile_rows + m; };
    float x[RW][PRE][E];
    auto fetch = [&](int w, int k) {
#pragma unroll
        for (int u = 0; u < PRE; ++u)
            if (k + u < parts && m0 + w < item.rows) {
                const float *src = a.part_o + at(k + u, m0 + w) * HD + lane * E;
                if constexpr (E == 4) {
                    const float4 y = *reinterpret_cast<const float4 *>(src);
                    x[w][u][0] = y.x; x[w][u][1] = y.y; x[w][u][2] = y.z; x[w][u][3] = y.w;
                } else {
                    const float2 y = *reinterpret_cast<const float2 *>(src);
                    x[w][u][0] = y.x; x[w][u][1] = y.y;
                }
            }
    };
    auto ml_of = [&](int w, int k) {
        return k < parts && m0 + w < item.rows ? *reinterpret_cast<const float2 *>(a.part_ml + 2 * at(k, m0 + w))
                                               : make_float2(-INFINITY, 0.f);
    };
    float2 first[RW];
#pragma unroll
    for (int w = 0; w < RW; ++w) {
        first[w] = ml_of(w, lane);
        fetch(w, 0);
    }
#pragma unroll
    for (int w = 0; w < RW; ++w) {
        if (m0 + w >= item.rows) break;
        float top = first[w].y != 0.f ? first[w].x : -INFINITY;
        for (int k = lane + 32; k < parts; k += 32) {
            const float2 ml = ml_of(w, k);
            if (ml.y != 0.f) top = fmaxf(top, ml.x);
        }
        top = warp_max(top);
        float acc[E] = {}, sum = 0.f;
        for (int k0 = 0; k0 < parts; k0 += 32) {
            const float2 ml = k0 ? ml_of(w, k0 + lane) : first[w];
            float f = 0.f;
            if (ml.y != 0.f) {                        // (else nothing was seen there)
                f = ml.x == top ? 1.f : exp2f(ml.x - top);
                sum += ml.y * f;
            }
            for (int k = k0; k < min(k0 + 32, parts); k += PRE) {
                if (k) fetch(w, k);
#pragma unroll
                for (int u = 0; u < PRE; ++u) {
                    const float fu = __shfl_sync(0xffffffffu, f, (k + u) & 31);
                    if (k + u < parts && fu != 0.f) {
#pragma unroll
                        for (int e = 0; e < E; ++e) acc[e] = fmaf(x[w][u][e], fu, acc[e]);
                    }
                }
            }
        }
        sum = warp_sum(sum);
        const int pm = item.m0 + m0 + w, q = group_div(a, pm), r = item.start + q, head = item.h * a.group + pm - q * a.group;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        T *out = static_cast<T *>(a.out) + r * a.ldo + (long)head * HD + lane * E;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < E; e += 2) *reinterpret_cast<float2 *>(out + e) = make_float2(acc[e] * inv, acc[e + 1] * inv);
        } else if constexpr (E == 4) {
            const __nv_bfloat162 b0 = __floats2bfloat162_rn(acc[0] * inv, acc[1] * inv),
                                 b1 = __floats2bfloat162_rn(acc[2] * inv, acc[3] * inv);
            *reinterpret_cast<uint2 *>(out) = make_uint2(*reinterpret_cast<const uint32_t *>(&b0), *reinterpret_cast<const uint32_t *>(&b1));
        } else {
            *reinterpret_cast<__nv_bfloat162 *>(out) = __floats2bfloat162_rn(acc[0] * inv, acc[1] * inv);
        }
        if (a.lse && lane == 0)
            a.lse[(long)r * a.pv.heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
}

template <typename T, int HD>
cudaError_t launch_join(const PagesAttn &a, int ctas, int tile_rows, cudaStream_t s) {
    const int rows = JOIN_WARPS * (tile_rows > 128 ? 2 : 1);
    const dim3 grid(ctas, (tile_rows + rows - 1) / rows), block(32 * JOIN_WARPS);
    return tile_rows > 128 ? launch_chain(pages_attn_join_kernel<T, HD, 2, 2>, grid, block, 0, s, a, tile_rows)
                           : launch_chain(pages_attn_join_kernel<T, HD, 1, 8>, grid, block, 0, s, a, tile_rows);
}

template <int HD, int ROWS>
cudaError_t launch(const PagesAttn &a, int sms, cudaStream_t s) {
    const int ctas = sms * (HD == 64 || ROWS == 16 ? 2 : 1);
    cudaError_t e = launch_chain(pages_attn_simt_kernel<HD, ROWS>, dim3(ctas), dim3(THREADS), Lay<HD, ROWS>::SMEM, s, a);
    note_launch();
    return e != cudaSuccess ? e : launch_pages_attn_join(a, MSD_F32, ctas, ROWS, s);
}

template <int HD, int ROWS>
bool setup() {
    return cudaFuncSetAttribute(pages_attn_simt_kernel<HD, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                Lay<HD, ROWS>::SMEM) == cudaSuccess;
}

}  // namespace

size_t pages_attn_part_rows(int sms) { return 2 * 256 * (size_t)sms; }

cudaError_t launch_pages_attn_join(const PagesAttn &a, int dtype, int ctas, int tile_rows, cudaStream_t s) {
    const bool wide = a.pv.head_dim == 128;
    const cudaError_t e = dtype == MSD_F32 ? wide ? launch_join<float, 128>(a, ctas, tile_rows, s) : launch_join<float, 64>(a, ctas, tile_rows, s)
                          : wide           ? launch_join<bf16, 128>(a, ctas, tile_rows, s)
                                           : launch_join<bf16, 64>(a, ctas, tile_rows, s);
    note_launch();
    return e;
}

bool pages_attn_simt_setup() { return setup<64, 16>() && setup<64, 64>() && setup<128, 16>() && setup<128, 64>(); }

cudaError_t launch_pages_attn_simt(const PagesAttn &a, int sms, cudaStream_t s) {
    // few packed rows to a sequence: tiles of 16, whose steps are short
    const bool few = a.packed <= 16;
    if (a.pv.head_dim == 64) return few ? launch<64, 16>(a, sms, s) : launch<64, 64>(a, sms, s);
    return few ? launch<128, 16>(a, sms, s) : launch<128, 64>(a, sms, s);
}

}  // namespace msd
