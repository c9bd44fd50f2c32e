// Attention over pages on CUDA cores (fp32 pools), and the launch that joins partial results.
//
// A CTA takes 64 packed rows (pages_attn.cuh) against key tiles of 64: scores as register
// tiles of 4 x 4, an online softmax in base 2 over the 16 threads that share a row, O in
// registers. A key that a row does not see has the weight -0, and in a tile whose V holds a
// NaN or an infinity such keys are skipped; slots past the sequence's end are not read.
#include "pages_attn.cuh"

namespace msd {
namespace {

constexpr int ROWS = 64, KT = 64, THREADS = 256, PLD = KT + 4;
constexpr float HIDDEN = -0.f;
constexpr int JOIN_WARPS = 8;

template <int HD>
struct Lay {
    static constexpr int LD = HD + 4;                 // padded: the rows a warp reads together sit in different banks
    static constexpr int Q = 0, K = Q + ROWS * LD, V = K + KT * LD, P = V + KT * LD;
    static constexpr int SCHED = P + ROWS * PLD;      // floats before the schedule
    static constexpr int SMEM = SCHED * 4 + (int)sizeof(AttnSched);
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int HD>
__global__ void __launch_bounds__(THREADS) pages_attn_simt_kernel(const PagesAttn a) {
    using L = Lay<HD>;
    extern __shared__ __align__(16) float sm[];
    float *sQ = sm + L::Q, *sK = sm + L::K, *sV = sm + L::V, *sP = sm + L::P;
    AttnSched &sched = *reinterpret_cast<AttnSched *>(sm + L::SCHED);
    wait_prior();
    allow_dependents();
    if (a.b.n > ATTN_WARP_SEQS) attn_schedule<ROWS, KT, THREADS>(a, sched, blockIdx.x, gridDim.x);
    else if (threadIdx.x < 32) attn_schedule<ROWS, KT, 32>(a, sched, blockIdx.x, gridDim.x);
    __syncthreads();
    const PagesView &v = a.pv;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, G = a.group;
    if (tid == 0) name_parts<ROWS, KT>(a, sched, blockIdx.x);
    const float *kv = static_cast<const float *>(v.kv) + (long)a.layer * v.n_pages * v.page_elems();
    AttnWalk<ROWS, KT> walk(a, sched);
    Segment g;
    while (walk.next(g)) {
        const int len = sched.len[g.i], rows = sched.rows[g.i], start = a.b.row_start[g.i], base = len - rows;
        const int m0 = g.tile * ROWS, nm = min(rows * G - m0, ROWS);
        const int live_rows = a.mask && a.n_nodes ? min(rows, a.n_nodes[g.i]) : rows;
        const int *table = v.table + (long)a.b.seqs[g.i] * v.max_pages;
        __syncthreads();
        for (int e = tid; e < ROWS * (HD / 4); e += THREADS) {
            const int m = e / (HD / 4), c = (e - m * (HD / 4)) * 4, r = (m0 + m) / G;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (m < nm)
                x = *reinterpret_cast<const float4 *>(static_cast<const float *>(a.q) + (start + r) * a.ldq +
                                                     (long)(g.h * G + (m0 + m) % G) * HD + c);
            *reinterpret_cast<float4 *>(sQ + m * L::LD + c) = x;
        }
        // this thread's four rows
        int qrow[4], place[4];
        const uint64_t *mrow[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int m = m0 + 4 * ty + x, r = m / G;
            const bool in = 4 * ty + x < nm && r < live_rows;
            qrow[x] = in ? r : -1;
            const long at = (long)g.i * a.nodes + r;
            mrow[x] = in && a.mask ? a.mask + at * a.words : nullptr;
            place[x] = base + (a.mask ? (in && a.window ? a.depth[at] : 0) : r);
        }
        float acc[4][HD / 16], mx[4], sum[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            mx[x] = -INFINITY;
            sum[x] = 0.f;
#pragma unroll
            for (int c = 0; c < HD / 16; ++c) acc[x][c] = 0.f;
        }
        for (int j = g.j0; j < g.j1; ++j) {
            const int kt = j < g.range.sink_tiles ? j : g.range.lo + j - g.range.sink_tiles;
            const int key0 = kt * KT;
            __syncthreads();
            bool odd = false;                        // V holds a value that is not finite
            for (int e = tid; e < KT * (HD / 4); e += THREADS) {
                const int k = e / (HD / 4), c = (e - k * (HD / 4)) * 4, slot = key0 + k;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
                if (slot < len) {
                    const int id = table[slot >> v.page_shift];
                    if ((unsigned)id < (unsigned)v.n_pages) {
                        const float *src = kv + id * v.page_elems() + ((long)g.h * v.page + (slot & (v.page - 1))) * HD + c;
                        x = *reinterpret_cast<const float4 *>(src);
                        y = *reinterpret_cast<const float4 *>(src + (long)v.kv_heads * v.page * HD);
                    }
                }
                odd |= !(isfinite(y.x) && isfinite(y.y) && isfinite(y.z) && isfinite(y.w));
                *reinterpret_cast<float4 *>(sK + k * L::LD + c) = x;
                *reinterpret_cast<float4 *>(sV + k * L::LD + c) = y;
            }
            odd = __syncthreads_or(odd);
            float s[4][4] = {};
#pragma unroll 4
            for (int d = 0; d < HD; d += 4) {
                float4 q[4], k[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) q[x] = *reinterpret_cast<const float4 *>(sQ + (4 * ty + x) * L::LD + d);
#pragma unroll
                for (int y = 0; y < 4; ++y) k[y] = *reinterpret_cast<const float4 *>(sK + (tx + 16 * y) * L::LD + d);
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        s[x][y] = fmaf(q[x].x, k[y].x, s[x][y]);
                        s[x][y] = fmaf(q[x].y, k[y].y, s[x][y]);
                        s[x][y] = fmaf(q[x].z, k[y].z, s[x][y]);
                        s[x][y] = fmaf(q[x].w, k[y].w, s[x][y]);
                    }
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                bool see[4];
                float top = -INFINITY;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int slot = key0 + tx + 16 * y, node = slot - base;
                    bool ok = qrow[x] >= 0 && slot < len;
                    int at = slot;
                    if (ok && node >= 0) {
                        if (a.mask) {
                            ok = mrow[x][node >> 6] >> (node & 63) & 1;
                            if (a.window) at = base + a.depth[(long)g.i * a.nodes + node];
                        } else {
                            ok = node <= qrow[x];
                        }
                    }
                    if (a.window) ok = ok && (place[x] - at < a.window || at < a.sinks);
                    see[y] = ok;
                    if (ok) top = fmaxf(top, s[x][y]);
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
                    const float p = see[y] ? exp2_fast(fmaf(s[x][y], a.scale_log2, -use)) : HIDDEN;
                    part += p;
                    sP[(4 * ty + x) * PLD + tx + 16 * y] = p;
                }
                sum[x] = sum[x] * f + part;
#pragma unroll
                for (int c = 0; c < HD / 16; ++c) acc[x][c] *= f;
            }
            __syncthreads();
            auto add = [&](auto skip) {
#pragma unroll 2
                for (int k = 0; k < KT; ++k) {
                    float p[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) p[x] = sP[(4 * ty + x) * PLD + k];
#pragma unroll
                    for (int c = 0; c < HD / 64; ++c) {
                        const float4 w = *reinterpret_cast<const float4 *>(sV + k * L::LD + 64 * c + 4 * tx);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            if (decltype(skip)::value && __float_as_uint(p[x]) == 0x80000000u) continue;
                            acc[x][4 * c] = fmaf(p[x], w.x, acc[x][4 * c]);
                            acc[x][4 * c + 1] = fmaf(p[x], w.y, acc[x][4 * c + 1]);
                            acc[x][4 * c + 2] = fmaf(p[x], w.z, acc[x][4 * c + 2]);
                            acc[x][4 * c + 3] = fmaf(p[x], w.w, acc[x][4 * c + 3]);
                        }
                    }
                }
            };
            if (odd) add(std::true_type());
            else add(std::false_type());
        }
        const bool whole = segment_whole(g);
        const long slot = part_slot(g, blockIdx.x) * ROWS;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sum[x] += __shfl_xor_sync(0xffffffffu, sum[x], o, 16);
            const int m = 4 * ty + x;
            if (m >= nm) continue;
            const int r = start + (m0 + m) / G, head = g.h * G + (m0 + m) % G;
            if (whole) {
                // (a sum that is not a number is kept; only an empty row divides by nothing)
                const float inv = sum[x] == 0.f ? 0.f : 1.f / sum[x];
                float *out = static_cast<float *>(a.out) + r * a.ldo + (long)head * HD;
#pragma unroll
                for (int c = 0; c < HD / 64; ++c)
                    *reinterpret_cast<float4 *>(out + 64 * c + 4 * tx) =
                        make_float4(acc[x][4 * c] * inv, acc[x][4 * c + 1] * inv, acc[x][4 * c + 2] * inv, acc[x][4 * c + 3] * inv);
                if (a.lse && tx == 0)
                    a.lse[(long)r * v.heads + head] = sum[x] == 0.f ? -INFINITY : (mx[x] + log2f(sum[x])) * 0.6931471805599453f;
            } else {
                float *o = a.part_o + (slot + m) * HD;
#pragma unroll
                for (int c = 0; c < HD / 64; ++c)
                    *reinterpret_cast<float4 *>(o + 64 * c + 4 * tx) =
                        make_float4(acc[x][4 * c], acc[x][4 * c + 1], acc[x][4 * c + 2], acc[x][4 * c + 3]);
                if (tx == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * (slot + m)) = make_float2(mx[x], sum[x]);
            }
        }
    }
}

// Joins the partial results of items that several CTAs worked on: block (CTA that ended an item, rows), a warp
// a row. A lane holds the weight of a part (32 at a time); the parts' O are added in the order of the keys, eight
// requested at once, the first ones before the weights are known.
template <typename T, int HD>
__global__ void __launch_bounds__(32 * JOIN_WARPS) pages_attn_join_kernel(const PagesAttn a, int tile_rows) {
    wait_prior();
    allow_dependents();
    const PartItem item = a.part_item[blockIdx.x];
    const int lane = threadIdx.x & 31, m = blockIdx.y * JOIN_WARPS + (threadIdx.x >> 5);
    if (m >= item.rows) return;
    constexpr int E = HD / 32;
    const int c0 = item.cta, parts = (int)blockIdx.x - c0 + 1;
    auto at = [&](int k) { return (2l * (c0 + k) + (k == 0 ? 1 : 0)) * tile_rows + m; };
    float x[8][E];
    auto fetch = [&](int k) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (k + u < parts) {
                const float *src = a.part_o + at(k + u) * HD + lane * E;
                if constexpr (E == 4) {
                    const float4 y = *reinterpret_cast<const float4 *>(src);
                    x[u][0] = y.x; x[u][1] = y.y; x[u][2] = y.z; x[u][3] = y.w;
                } else {
                    const float2 y = *reinterpret_cast<const float2 *>(src);
                    x[u][0] = y.x; x[u][1] = y.y;
                }
            }
    };
    auto ml_of = [&](int k) {
        return k < parts ? *reinterpret_cast<const float2 *>(a.part_ml + 2 * at(k)) : make_float2(-INFINITY, 0.f);
    };
    const float2 first = ml_of(lane);
    fetch(0);
    float top = first.y != 0.f ? first.x : -INFINITY;
    for (int k = lane + 32; k < parts; k += 32) {
        const float2 ml = ml_of(k);
        if (ml.y != 0.f) top = fmaxf(top, ml.x);
    }
    top = warp_max(top);
    float acc[E] = {}, sum = 0.f;
    for (int k0 = 0; k0 < parts; k0 += 32) {
        const float2 ml = k0 ? ml_of(k0 + lane) : first;
        float w = 0.f;
        if (ml.y != 0.f) {                            // (else nothing was seen there)
            w = ml.x == top ? 1.f : exp2f(ml.x - top);
            sum += ml.y * w;
        }
        for (int k = k0; k < min(k0 + 32, parts); k += 8) {
            if (k) fetch(k);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float wu = __shfl_sync(0xffffffffu, w, (k + u) & 31);
                if (k + u < parts && wu != 0.f) {
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = fmaf(x[u][e], wu, acc[e]);
                }
            }
        }
    }
    sum = warp_sum(sum);
    const int pm = item.m0 + m, q = group_div(a, pm), r = item.start + q, head = item.h * a.group + pm - q * a.group;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T *out = static_cast<T *>(a.out) + r * a.ldo + (long)head * HD + lane * E;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < E; e += 2) *reinterpret_cast<float2 *>(out + e) = make_float2(acc[e] * inv, acc[e + 1] * inv);
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 2)
            *reinterpret_cast<__nv_bfloat162 *>(out + e) = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
    }
    if (a.lse && lane == 0)
        a.lse[(long)r * a.pv.heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

template <int HD>
cudaError_t launch(const PagesAttn &a, int sms, cudaStream_t s) {
    const int ctas = sms * (HD == 64 ? 2 : 1);
    cudaError_t e = launch_chain(pages_attn_simt_kernel<HD>, dim3(ctas), dim3(THREADS), Lay<HD>::SMEM, s, a);
    note_launch();
    return e != cudaSuccess ? e : launch_pages_attn_join(a, MSD_F32, ctas, ROWS, s);
}

}  // namespace

size_t pages_attn_part_rows(int sms) { return 2 * 256 * (size_t)sms; }

cudaError_t launch_pages_attn_join(const PagesAttn &a, int dtype, int ctas, int tile_rows, cudaStream_t s) {
    const dim3 grid(ctas, (tile_rows + JOIN_WARPS - 1) / JOIN_WARPS), block(32 * JOIN_WARPS);
    cudaError_t e;
    if (dtype == MSD_F32)
        e = a.pv.head_dim == 64 ? launch_chain(pages_attn_join_kernel<float, 64>, grid, block, 0, s, a, tile_rows)
                                : launch_chain(pages_attn_join_kernel<float, 128>, grid, block, 0, s, a, tile_rows);
    else
        e = a.pv.head_dim == 64 ? launch_chain(pages_attn_join_kernel<bf16, 64>, grid, block, 0, s, a, tile_rows)
                                : launch_chain(pages_attn_join_kernel<bf16, 128>, grid, block, 0, s, a, tile_rows);
    note_launch();
    return e;
}

bool pages_attn_simt_setup() {
    auto set = [](const void *f, int bytes) {
        return cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
    };
    return set((const void *)pages_attn_simt_kernel<64>, Lay<64>::SMEM) &&
           set((const void *)pages_attn_simt_kernel<128>, Lay<128>::SMEM);
}

cudaError_t launch_pages_attn_simt(const PagesAttn &a, int sms, cudaStream_t s) {
    return a.pv.head_dim == 64 ? launch<64>(a, sms, s) : launch<128>(a, sms, s);
}

}  // namespace msd
