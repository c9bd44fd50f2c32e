// Tokens from logits: what temperature, top-k, top-p and min-p leave of a row, a token drawn from
// it with a given uniform (msd_sample), and speculative sampling over drafted trees on it
// (msd_accept_batch).
//
// Every setting leaves a run from the front of the order (larger logit first, then lower id), so
// what is left is described by the last logit in it, by how many of the tokens that have just
// this logit are in it (the ones with the lowest ids), and by the exponent that min-p allows.
// Weights are integers (weight_exp.cuh), so sums over any part of a row are exact, and every
// search below is one for the place where an exact, monotone sum passes a bound.
#include <algorithm>

#include "msd.h"
#include "weight_exp.cuh"

namespace msd {

typedef unsigned long long u64;

static __device__ const ExpTable g_exp_table = ExpTable();

constexpr int ROW_THREADS = 512;
constexpr int MAX_VOCAB = 393216;
constexpr int MAX_CHILDREN = 256;
constexpr int MAX_TREE_NODES = 1024;

template <typename T> __device__ __forceinline__ float logit_at(const T *row, int i);
template <> __device__ __forceinline__ float logit_at<float>(const float *row, int i) { return row[i]; }
template <> __device__ __forceinline__ float logit_at<bf16>(const bf16 *row, int i) { return __bfloat162float(row[i]); }

// floor(f * z) and ceil(f * z) for f in [0, 1): f is an integer of 24 bits times a power of two.
__device__ __forceinline__ u64 share_floor(float f, u64 z, bool up) {
    const unsigned b = __float_as_uint(f);
    const int e = (int)(b >> 23);
    const u64 m = (b & 0x7FFFFFu) | (e ? 0x800000u : 0u);
    const int s = 150 - max(e, 1);                      // f = m * 2^-s, s >= 24
    const u64 lo = m * z, hi = __umul64hi(m, z);
    if (s >= 128) return up && (lo | hi) ? 1 : 0;
    const u64 q = s >= 64 ? hi >> (s - 64) : hi << (64 - s) | lo >> s;
    const bool rest = s >= 64 ? lo != 0 || (s > 64 && hi << (128 - s) != 0) : lo << (64 - s) != 0;
    return q + (up && rest ? 1 : 0);
}

struct Settings {
    const float *temperature;
    const int *top_k;
    const float *top_p, *min_p;
};

// What is left of a row.
struct Left {
    RowScale scale;
    unsigned key;             // smallest key in it
    int tie;                  // of the ids with this key, the ones up to here
    float2 limit;             // largest exponent (min-p)
    u64 total;                // its weight; 0: nothing is left
};

__device__ __forceinline__ u64 weight_left(const Left &l, float x, int id, const float2 *table) {
    const unsigned k = key_of(x);
    if (k < l.key || (k == l.key && id > l.tie) || k == 0) return 0;
    if (x == l.scale.top) return 1ull << WEIGHT_BITS;   // also where it is +inf
    const float2 y = exponent_of(x, l.scale);
    if (!((y.x - l.limit.x) + (y.y - l.limit.y) <= 0.f)) return 0;
    return weight_of(y, table);
}

struct Shared {
    float2 table[EXP_STEPS];
    u64 red[33];
};

__device__ __forceinline__ u64 block_total(u64 v, u64 *red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        u64 t = threadIdx.x < blockDim.x >> 5 ? red[threadIdx.x] : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (threadIdx.x == 0) red[32] = t;
    }
    __syncthreads();
    return red[32];
}

// Sum of f(id, logit) over the row.
template <typename T, typename F>
__device__ __forceinline__ u64 row_total(const T *row, int V, Shared &sh, F f) {
    u64 v = 0;
    for (int i = threadIdx.x; i < V; i += blockDim.x) v += f(i, logit_at(row, i));
    return block_total(v, sh.red);
}

__device__ __forceinline__ void load_table(Shared &sh) {
    for (int i = threadIdx.x; i < EXP_STEPS; i += blockDim.x)
        sh.table[i] = make_float2(g_exp_table.hi[i], g_exp_table.lo[i]);
    __syncthreads();
}

// What the settings of entry `at` leave of a row.
template <typename T>
__device__ Left filter_row(const T *row, int V, const Settings &f, int at, Shared &sh) {
    Left l;
    unsigned best = 0;
    for (int i = threadIdx.x; i < V; i += blockDim.x) best = max(best, key_of(logit_at(row, i)));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.red[threadIdx.x >> 5] = best;
    __syncthreads();
    for (int i = 0; i < (int)(blockDim.x >> 5); ++i) best = max(best, (unsigned)sh.red[i]);
    l.total = 0;
    l.key = 1;
    l.tie = V;
    l.limit = make_float2(INFINITY, 0.f);
    l.scale = RowScale{logit_of(best), 0.f, 0.f};
    if (best == 0) return l;

    float temp = f.temperature ? f.temperature[at] : 1.f;
    int k = f.top_k ? f.top_k[at] : 0;
    const float p = f.top_p ? f.top_p[at] : 1.f, m = f.min_p ? f.min_p[at] : 0.f;
    if (!(temp >= 0x1p-100f) || m > 1.f || p <= 0.f) k = 1;
    temp = fminf(fmaxf(temp, 0x1p-100f), 0x1p100f);
    if (!(temp > 0.f)) temp = 1.f;
    const double c = 1.4426950408889634074 / (double)temp;
    l.scale.c_hi = (float)c;
    l.scale.c_lo = (float)(c - (double)l.scale.c_hi);

    u64 need = ~0ull;                                   // ids with the last key that are left
    const auto weigh = [&](float x) {
        Left all = l;
        all.key = 1;
        return weight_left(all, x, 0, sh.table);
    };
    if (k > 0 && k < V) {
        unsigned t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const unsigned c2 = t | 1u << bit;
            if (row_total(row, V, sh, [&](int, float x) { return (u64)(key_of(x) >= c2); }) >= (u64)k) t = c2;
        }
        if (t > 0) {
            l.key = t;
            need = k - row_total(row, V, sh, [&](int, float x) { return (u64)(key_of(x) > t); });
        }
    }
    if (p < 1.f && k != 1) {
        const u64 above = row_total(row, V, sh, [&](int, float x) { return key_of(x) > l.key ? weigh(x) : 0; });
        const u64 ties = row_total(row, V, sh, [&](int, float x) { return (u64)(key_of(x) == l.key); });
        const u64 goal = max(share_floor(p, above + (ties ? min(need, ties) * weigh(logit_of(l.key)) : 0), true), 1ull);
        unsigned t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const unsigned c2 = t | 1u << bit;
            if (c2 <= l.key || row_total(row, V, sh, [&](int, float x) { return key_of(x) >= c2 ? weigh(x) : 0; }) >= goal)
                t = c2;
        }
        const u64 over = row_total(row, V, sh, [&](int, float x) { return key_of(x) > t ? weigh(x) : 0; });
        const u64 each = max(weigh(logit_of(t)), 1ull);
        const u64 some = (goal - over + each - 1) / each;
        need = t == l.key ? min(need, some) : some;
        l.key = t;
    }
    if (m > 0.f) {
        const double y = -log2((double)fminf(m, 1.f));
        l.limit.x = (float)y;
        l.limit.y = (float)(y - (double)l.limit.x);
    }
    if (need < (u64)V) {
        // the need-th id with the last key
        unsigned t = 0;
        for (int bit = 18; bit >= 0; --bit) {
            const unsigned c2 = t | 1u << bit;          // ids below c2
            if (row_total(row, V, sh, [&](int i, float x) { return (u64)((unsigned)i < c2 && key_of(x) == l.key); }) < need)
                t = c2;
        }
        l.tie = (int)t;
    }
    l.total = row_total(row, V, sh, [&](int i, float x) { return weight_left(l, x, i, sh.table); });
    return l;
}

// The smallest id whose cumulative weight exceeds u of all; w(id, logit) are the weights, total their sum.
template <typename T, typename F>
__device__ int draw_row(const T *row, int V, float u, u64 total, Shared &sh, F w) {
    if (total == 0) return -1;
    u = fminf(u > 0.f ? u : 0.f, 0x1.fffffep-1f);
    const u64 goal = share_floor(u, total, false);
    unsigned t = 0;
    for (int bit = 18; bit >= 0; --bit) {
        const unsigned c2 = t | 1u << bit;
        if (row_total(row, V, sh, [&](int i, float x) { return (unsigned)i < c2 ? w(i, x) : 0; }) <= goal) t = c2;
    }
    return (int)t;
}

template <typename T>
__global__ void __launch_bounds__(ROW_THREADS)
sample_kernel(const T *__restrict__ logits, long ld, int V, Settings f, const float *__restrict__ u,
              int *__restrict__ tokens, float *__restrict__ logp, float *__restrict__ probs, long ldp) {
    wait_prior();
    allow_dependents();
    __shared__ Shared sh;
    load_table(sh);
    const T *row = logits + (long)blockIdx.x * ld;
    const Left l = filter_row(row, V, f, blockIdx.x, sh);
    const int t = draw_row(row, V, u[blockIdx.x], l.total, sh,
                           [&](int i, float x) { return weight_left(l, x, i, sh.table); });
    if (threadIdx.x == 0) {
        tokens[blockIdx.x] = t;
        if (logp) {
            const float x = t < 0 ? 0.f : logit_at(row, t);
            const float2 y = t < 0 || x == l.scale.top ? make_float2(0.f, 0.f) : exponent_of(x, l.scale);
            logp[blockIdx.x] = t < 0 ? -INFINITY : (float)(-0.69314718055994530942 * ((double)y.x + (double)y.y + log2((double)l.total) - WEIGHT_BITS));
        }
    }
    if (probs) {
        const double inv = l.total ? 1.0 / (double)l.total : 0.0;
        const float scale = (float)(inv * 0x1p44);
        for (int i = threadIdx.x; i < V; i += blockDim.x) {
            const float x = logit_at(row, i);
            float w = 0.f;
            const unsigned k = key_of(x);
            if (k > l.key || (k == l.key && i <= l.tie && k)) {
                const float2 y = x == l.scale.top ? make_float2(0.f, 0.f) : exponent_of(x, l.scale);
                if ((y.x - l.limit.x) + (y.y - l.limit.y) <= 0.f) w = exp2f(-y.x) * (1.f - 0.69314718f * y.y) * scale;
            }
            probs[(long)blockIdx.x * ldp + i] = w;
        }
    }
}

// Per node of the trees: the child that is accepted there, or -1 and the token drawn there.
struct TreeArgs {
    int n, nodes, depth, children;
    const int *row_start, *tokens, *parent, *n_nodes;
    const float *u;
    int *next, *drawn;        // [rows]
    int *path, *accept_len, *bonus;
};

__device__ __forceinline__ int nodes_of(const TreeArgs &a, int b) {
    const int rows = min(a.row_start[b + 1] - a.row_start[b], a.nodes);
    return a.n_nodes ? min(rows, a.n_nodes[b]) : rows;
}

template <typename T>
__global__ void __launch_bounds__(ROW_THREADS)
accept_rows_kernel(const T *__restrict__ logits, long ld, int V, Settings f, TreeArgs a) {
    wait_prior();
    allow_dependents();
    __shared__ Shared sh;
    __shared__ int s_next, s_gone[MAX_CHILDREN], s_gones;
    __shared__ u64 s_left;
    const int r = blockIdx.x;
    int b = 0;
    for (int hi = a.n; hi - b > 1;) {                   // the last sequence that starts at or before the row
        const int mid = (b + hi) >> 1;
        if (a.row_start[mid] <= r) b = mid; else hi = mid;
    }
    const int node = r - a.row_start[b], n = nodes_of(a, b);
    const int *parent = a.parent + (long)b * a.nodes, *tokens = a.tokens + (long)b * a.nodes;
    if (node >= n) return;
    int d = 0;
    for (int i = node; i > 0; ++d) {
        const int up = parent[i];
        if (up < 0 || up >= i) { d = a.depth + 1; break; }
        i = up;
    }
    if (d > a.depth) return;                            // never reached
    load_table(sh);
    const T *row = logits + (long)r * ld;
    const Left l = filter_row(row, V, f, b, sh);
    const float *u = a.u + ((long)b * (a.depth + 1) + d) * (a.children + 1);
    if (threadIdx.x == 0) {
        u64 left = l.total;
        int gone = 0, next = -1;
        for (int j = node + 1, c = 0; j < n && c < a.children && d < a.depth && next < 0; ++j) {
            if (parent[j] != node) continue;
            const int t = tokens[j];
            u64 w = t >= 0 && t < V && l.total ? weight_left(l, logit_at(row, t), t, sh.table) : 0;
            for (int i = 0; i < gone; ++i)
                if (s_gone[i] == t) w = 0;
            const float v = fminf(u[c] > 0.f ? u[c] : 0.f, 0x1.fffffep-1f);
            if (share_floor(v, left, false) < w) next = j;
            else if (w) { left -= w; s_gone[gone++] = t; }
            ++c;
        }
        s_next = next;
        s_gones = gone;
        s_left = left;
    }
    __syncthreads();
    int t = -1;
    if (s_next < 0)
        t = draw_row(row, V, u[a.children], s_left, sh, [&](int i, float x) {
            const u64 w = weight_left(l, x, i, sh.table);
            if (w)
                for (int g = 0; g < s_gones; ++g)
                    if (s_gone[g] == i) return 0ull;
            return w;
        });
    if (threadIdx.x == 0) {
        a.next[r] = s_next;
        a.drawn[r] = t;
    }
}

__global__ void accept_walk_kernel(TreeArgs a) {
    wait_prior();
    allow_dependents();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= a.n) return;
    int *path = a.path + (long)b * (a.depth + 1);
    int at = nodes_of(a, b) > 0 ? 0 : -1, d = 0, bonus = -1;
    const int start = a.row_start[b];
    for (; at >= 0 && d <= a.depth; ++d) {
        path[d] = at;
        const int next = a.next[start + at];
        if (next < 0) bonus = a.drawn[start + at];
        at = next;
    }
    a.accept_len[b] = max(d - 1, 0);
    a.bonus[b] = bonus;
    for (; d <= a.depth; ++d) path[d] = -1;
}

static bool take_filter(const msd_filter *f, Settings *s) {
    *s = f ? Settings{f->temperature, f->top_k, f->top_p, f->min_p} : Settings{};
    return true;
}

static bool bad_logits(const void *logits, long ld, int dtype, int V) {
    return !logits || (dtype != MSD_F32 && dtype != MSD_BF16) || V < 1 || V > MAX_VOCAB || ld < V ||
           reinterpret_cast<uintptr_t>(logits) % (dtype == MSD_F32 ? 4 : 2);
}

}  // namespace msd

using namespace msd;

extern "C" {

msd_status msd_sample(const void *logits, int64_t ld, int32_t dtype, int32_t rows, int32_t vocab,
                      const msd_filter *f, const float *u, int32_t *tokens, float *logp, float *probs,
                      int64_t ldp, void *stream) {
    if (rows < 0) return MSD_ERR_INVALID;
    if (rows == 0) return MSD_OK;
    if (bad_logits(logits, ld, dtype, vocab) || !u || !tokens || (probs && (ldp < vocab || reinterpret_cast<uintptr_t>(probs) % 4)))
        return MSD_ERR_INVALID;
    Settings s;
    take_filter(f, &s);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e =
        dtype == MSD_F32
            ? launch_chain(sample_kernel<float>, rows, ROW_THREADS, 0, st, static_cast<const float *>(logits), (long)ld,
                           vocab, s, u, tokens, logp, probs, (long)ldp)
            : launch_chain(sample_kernel<bf16>, rows, ROW_THREADS, 0, st, static_cast<const bf16 *>(logits), (long)ld,
                           vocab, s, u, tokens, logp, probs, (long)ldp);
    if (e != cudaSuccess) return MSD_ERR_CUDA;
    note_launch();
    return MSD_OK;
}

msd_status msd_accept_batch(const void *logits, int64_t ld, int32_t dtype, int32_t vocab, const msd_batch *batch,
                            const msd_tree *tree, int32_t tree_nodes, const msd_filter *f, const float *u,
                            int32_t depth, int32_t children, int32_t *scratch, int32_t *path, int32_t *accept_len,
                            int32_t *bonus, void *stream) {
    if (!batch || batch->n < 0 || batch->rows < 0) return MSD_ERR_INVALID;
    if (batch->n == 0) return MSD_OK;
    if (!batch->row_start || !tree || !tree->tokens || !tree->parent || tree_nodes < 1 || tree_nodes > MAX_TREE_NODES ||
        !u || depth < 0 || depth > (1 << 20) || children < 1 || children > MAX_CHILDREN || !path || !accept_len || !bonus)
        return MSD_ERR_INVALID;
    if (batch->rows > 0 && (bad_logits(logits, ld, dtype, vocab) || !scratch)) return MSD_ERR_INVALID;
    Settings s;
    take_filter(f, &s);
    const TreeArgs a{batch->n, tree_nodes, depth, children, batch->row_start, tree->tokens, tree->parent, tree->n_nodes, u,
                     scratch, scratch + batch->rows, path, accept_len, bonus};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (batch->rows > 0) {
        const cudaError_t e =
            dtype == MSD_F32
                ? launch_chain(accept_rows_kernel<float>, batch->rows, ROW_THREADS, 0, st,
                               static_cast<const float *>(logits), (long)ld, vocab, s, a)
                : launch_chain(accept_rows_kernel<bf16>, batch->rows, ROW_THREADS, 0, st,
                               static_cast<const bf16 *>(logits), (long)ld, vocab, s, a);
        if (e != cudaSuccess) return MSD_ERR_CUDA;
        note_launch();
    }
    if (launch_chain(accept_walk_kernel, (batch->n + 31) / 32, 32, 0, st, a) != cudaSuccess) return MSD_ERR_CUDA;
    note_launch();
    return MSD_OK;
}

}  // extern "C"
