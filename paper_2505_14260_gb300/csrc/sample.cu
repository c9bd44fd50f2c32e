// Tokens from logits: what temperature, top-k, top-p and min-p leave of a row, a token drawn from
// it with a given uniform (msd_sample), and speculative sampling over drafted trees on it
// (msd_accept_batch).
//
// Every setting leaves a run from the front of the order (larger logit first, then lower id), so
// what is left is described by the last logit in it, by the last of the ids that have just this
// logit, and by the exponent that min-p allows. Weights are integers (weight_exp.cuh), so sums over
// any part of a row are exact, and every search below is one for the place where an exact,
// monotone sum passes a bound.
//
// A row belongs to a cluster of 1 to 8 CTAs, each with a slice of it in shared memory: it is read
// from memory once. The end of the run is found by a histogram of the order (1024 buckets, linear
// in the exponent; counts for top-k, exact masses in three 32-bit pieces for top-p), a look at the
// one bucket that the bound falls into, and the comparison of its few tokens with one another. A
// bucket with too many tokens is split again by the logits' bits, down to equal logits, where ids
// decide; so nothing depends on how logits are spread. Sums of blocks of 128 or 256 ids then lead to the token.
#include <algorithm>

#include "msd.h"
#include "weight_exp.cuh"

namespace msd {

typedef unsigned long long u64;

static __device__ const ExpTable g_exp_table = ExpTable();

constexpr int ROW_THREADS = 512, WARPS = ROW_THREADS / 32;
constexpr int BUCKETS = 1024, LIST = 512;
constexpr float Y_MOST = 46.f;                  // exponents from here on have weight 0
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

// What is left of a row: logits above `end`, and of the ids with just this logit the ones up to `tie`.
struct Left {
    RowScale scale;
    float end;
    int tie;
    float2 limit;             // largest exponent (min-p)
    u64 total;                // its weight; 0: nothing is left

    // (NaN and -inf are in no run: it starts at -inf with no id)
    __device__ __forceinline__ bool has(float x, int id) const { return x > end || (x == end && id <= tie); }
};

// Weight of a token of a run, without min-p.
__device__ __forceinline__ u64 weight_in(const RowScale &r, float x, const float2 *table) {
    return x == r.top ? 1ull << WEIGHT_BITS : weight_of(exponent_of(x, r), table);      // (top may be +inf)
}

__device__ __forceinline__ u64 weight_left(const Left &l, float x, int id, const float2 *table) {
    if (!l.has(x, id)) return 0;
    if (x == l.scale.top) return 1ull << WEIGHT_BITS;
    const float2 y = exponent_of(x, l.scale);
    if (!((y.x - l.limit.x) + (y.y - l.limit.y) <= 0.f)) return 0;
    return weight_of(y, table);
}

// ---------------------------------------------------------------------------
// A row over the CTAs of a cluster
// ---------------------------------------------------------------------------
struct Shared {
    float2 table[EXP_STEPS];
    unsigned hist[3][BUCKETS];                  // own: counts, or masses in pieces of 15, 15 and 14 bits
    u64 all[BUCKETS];                           // of the whole row
    u64 red[WARPS + 1];
    u64 total[8];                               // of each CTA of the cluster
    float top[8], low[8];
    unsigned valid[8];
    u64 above;
    unsigned bucket;
    unsigned own_n, list_n, base[8];
    unsigned range_lo, range_hi;                // keys of the bucket's tokens
    float end;
    int tie, token;
    int next, gones, gone[MAX_CHILDREN];
    u64 left;
    // where the histogram was, once it is added up: weights of a bucket's tokens, and these, of the slice and of the row
    __device__ __forceinline__ u64 *list_w() { return reinterpret_cast<u64 *>(hist[0]); }
    __device__ __forceinline__ float *own_x() { return reinterpret_cast<float *>(hist[1]); }
    __device__ __forceinline__ int *own_id() { return reinterpret_cast<int *>(hist[1]) + LIST; }
    __device__ __forceinline__ float *list_x() { return reinterpret_cast<float *>(hist[2]); }
    __device__ __forceinline__ int *list_id() { return reinterpret_cast<int *>(hist[2]) + LIST; }
};
static_assert(2 * LIST <= BUCKETS && sizeof(Shared) + 771 * 512 / 2 + 771 / 2 * 8 + 32 <= 227 * 1024, "the largest slice of 8 fits");

__device__ __forceinline__ uint32_t peer_address(const void *p, int rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ void put(u64 *p, int rank, u64 v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer_address(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ void put(unsigned *p, int rank, unsigned v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_address(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void put(int *p, int rank, int v) { put(reinterpret_cast<unsigned *>(p), rank, (unsigned)v); }
__device__ __forceinline__ void put(float *p, int rank, float v) { put(reinterpret_cast<unsigned *>(p), rank, __float_as_uint(v)); }
__device__ __forceinline__ void add(u64 *p, int rank, u64 v) {
    asm volatile("red.shared::cluster.add.u64 [%0], %1;" ::"r"(peer_address(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ void least(unsigned *p, int rank, unsigned v) {
    asm volatile("red.shared::cluster.min.u32 [%0], %1;" ::"r"(peer_address(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void most(unsigned *p, int rank, unsigned v) {
    asm volatile("red.shared::cluster.max.u32 [%0], %1;" ::"r"(peer_address(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ unsigned take(unsigned *p, int rank, unsigned n) {
    unsigned v;
    asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(v) : "r"(peer_address(p, rank)), "r"(n) : "memory");
    return v;
}

__device__ __forceinline__ u64 warp_total(u64 v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// 16 bytes of a row.
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void get(const uint4 &v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
};
template <> struct Vec<bf16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void get(const uint4 &v, float (&x)[8]) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
        }
    }
};

template <typename T>
struct Row {
    static constexpr int E = Vec<T>::E, BLOCK = 32 * E;
    const T *row;             // in memory
    int V, ctas, rank;
    Shared *sh;
    u64 *sums;                // of the slice's blocks
    uint4 *data;              // the slice, -inf around it, in whole blocks
    int first, count, mis, blocks;              // ids of the slice; element `first` is data's element `mis`
    float top, low;           // largest and smallest logit above -inf
    unsigned valid;           // how many there are
    float bucket_scale;

    __device__ __forceinline__ void sync() const {
        if (ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        else __syncthreads();
    }
    template <typename U> __device__ __forceinline__ void tell(U *p, U v) const {          // one thread: to every CTA
        for (int r = 0; r < ctas; ++r) put(p, r, v);
    }
    __device__ __forceinline__ u64 block_sum(u64 v) const {
        v = warp_total(v);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh->red[threadIdx.x >> 5] = v;
        __syncthreads();
        if (threadIdx.x < 32) {
            const u64 t = warp_total(threadIdx.x < WARPS ? sh->red[threadIdx.x] : 0);
            if (threadIdx.x == 0) sh->red[WARPS] = t;
        }
        __syncthreads();
        return sh->red[WARPS];
    }

    // f(logits, first id, block) for the blocks of this warp, whole warps at a time, two blocks in flight. Around the
    // slice there is -inf.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        const int lane = threadIdx.x & 31, at = first - mis + lane * E;
        int b = threadIdx.x >> 5;
        for (; b + WARPS < blocks; b += 2 * WARPS) {
            const uint4 v0 = data[b * 32 + lane], v1 = data[(b + WARPS) * 32 + lane];
            float x[E];
            Vec<T>::get(v0, x);
            f(x, at + b * BLOCK, b);
            Vec<T>::get(v1, x);
            f(x, at + (b + WARPS) * BLOCK, b + WARPS);
        }
        if (b < blocks) {
            float x[E];
            Vec<T>::get(data[b * 32 + lane], x);
            f(x, at + b * BLOCK, b);
        }
    }

    // The slice into shared memory; largest and smallest logit of the row, tokens that have weight.
    __device__ void load() {
        const int tid = threadIdx.x;
        if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        for (int i = tid; i < EXP_STEPS; i += ROW_THREADS) {
            sh->table[i] = make_float2(g_exp_table.hi[i], g_exp_table.lo[i]);
            sh->all[i] = 0;                                                 // (as many buckets)
        }
        const T *from = row + first - mis;                                  // 16-byte aligned
        const uint4 *from16 = reinterpret_cast<const uint4 *>(from);
        const int vecs = blocks * 32;
        float hi = -INFINITY, lo = INFINITY;
        unsigned n = 0;
        constexpr int U = 8;
        for (int v0 = tid; v0 < vecs; v0 += U * ROW_THREADS) {
            uint4 q[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = v0 + u * ROW_THREADS, i = v * E;              // first element of the vector
                if (i >= mis && i + E <= mis + count) {
                    q[u] = __ldcs(from16 + v);
                } else {
                    constexpr unsigned NONE = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
                    q[u] = make_uint4(NONE, NONE, NONE, NONE);
                    if (v < vecs)
                        for (int e = 0; e < E; ++e)
                            if (i + e >= mis && i + e < mis + count) {
                                if constexpr (sizeof(T) == 4) {
                                    (&q[u].x)[e] = __float_as_uint(from[i + e]);
                                } else {
                                    const unsigned b = __bfloat16_as_ushort(from[i + e]);
                                    unsigned &w = (&q[u].x)[e >> 1];
                                    w = e & 1 ? (w & 0xFFFFu) | b << 16 : (w & 0xFFFF0000u) | b;
                                }
                            }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = v0 + u * ROW_THREADS;
                if (v >= vecs) break;
                data[v] = q[u];
                float x[E];
                Vec<T>::get(q[u], x);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool is = x[e] > -INFINITY;
                    hi = fmaxf(hi, x[e]);                                   // (leaves NaN out)
                    lo = is ? fminf(lo, x[e]) : lo;
                    n += is;
                }
            }
        }
        hi = warp_max(hi);
        lo = -warp_max(-lo);
        n = __reduce_add_sync(0xffffffffu, n);
        float *part = reinterpret_cast<float *>(sh->hist[0]);
        const int warp = tid >> 5;
        if ((tid & 31) == 0) { part[warp] = hi; part[32 + warp] = lo; sh->hist[1][warp] = n; }
        if (ctas > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");     // all CTAs run: their shared memory is there
        __syncthreads();
        if (tid < 32) {
            hi = warp_max(tid < WARPS ? part[tid] : -INFINITY);
            lo = -warp_max(tid < WARPS ? -part[32 + tid] : -INFINITY);
            n = __reduce_add_sync(0xffffffffu, tid < WARPS ? sh->hist[1][tid] : 0u);
            if (tid < ctas) {
                put(&sh->top[rank], tid, hi);
                put(&sh->low[rank], tid, lo);
                put(&sh->valid[rank], tid, n);
            }
        }
        sync();
        top = -INFINITY;
        low = INFINITY;
        valid = 0;
        for (int r = 0; r < ctas; ++r) {
            top = fmaxf(top, sh->top[r]);
            low = fminf(low, sh->low[r]);
            valid += sh->valid[r];
        }
    }

    // Buckets of equal width in the exponent between the largest logit and x_end.
    __device__ __forceinline__ void spread(const Left &l, float x_end) {
        const float y = fminf((l.scale.top - x_end) * l.scale.c_hi, Y_MOST);
        bucket_scale = y > 0.f ? (float)(BUCKETS - 1) / y * l.scale.c_hi : 0.f;
    }
    __device__ __forceinline__ unsigned bucket_of(float x, const Left &l) const {
        return x == l.scale.top ? 0u : (unsigned)__float2int_rz(fminf((l.scale.top - x) * bucket_scale, (float)(BUCKETS - 1)));
    }

    // Where the run of tokens of `l` ends whose count (mass false) reaches `goal`, or whose weight reaches the share
    // `p` of theirs (mass true): narrows l.end and l.tie. The bound lies within the run. Every CTA finds it by itself
    // from the whole row's histogram and the bucket's tokens, which all are sent.
    __device__ void cut(Left &l, bool mass, u64 goal, float p) {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        u64 above = 0;
        unsigned k_lo = 0, k_hi = 0;                                        // from the second round on: keys that the bound lies among
        int shift = -1;                                                     // -1: buckets of the exponent; else of the keys' bits
        const auto is_in = [&](float x, int id) {
            if (!l.has(x, id)) return false;
            if (shift < 0) return true;
            const unsigned k = key_of(x);
            return k >= k_lo && k <= k_hi;
        };
        const auto place = [&](float x) { return shift < 0 ? bucket_of(x, l) : (k_hi - key_of(x)) >> shift; };
        for (int round = 0;; ++round) {
            for (int i = tid; i < BUCKETS; i += ROW_THREADS) sh->hist[0][i] = sh->hist[1][i] = sh->hist[2][i] = 0;
            if (tid == 0) { sh->own_n = sh->list_n = 0; sh->range_lo = ~0u; sh->range_hi = 0; }
            __syncthreads();
            each([&](const float (&x)[E], int id, int) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (!is_in(x[e], id + e)) continue;
                    const unsigned b = place(x[e]);
                    if (mass) {
                        const u64 w = weight_in(l.scale, x[e], sh->table);
                        atomicAdd(&sh->hist[0][b], (unsigned)w & 0x7FFFu);
                        atomicAdd(&sh->hist[1][b], (unsigned)(w >> 15) & 0x7FFFu);
                        atomicAdd(&sh->hist[2][b], (unsigned)(w >> 30));
                    } else {
                        atomicAdd(&sh->hist[0][b], 1u);
                    }
                }
            });
            __syncthreads();
            for (int i = tid; i < BUCKETS; i += ROW_THREADS) {
                const u64 v = mass ? sh->hist[0][i] + ((u64)sh->hist[1][i] << 15) + ((u64)sh->hist[2][i] << 30) : sh->hist[0][i];
                if (v)
                    for (int r = 0; r < ctas; ++r) add(&sh->all[i], r, v);
            }
            sync();
            // the bucket that the bound falls into
            constexpr int PER = BUCKETS / ROW_THREADS;
            u64 v[PER], run = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                v[i] = sh->all[tid * PER + i];
                sh->all[tid * PER + i] = 0;                                 // (the next time that it is added to lies behind a sync)
                run += v[i];
            }
            const u64 own = run;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 t = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += t;
            }
            if (lane == 31) sh->red[warp] = run;
            __syncthreads();
            u64 before = above, all = 0;
            for (int i = 0; i < WARPS; ++i) {
                if (i < warp) before += sh->red[i];
                all += sh->red[i];
            }
            if (round == 0 && mass) goal = max(share_floor(p, all, true), 1ull);
            u64 at = before + run - own;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (at < goal && goal <= at + v[i]) { sh->bucket = tid * PER + i; sh->above = at; }
                at += v[i];
            }
            __syncthreads();
            const unsigned bucket = sh->bucket;
            above = sh->above;
            // its tokens, and the range of their keys
            unsigned lo = ~0u, hi = 0;
            each([&](const float (&x)[E], int id, int) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (!is_in(x[e], id + e) || place(x[e]) != bucket) continue;
                    const unsigned k = key_of(x[e]), slot = atomicAdd(&sh->own_n, 1u);
                    lo = min(lo, k);
                    hi = max(hi, k);
                    if (slot < LIST) { sh->own_x()[slot] = x[e]; sh->own_id()[slot] = id + e; }
                }
            });
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            if (lane == 0 && hi)
                for (int r = 0; r < ctas; ++r) { least(&sh->range_lo, r, lo); most(&sh->range_hi, r, hi); }
            __syncthreads();
            const unsigned own_n = sh->own_n;
            if (own_n && tid < ctas) sh->base[tid] = take(&sh->list_n, tid, own_n);
            __syncthreads();
            for (unsigned i = tid; i < min(own_n, (unsigned)LIST); i += ROW_THREADS)
                for (int r = 0; r < ctas; ++r) {
                    const unsigned slot = sh->base[r] + i;
                    if (slot < LIST) {
                        put(&sh->list_x()[slot], r, sh->own_x()[i]);
                        put(&sh->list_id()[slot], r, sh->own_id()[i]);
                    }
                }
            sync();
            const unsigned n = sh->list_n;
            k_lo = sh->range_lo;
            k_hi = sh->range_hi;
            if (n <= LIST) {
                // each token's place among them
                u64 *w = sh->list_w();
                for (unsigned i = tid; i < n; i += ROW_THREADS) w[i] = mass ? weight_in(l.scale, sh->list_x()[i], sh->table) : 1;
                __syncthreads();
                for (unsigned i = tid; i < n; i += ROW_THREADS) {
                    const float x = sh->list_x()[i];
                    const int id = sh->list_id()[i];
                    u64 s = above;
                    for (unsigned j = 0; j < n; ++j) {
                        const float xj = sh->list_x()[j];
                        if (xj > x || (xj == x && sh->list_id()[j] < id)) s += w[j];
                    }
                    if (s < goal && goal <= s + w[i]) { sh->end = x; sh->tie = id; }
                }
                __syncthreads();
                l.end = sh->end;
                l.tie = sh->tie;
                return;
            }
            if (k_lo == k_hi) {                                             // equal logits: ids decide
                const u64 each_w = mass ? max(weight_in(l.scale, sh->list_x()[0], sh->table), 1ull) : 1;
                const u64 need = (goal - above + each_w - 1) / each_w;
                const float x_end = sh->list_x()[0];
                const auto one = [&](float x, int id) { return (u64)(x == x_end && l.has(x, id)); };
                add_up(one);
                const int id = locate(need - 1, one);
                if (id >= 0)
                    for (int r = 0; r < ctas; ++r) put(&sh->token, r, id);
                sync();
                const int found = sh->token;
                l.end = x_end;
                l.tie = found;
                return;
            }
            shift = max(0, 22 - __clz(k_hi - k_lo));                        // (k_hi - k_lo) >> shift < BUCKETS
            __syncthreads();                                                // all have read the list's length and the range
        }
    }

    // Sums of w(logit, id) over each block, this CTA's, and all.
    template <typename W>
    __device__ u64 add_up(W w) {
        u64 sum = 0;
        each([&](const float (&x)[E], int id, int b) {
            u64 v = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) v += w(x[e], id + e);
            if (__any_sync(0xffffffffu, v != 0)) v = warp_total(v);
            if ((threadIdx.x & 31) == 0) { sums[b] = v; sum += v; }
        });
        sum = block_sum(sum);
        if (threadIdx.x == 0) tell(&sh->total[rank], sum);
        sync();
        u64 all = 0;
        for (int r = 0; r < ctas; ++r) all += sh->total[r];
        return all;
    }

    // After add_up: the smallest id whose cumulative w exceeds `goal`, which is less than the whole. One thread of one
    // CTA gets it, the others -1.
    template <typename W>
    __device__ int locate(u64 goal, W w) {
        int found = -1;
        u64 before = 0;
        for (int r = 0; r < rank; ++r) before += sh->total[r];
        if (before <= goal && goal < before + sh->total[rank] && threadIdx.x < 32) {
            const int lane = threadIdx.x;
            u64 rest = goal - before;
            int b0 = 0;
            u64 in = 0;
            for (;; b0 += 32) {                                             // the 32 blocks, then the one
                in = b0 + lane < blocks ? sums[b0 + lane] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 t = __shfl_up_sync(0xffffffffu, in, o);
                    if (lane >= o) in += t;
                }
                const u64 all = __shfl_sync(0xffffffffu, in, 31);
                if (rest < all || b0 + 32 >= blocks) break;
                rest -= all;
            }
            const unsigned over = __ballot_sync(0xffffffffu, in > rest);
            const int at = over ? __ffs(over) - 1 : 31;
            const u64 less = __shfl_sync(0xffffffffu, in, max(at - 1, 0));
            if (at > 0) rest -= less;
            const int b = b0 + at;
            float x[E];
            Vec<T>::get(data[b * 32 + lane], x);
            const int id = first - mis + b * BLOCK + lane * E;
            u64 v[E], sum = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) { v[e] = w(x[e], id + e); sum += v[e]; }
            u64 run = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 t = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += t;
            }
            u64 c = run - sum;
            if (c <= rest && rest < run)
                for (int e = 0; e < E; ++e) {
                    if (rest < c + v[e]) { found = id + e; break; }
                    c += v[e];
                }
        }
        return found;
    }

    // What the settings of entry `at` leave. `single`: a run of one token, which is then l.tie (no sums are made).
    __device__ Left filter(const Settings &f, int at, bool *single) {
        Left l;
        l.total = 0;
        l.end = -INFINITY;
        l.tie = -1;
        l.limit = make_float2(INFINITY, 0.f);
        l.scale = RowScale{top, 0.f, 0.f};
        *single = true;
        if (valid == 0) return l;
        float temp = f.temperature ? f.temperature[at] : 1.f;
        int k = f.top_k ? f.top_k[at] : 0;
        const float p = f.top_p ? f.top_p[at] : 1.f, m = f.min_p ? f.min_p[at] : 0.f;
        if (!(temp >= 0x1p-100f) || m > 1.f || p <= 0.f) k = 1;
        temp = temp > 0.f ? fminf(fmaxf(temp, 0x1p-100f), 0x1p100f) : 1.f;
        const double c = 1.4426950408889634074 / (double)temp;
        l.scale.c_hi = (float)c;
        l.scale.c_lo = (float)(c - (double)l.scale.c_hi);
        if (k == 1) {                                                       // the first token alone
            unsigned id = ~0u;
            const float best = top;
            each([&](const float (&x)[E], int first_id, int) {
#pragma unroll
                for (int e = E - 1; e >= 0; --e)
                    if (x[e] == best) id = min(id, (unsigned)(first_id + e));
            });
            id = __reduce_min_sync(0xffffffffu, id);
            if (threadIdx.x == 0) sh->range_lo = ~0u;
            sync();
            if ((threadIdx.x & 31) == 0 && id != ~0u)
                for (int r = 0; r < ctas; ++r) least(&sh->range_lo, r, id);
            sync();
            l.end = top;
            l.tie = (int)sh->range_lo;
            l.total = 1ull << WEIGHT_BITS;
            return l;
        }
        *single = false;
        float x_end = low;
        if (k > 0 && (unsigned)k < valid) {
            spread(l, x_end);
            cut(l, false, (u64)k, 1.f);
            x_end = l.end;
        }
        if (p < 1.f) {
            spread(l, x_end);
            cut(l, true, 0, p);
        }
        if (m > 0.f) {
            const double y = -log2((double)fminf(m, 1.f));
            l.limit.x = (float)y;
            l.limit.y = (float)(y - (double)l.limit.x);
        }
        l.total = add_up([&](float x, int id) { return weight_left(l, x, id, sh->table); });
        return l;
    }
};

__device__ __forceinline__ float uniform(float u) { return fminf(u > 0.f ? u : 0.f, 0x1.fffffep-1f); }

template <typename T>
__device__ __forceinline__ Row<T> open_row(const T *row, int V, int ctas, int rank, int slice, Shared *sh, uint8_t *behind) {
    Row<T> r;
    r.row = row;
    r.V = V;
    r.ctas = ctas;
    r.rank = rank;
    r.sh = sh;
    r.first = min(rank * slice, V);
    r.count = min(slice, V - r.first);
    r.mis = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));       // slices are multiples of 16 bytes
    r.blocks = (r.mis + r.count + Row<T>::BLOCK - 1) / Row<T>::BLOCK;
    const int most = (slice + 16 / (int)sizeof(T) + Row<T>::BLOCK - 1) / Row<T>::BLOCK;
    r.sums = reinterpret_cast<u64 *>(behind);
    r.data = reinterpret_cast<uint4 *>(behind + (most * 8 + 15) / 16 * 16);
    r.load();
    return r;
}

template <typename T>
__global__ void __launch_bounds__(ROW_THREADS, 2)
sample_kernel(const T *__restrict__ logits, long ld, int V, int ctas, int slice, Settings f, const float *__restrict__ u,
              int *__restrict__ tokens, float *__restrict__ logp, float *__restrict__ probs, long ldp) {
    wait_prior();
    allow_dependents();
    extern __shared__ __align__(16) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem);
    const int r = blockIdx.x / ctas, rank = blockIdx.x % ctas;
    Row<T> row = open_row(logits + (long)r * ld, V, ctas, rank, slice, &sh, smem + sizeof(Shared));
    bool single;
    const Left l = row.filter(f, r, &single);
    // the thread that knows the token writes it
    int t = -1;
    const bool speaks = rank == 0 && threadIdx.x == 0;
    if (single) t = l.tie;
    else t = row.locate(share_floor(uniform(u[r]), l.total, false), [&](float x, int id) { return weight_left(l, x, id, sh.table); });
    if (single ? speaks : t >= 0) {
        tokens[r] = t;
        if (logp) {
            const float x = t < 0 ? 0.f : logit_at(row.row, t);
            const float2 y = t < 0 || x == l.scale.top ? make_float2(0.f, 0.f) : exponent_of(x, l.scale);
            logp[r] = t < 0 ? -INFINITY : (float)(-0.69314718055994530942 * ((double)y.x + (double)y.y + log2((double)l.total) - WEIGHT_BITS));
        }
    }
    if (probs) {
        const float scale = l.total ? (float)(0x1p44 / (double)l.total) : 0.f;
        const T *data = reinterpret_cast<const T *>(row.data) + row.mis;
        float *to = probs + (long)r * ldp + row.first;
        for (int i = threadIdx.x; i < row.count; i += ROW_THREADS) {
            const float x = logit_at(data, i);
            float w = 0.f;
            if (l.has(x, row.first + i)) {
                const float2 y = x == l.scale.top ? make_float2(0.f, 0.f) : exponent_of(x, l.scale);
                if ((y.x - l.limit.x) + (y.y - l.limit.y) <= 0.f) w = exp2f(-y.x) * (1.f - 0.69314718f * y.y) * scale;
            }
            to[i] = w;
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
__global__ void __launch_bounds__(ROW_THREADS, 2)
accept_rows_kernel(const T *__restrict__ logits, long ld, int V, int ctas, int slice, Settings f, TreeArgs a) {
    wait_prior();
    allow_dependents();
    extern __shared__ __align__(16) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem);
    const int r = blockIdx.x / ctas, rank = blockIdx.x % ctas;
    int b = 0;
    for (int hi = a.n; hi - b > 1;) {                   // the last sequence that starts at or before the row
        const int mid = (b + hi) >> 1;
        if (a.row_start[mid] <= r) b = mid; else hi = mid;
    }
    const int node = r - a.row_start[b], n = nodes_of(a, b);
    const int *parent = a.parent + (long)b * a.nodes, *tokens = a.tokens + (long)b * a.nodes;
    if (node < 0 || node >= n) return;
    int d = 0;
    for (int i = node; i > 0; ++d) {
        const int up = parent[i];
        if (up < 0 || up >= i) { d = a.depth + 1; break; }
        i = up;
    }
    if (d > a.depth) return;                            // never reached (the whole cluster leaves)
    Row<T> row = open_row(logits + (long)r * ld, V, ctas, rank, slice, &sh, smem + sizeof(Shared));
    bool single;
    const Left l = row.filter(f, b, &single);
    const float *u = a.u + ((long)b * (a.depth + 1) + d) * (a.children + 1);
    if (rank == 0 && threadIdx.x < 32) {
        // the first `children` children, in index order; their weights; then the decisions one after another
        const int lane = threadIdx.x;
        u64 *kid_w = sh.all;
        int kids = 0;
        if (d < a.depth)
            for (int j0 = node + 1; j0 < n && kids < a.children; j0 += 32) {
                const int j = j0 + lane;
                const bool is = j < n && parent[j] == node;
                const unsigned all = __ballot_sync(0xffffffffu, is);
                const int slot = kids + __popc(all & ((1u << lane) - 1u));
                if (is && slot < a.children) {
                    const int t = tokens[j];
                    sh.own_id()[slot] = j;
                    sh.list_id()[slot] = t;
                    kid_w[slot] = t >= 0 && t < V && l.total ? weight_left(l, logit_at(row.row, t), t, sh.table) : 0;
                }
                kids = min(kids + __popc(all), a.children);
            }
        __syncwarp();
        u64 left = l.total;
        int gone = 0, next = -1;
        for (int c = 0; c < kids; ++c) {
            const int t = sh.list_id()[c];
            u64 w = kid_w[c];
            bool again = false;
            for (int i = lane; i < gone; i += 32) again |= sh.gone[i] == t;
            if (__any_sync(0xffffffffu, again)) w = 0;
            if (share_floor(uniform(u[c]), left, false) < w) {
                next = sh.own_id()[c];
                break;
            }
            if (w) {
                left -= w;
                if (lane == 0) sh.gone[gone] = t;
                ++gone;
                __syncwarp();
            }
        }
        if (lane == 0) {
            row.tell(&sh.next, next);
            row.tell(&sh.gones, gone);
            row.tell(&sh.left, left);
        }
        for (int p = 1; p < ctas; ++p)
            for (int i = lane; i < gone; i += 32) put(&sh.gone[i], p, sh.gone[i]);
    }
    row.sync();
    if (rank == 0 && threadIdx.x == 0) a.next[r] = sh.next;
    if (sh.next >= 0) return;
    const int gones = sh.gones;
    const u64 left = sh.left;
    if (single || left == 0) {
        if (rank == 0 && threadIdx.x == 0) a.drawn[r] = left ? l.tie : -1;
        return;
    }
    // the sums without the rejected tokens
    if (gones) {
        if (threadIdx.x == 0) {
            u64 less = 0;
            for (int g = 0; g < gones; ++g) {
                const int i = sh.gone[g] - row.first;
                if (i < 0 || i >= row.count) continue;
                const u64 v = weight_left(l, logit_at(reinterpret_cast<const T *>(row.data), row.mis + i), sh.gone[g], sh.table);
                row.sums[(row.mis + i) / Row<T>::BLOCK] -= v;
                less += v;
            }
            if (less) row.tell(&sh.total[rank], sh.total[rank] - less);
        }
        row.sync();
    }
    const int t = row.locate(share_floor(uniform(u[a.children]), left, false), [&](float x, int id) {
        u64 v = weight_left(l, x, id, sh.table);
        if (v)
            for (int g = 0; g < gones; ++g)
                if (sh.gone[g] == id) v = 0;
        return v;
    });
    if (t >= 0) a.drawn[r] = t;
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

// How many CTAs share a row, and the ids of each: as few as leave room for two CTAs on an SM, more where there are few
// rows (and 2048 ids for each).
struct Cut {
    int ctas, slice;
    size_t smem;
};
static Cut cut_rows(int rows, int V, int size) {
    const auto smem = [&](int slice) {
        const int block = 512 / size, most = (slice + 16 / size + block - 1) / block;
        return sizeof(Shared) + (most * 8 + 15) / 16 * 16 + (size_t)most * 512;
    };
    const auto slice_of = [&](int ctas) { return ((V + ctas - 1) / ctas + 7) / 8 * 8; };
    int c = 1;
    while (c < 8 && smem(slice_of(c)) > 112 * 1024) c *= 2;
    while (c < 8 && (long)rows * c * 2 <= 304 && slice_of(c * 2) >= 2048) c *= 2;
    return Cut{c, slice_of(c), smem(slice_of(c))};
}

template <typename... K, typename... A>
static cudaError_t launch_rows(void (*kernel)(K...), int rows, const Cut &c, cudaStream_t s, A... args) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)rows * c.ctas);
    lc.blockDim = ROW_THREADS;
    lc.dynamicSmemBytes = c.smem;
    lc.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = c.ctas;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = programmatic(s) ? 2 : 1;
    e = cudaLaunchKernelEx(&lc, kernel, K(args)...);
    note_launch();
    return e;
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
    const Cut c = cut_rows(rows, vocab, dtype == MSD_F32 ? 4 : 2);
    if ((long)rows * c.ctas > 0x7FFFFFFF) return MSD_ERR_INVALID;
    const cudaError_t e =
        dtype == MSD_F32
            ? launch_rows(sample_kernel<float>, rows, c, st, static_cast<const float *>(logits), (long)ld, vocab, c.ctas, c.slice, s, u,
                          tokens, logp, probs, (long)ldp)
            : launch_rows(sample_kernel<bf16>, rows, c, st, static_cast<const bf16 *>(logits), (long)ld, vocab, c.ctas, c.slice, s, u,
                          tokens, logp, probs, (long)ldp);
    return e == cudaSuccess ? MSD_OK : MSD_ERR_CUDA;
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
        const Cut c = cut_rows(batch->rows, vocab, dtype == MSD_F32 ? 4 : 2);
        if ((long)batch->rows * c.ctas > 0x7FFFFFFF) return MSD_ERR_INVALID;
        const cudaError_t e =
            dtype == MSD_F32
                ? launch_rows(accept_rows_kernel<float>, batch->rows, c, st, static_cast<const float *>(logits), (long)ld, vocab, c.ctas,
                              c.slice, s, a)
                : launch_rows(accept_rows_kernel<bf16>, batch->rows, c, st, static_cast<const bf16 *>(logits), (long)ld, vocab, c.ctas,
                              c.slice, s, a);
        if (e != cudaSuccess) return MSD_ERR_CUDA;
    }
    if (launch_chain(accept_walk_kernel, (batch->n + 31) / 32, 32, 0, st, a) != cudaSuccess) return MSD_ERR_CUDA;
    note_launch();
    return MSD_OK;
}

}  // extern "C"
