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
// decide; so nothing depends on how logits are spread. Where few tokens come before the bucket's end, all are gathered in one
// CTA, and the rest is done on that list; else sums of blocks of 128 ids lead to the token.
//
// What bounds it: for one row its phases in turn, 4 of them meetings of the cluster (a row of 32000 fp32 logits, top-k 50, top-p
// 0.9: 12 to 13 us); for many, issue slots, 60 to 70 instructions a token for each pass with exact weights, two of them for top-p of
// a row that leaves many tokens (64 rows of 100003 bf16 logits, top-p 0.95: 60 us in a graph, 61% of slots), 35 for a pass that counts.
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
constexpr int MAX_DEPTH = 1 << 20;
constexpr int MAX_TREE_ROWS = 1 << 30;          // and sequences: a loop's next index, and the sum of two, stay in 32 bits

__device__ __forceinline__ float logit_at(const float *row, int i) { return row[i]; }
__device__ __forceinline__ float logit_at(const bf16 *row, int i) { return __bfloat162float(row[i]); }

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

// The settings of a row: what they say, and the scale log2(e) / temperature as a pair.
struct RowSettings {
    float temperature, top_p, min_p, c_hi, c_lo;
    int top_k;                // 1: the first token alone; 0: off
    u64 least;
    __device__ __forceinline__ void request(const Settings &f, int at) {
        temperature = f.temperature ? f.temperature[at] : 1.f;
        top_k = f.top_k ? f.top_k[at] : 0;
        top_p = f.top_p ? f.top_p[at] : 1.f;
        min_p = f.min_p ? f.min_p[at] : 0.f;
    }
    __device__ __forceinline__ void prepare() {
        if (!(temperature >= 0x1p-100f) || min_p > 1.f || top_p <= 0.f) top_k = 1;
        const float t = temperature > 0.f ? fminf(fmaxf(temperature, 0x1p-100f), 0x1p100f) : 1.f;
        // (the remainder of the division is exact; in fp64, a few lanes a cycle, it took 3 us)
        constexpr float LOG2E = 1.44269504088896340736f, LOG2E_LO = (float)(1.44269504088896340736 - (double)1.44269504088896340736f);
        c_hi = __fdiv_rn(LOG2E, t);
        c_lo = __fdiv_rn(fmaf(-c_hi, t, LOG2E) + LOG2E_LO, t);
        least = !(min_p > 0.f) ? 0 : min_p < 1.f ? share_floor(min_p, 1ull << WEIGHT_BITS, true) : 1ull << WEIGHT_BITS;
    }
};

// What is left of a row: logits above `end`, and of the ids with just this logit the ones up to `tie`.
struct Left {
    RowScale scale;
    float end;
    int tie;
    u64 least;                // smallest weight (min-p)
    u64 total;                // its weight; 0: nothing is left

    // (NaN and -inf are in no run: it starts at -inf with no id)
    __device__ __forceinline__ bool has(float x, int id) const { return x > end | (x == end & id <= tie); }
};

// Weight of a token of a run, without min-p.
__device__ __forceinline__ u64 weight_in(const RowScale &r, float x, const float2 *table) {
    return weight_of(exponent_of(x, r), table);
}

// A row whose largest logit is +inf counts as one of zeros at its infinities and -inf elsewhere.
__device__ __forceinline__ float tame(float x, bool infinite) { return !infinite ? x : x == INFINITY ? 0.f : -INFINITY; }

__device__ __forceinline__ u64 weight_left(const Left &l, float x, int id, const float2 *table) {
    const u64 w = weight_in(l.scale, x, table);         // (no branch: several are under way at once)
    return l.has(x, id) && w >= l.least ? w : 0;
}

// ---------------------------------------------------------------------------
// A row over the CTAs of a cluster
//
// The code is kept short (functions that are called, state of the row in shared memory, loops over
// single elements): with everything inlined and unrolled, warps waited for instructions half of the time.
// ---------------------------------------------------------------------------
// A token of a list: order_of() it, and its weight.
struct __align__(16) Token {
    u64 order, w;
};
// Larger for a token that comes earlier in the order (larger logit, then lower id).
__device__ __forceinline__ u64 order_of(float x, int id) { return (u64)key_of(x) << 32 | (unsigned)~id; }
__device__ __forceinline__ float logit_of_order(u64 o) { return logit_of((unsigned)(o >> 32)); }
__device__ __forceinline__ int id_of_order(u64 o) { return (int)~(unsigned)o; }

struct __align__(16) Shared {                   // (the sums and the slice lie behind it)
    float2 table[EXP_STEPS];
    union {
        unsigned hist[3][BUCKETS];              // own: counts, or masses in pieces of 15, 15 and 14 bits
        struct {                                // once they are added up: tokens gathered, of the row and of the slice
            Token list[LIST];
            u64 own[LIST];
        };
    };
    u64 all[BUCKETS];                           // of the whole row; 0 between uses
    u64 red[WARPS + 1];
    u64 total[8];                               // of each CTA of the cluster
    float top[8], low[8];
    u64 above, left;
    double log_total;
    unsigned bucket, own_n[2], list_n[2], base[8];            // (a round may gather twice)
    unsigned range_lo, range_hi;                // keys of a bucket's tokens
    float end;
    int tie;
    int next, gones, gone[MAX_CHILDREN];
    unsigned short kid[MAX_CHILDREN];           // children of a node, and their tokens
    int kid_token[MAX_CHILDREN];
    // the slice: ids [first, first + count), element i of it at data[mis + i], -inf around it, in whole blocks
    int ctas, rank, first, count, mis, blocks, data_at;
};
constexpr int BLOCK = 128;                      // ids that have a sum of their own

extern __shared__ __align__(16) uint8_t g_smem[];
__device__ __forceinline__ Shared &shared() { return *reinterpret_cast<Shared *>(g_smem); }
__device__ __forceinline__ u64 *block_sums() { return reinterpret_cast<u64 *>(g_smem + sizeof(Shared)); }
template <typename T> __device__ __forceinline__ T *slice_data() { return reinterpret_cast<T *>(g_smem + shared().data_at); }
constexpr size_t data_offset(int blocks) { return sizeof(Shared) + (size_t)(blocks * 8 + 15) / 16 * 16; }
constexpr int most_blocks(int slice, int size) { return (slice + 16 / size + BLOCK - 1) / BLOCK; }

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

__device__ __forceinline__ void meet() {        // of all threads of the row
    if (shared().ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
}
template <typename U> __device__ __forceinline__ void tell(U *p, U v) {                    // one thread: to every CTA
    for (int r = 0; r < shared().ctas; ++r) put(p, r, v);
}

struct Extent {               // of the row's logits above -inf
    float top, low;           // low: about the smallest (of a part of them)
    bool infinite;            // the largest was +inf; the slice holds what tame() gives
};

// A lane's 4 of the 128 ids of a block.
template <typename T> __device__ __forceinline__ void block_logits(int b, float (&x)[4]) {
    const int at = b * 32 + (threadIdx.x & 31);
    if constexpr (sizeof(T) == 4) {
        const float4 q = slice_data<float4>()[at];
        x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
    } else {
        const uint2 q = slice_data<uint2>()[at];
        x[0] = __uint_as_float(q.x << 16); x[1] = __uint_as_float(q.x & 0xFFFF0000u);
        x[2] = __uint_as_float(q.y << 16); x[3] = __uint_as_float(q.y & 0xFFFF0000u);
    }
}

// f(logit, id) for every logit of the slice, whole warps at a time; around it there is -inf.
template <typename T, typename F>
__device__ __forceinline__ void each(F f) {
    Shared &sh = shared();
    const int blocks = sh.blocks, id0 = sh.first - sh.mis + (int)(threadIdx.x & 31) * 4;
#pragma unroll 1
    for (int b = threadIdx.x >> 5; b < blocks; b += WARPS) {
        float x[4];
        block_logits<T>(b, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) f(x[e], id0 + b * BLOCK + e);
    }
}

// This CTA's slice into shared memory, and the row's extent. meanwhile(): done while the first of it is on its way.
template <typename T, typename F>
__device__ __forceinline__ Extent load_row(const T *row, int V, int ctas, int rank, int slice, F meanwhile) {
    constexpr int E = 16 / sizeof(T), U = 4;
    Shared &sh = shared();
    const int tid = threadIdx.x, warp = tid >> 5;
    if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int first = min(rank * slice, V), count = min(slice, V - first);
    const int mis = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));               // slices are multiples of 16 bytes
    const int blocks = (mis + count + BLOCK - 1) / BLOCK;
    const int data_at = (int)data_offset(most_blocks(slice, sizeof(T)));
    T *const data = reinterpret_cast<T *>(g_smem + data_at);
    const T *const from = row + first - mis;                                                // 16-byte aligned
    const int v0 = mis ? 1 : 0, v1 = max((mis + count) / E, v0);                            // whole vectors
    const uint4 table = reinterpret_cast<const uint4 *>(g_exp_table.pair)[tid];
    float hi = -INFINITY, lo = INFINITY;
    const auto low = [&](float x) { lo = x > -INFINITY ? fminf(lo, x) : lo; };
    uint4 q[U];
    const auto request = [&](int v) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v + u * ROW_THREADS < v1) q[u] = __ldcs(reinterpret_cast<const uint4 *>(from) + v + u * ROW_THREADS);
    };
    request(v0 + tid);
    meanwhile();
    // what a cut starts with
    for (int i = tid; i < 3 * BUCKETS; i += ROW_THREADS) (&sh.hist[0][0])[i] = 0;
    for (int i = tid; i < BUCKETS; i += ROW_THREADS) sh.all[i] = 0;
    if (tid < 2) sh.own_n[tid] = sh.list_n[tid] = 0;
    if (tid == 0) {
        sh.ctas = ctas; sh.rank = rank; sh.first = first; sh.count = count; sh.mis = mis; sh.blocks = blocks; sh.data_at = data_at;
        sh.range_lo = ~0u;
        sh.range_hi = 0;
    }
    // the edges: elements before the first whole vector and behind the last one
    for (int i = tid; i < v0 * E + blocks * BLOCK - v1 * E; i += ROW_THREADS) {
        const int at = i < v0 * E ? i : i - v0 * E + v1 * E;
        const bool is = at >= mis && at < mis + count;
        const float x = is ? logit_at(from, at) : -INFINITY;
        data[at] = (T)x;
        hi = fmaxf(hi, x);
        low(x);
    }
    for (int v = v0 + tid; v < v1;) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (v + u * ROW_THREADS >= v1) break;
            reinterpret_cast<uint4 *>(data)[v + u * ROW_THREADS] = q[u];
            const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {                                                   // (fmaxf leaves NaN out)
                if constexpr (E == 4) {
                    hi = fmaxf(hi, __uint_as_float(w[e]));
                } else {
                    hi = fmaxf(hi, fmaxf(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xFFFF0000u)));
                }
            }
            if (u == 0) low(__uint_as_float(E == 4 ? w[0] : w[0] & 0xFFFF0000u));
        }
        v += U * ROW_THREADS;
        request(v);
    }
    reinterpret_cast<uint4 *>(sh.table)[tid] = table;
    static_assert(EXP_STEPS * 8 == ROW_THREADS * 16, "");
    hi = warp_max(hi);
    lo = -warp_max(-lo);
    float *part = reinterpret_cast<float *>(sh.gone);                                       // (not in use yet)
    if ((tid & 31) == 0) { part[warp] = hi; part[32 + warp] = lo; }
    if (ctas > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");               // all CTAs run: their shared memory is there
    __syncthreads();
    if (tid < 32) {
        hi = warp_max(tid < WARPS ? part[tid] : -INFINITY);
        lo = -warp_max(tid < WARPS ? -part[32 + tid] : -INFINITY);
        if (tid < ctas) {
            put(&sh.top[rank], tid, hi);
            put(&sh.low[rank], tid, lo);
        }
    }
    meet();
    Extent e{-INFINITY, INFINITY, false};
    for (int r = 0; r < ctas; ++r) {
        e.top = fmaxf(e.top, sh.top[r]);
        e.low = fminf(e.low, sh.low[r]);
    }
    if (e.top == INFINITY) {
        e = Extent{0.f, 0.f, true};
        for (int i = tid; i < blocks * BLOCK; i += ROW_THREADS) data[i] = (T)tame(logit_at(data, i), true);
        __syncthreads();
    }
    e.low = fminf(e.low, e.top);
    return e;
}

// What a token counts for: its weight, or, to count equal logits, 1 for the ids of `l` that have just l.end.
__device__ __forceinline__ u64 value_of(const Left &l, bool ties, float x, int id, const float2 *table) {
    return ties ? (u64)(x == l.end && id <= l.tie) : weight_left(l, x, id, table);
}

// Sums of value_of over each block, this CTA's, and all (returned).
template <typename T>
__device__ __noinline__ u64 add_up(const Left l, bool ties) {
    Shared &sh = shared();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, id0 = sh.first - sh.mis + lane * 4, blocks = sh.blocks;
    u64 sum = 0;
#pragma unroll 1
    for (int b = warp; b < blocks; b += WARPS) {
        float x[4];
        block_logits<T>(b, x);
        const int id = id0 + b * BLOCK;
        const bool any = l.has(x[0], id) || l.has(x[1], id + 1) || l.has(x[2], id + 2) || l.has(x[3], id + 3);
        u64 v = 0;
        if (__any_sync(0xffffffffu, any)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v += value_of(l, ties, x[e], id + e, sh.table);
            // less than 2^46 a lane: three sums of 16 bits
            const u64 lo = __reduce_add_sync(0xffffffffu, (unsigned)v & 0xFFFFu), mid = __reduce_add_sync(0xffffffffu, (unsigned)v >> 16),
                      hi = __reduce_add_sync(0xffffffffu, (unsigned)(v >> 32));
            v = lo + (mid << 16) + (hi << 32);
        }
        if (lane == 0) block_sums()[b] = v;
        sum += v;
    }
    __syncthreads();
    if (lane == 0) sh.red[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        sum = warp_total(lane < WARPS ? sh.red[lane] : 0);
        if (lane < sh.ctas) put(&sh.total[sh.rank], lane, sum);
    }
    meet();
    u64 all = 0;
    for (int r = 0; r < sh.ctas; ++r) all += sh.total[r];
    return all;
}

// After add_up: the smallest id whose cumulative value exceeds `goal`, which is less than the whole; tokens
// gone[0 .. gones) count for nothing. One thread of one CTA gets it, the others -1.
template <typename T>
__device__ __noinline__ int locate(const Left l, bool ties, u64 goal, int gones) {
    Shared &sh = shared();
    u64 rest = goal;
    for (int r = 0; r < sh.rank; ++r) {
        if (rest < sh.total[r]) return -1;
        rest -= sh.total[r];
    }
    if (rest >= sh.total[sh.rank] || threadIdx.x >= 32) return -1;
    const int lane = threadIdx.x, blocks = sh.blocks;
    const auto scan = [&](u64 v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 t = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += t;
        }
        return v;
    };
    int b = 0;
    for (int b0 = 0; b0 < blocks; b0 += 32) {                               // the 32 blocks, then the one
        const u64 own = b0 + lane < blocks ? block_sums()[b0 + lane] : 0, in = scan(own);
        const unsigned over = __ballot_sync(0xffffffffu, in > rest);
        if (over) {
            const int at = __ffs(over) - 1;
            rest -= __shfl_sync(0xffffffffu, in - own, at);
            b = b0 + at;
            break;
        }
        rest -= __shfl_sync(0xffffffffu, in, 31);
    }
    const int id = sh.first - sh.mis + b * BLOCK + lane * 4;
    float x[4];
    block_logits<T>(b, x);
    u64 v[4], own = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = value_of(l, ties, x[e], id + e, sh.table);
        for (int g = 0; g < gones; ++g)
            if (sh.gone[g] == id + e) v[e] = 0;
        own += v[e];
    }
    u64 upto = scan(own) - own;
    int found = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (upto <= rest && rest < upto + v[e]) found = id + e;
        upto += v[e];
    }
    return found;
}

// Larger values first: thread i gets the i-th of the block's. n of them are not 0.
__device__ u64 sorted(u64 v, unsigned n) {
    u64 *const buf = shared().own;                                          // (sent by now)
    const unsigned tid = threadIdx.x;
    unsigned size = 32;
    while (size < n) size *= 2;
#pragma unroll 1
    for (unsigned k = 2; k <= size; k *= 2)
#pragma unroll 1
        for (unsigned j = k / 2; j > 0; j /= 2) {
            u64 o;
            if (j < 32) {
                o = __shfl_xor_sync(0xffffffffu, v, j);
            } else {
                __syncthreads();
                buf[tid] = v;
                __syncthreads();
                o = buf[tid ^ j];
            }
            const bool larger = ((tid & j) == 0) == ((tid & k) == 0 || k == size);
            v = (o > v) == larger ? o : v;
        }
    return v;
}

// Sum over the threads up to this one, and of all.
__device__ u64 sum_up_to(u64 v, u64 *all) {
    Shared &sh = shared();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    __syncthreads();
    if (lane == 31) sh.red[warp] = v;
    __syncthreads();
    static_assert(WARPS == 16, "");
    u64 sum = sh.red[lane & 15];                        // every warp adds the warps' sums up
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
        const u64 t = __shfl_up_sync(0xffffffffu, sum, o);
        if ((lane & 15) >= o) sum += t;
    }
    *all = __shfl_sync(0xffffffffu, sum, 15);
    const u64 before = __shfl_sync(0xffffffffu, sum, max(warp - 1, 0));
    return warp ? v + before : v;
}

// The list's n tokens by order, or by id: thread i gets the i-th. Up to 256 by counting, with all threads, how many come before each,
// more by sorting (for 64 tokens counting takes 1 us less, for 512 3 us more). The weights come along only by id.
template <bool BY_ID>
__device__ __noinline__ Token ordered(int n) {
    Shared &sh = shared();
    const unsigned tid = threadIdx.x;
    if (n > LIST / 2) {
        const u64 o = tid < (unsigned)n ? sh.list[tid].order : 0;
        if constexpr (BY_ID) {                          // (the order's lower half is larger for a lower id)
            const u64 at = sorted(o << 32 | tid, n);
            return tid < (unsigned)n ? sh.list[(unsigned)at] : Token{0, 0};
        } else {
            return Token{sorted(o, n), 0};
        }
    }
    const int bits = min(5, __clz(max(n - 1, 1)) - 23), per = 1 << bits;    // 512 / per >= n
    const int i = (int)tid >> bits, part = (int)tid & (per - 1);
    int rank = 0;
    Token own{0, 0};
    if (i < n) {
        own = sh.list[i];
#pragma unroll 4
        for (int j = part; j < n; j += per) {
            const u64 o = sh.list[j].order;
            rank += BY_ID ? (unsigned)o > (unsigned)own.order : o > own.order;
        }
    }
    for (int o = 1; o < per; o *= 2) rank += __shfl_xor_sync(0xffffffffu, rank, o);
    __syncthreads();
    if (i < n && part == 0) sh.list[rank] = own;
    __syncthreads();
    return tid < (unsigned)n ? sh.list[tid] : Token{0, 0};
}

// A run of few tokens, gathered in the first CTA: what top-k, top-p and min-p leave of it. mass: the weight that top-p's
// share is taken of, where top-k is off. The list's weights become what is left of them.
__device__ __noinline__ Left rest_of_list(Left l, int n, int k, float p, u64 mass) {
    Shared &sh = shared();
    const int i = threadIdx.x;
    const u64 order = ordered<false>(n).order;
    const u64 w = i < n ? weight_in(l.scale, logit_of_order(order), sh.table) : 0;
    bool in = i < n && (k <= 0 || i < k);
    if (p < 1.f) {
        u64 all;
        const u64 before = sum_up_to(in ? w : 0, &all) - w;                 // (of those that top-k leaves; i is one of them or out)
        in = in && before < max(share_floor(p, k > 0 ? all : mass, true), 1ull);
    }
    // the run's end: min-p, which goes by weights, may leave a hole in it (a lower logit's weight can be the larger one by a unit)
    const int left = __syncthreads_count(in);
    in = in && w >= l.least;
    sum_up_to(in ? w : 0, &l.total);
    if (i < n) sh.list[i] = Token{order, in ? w : 0};
    if (i == left - 1) { sh.end = logit_of_order(order); sh.tie = id_of_order(order); }
    __syncthreads();
    l.end = sh.end;
    l.tie = sh.tie;
    return l;
}

// The smallest id of the list whose cumulative weight exceeds `goal`; gone[0 .. gones) have none. One thread gets it, the others -1.
__device__ __noinline__ int locate_in_list(int n, u64 goal, int gones) {
    Shared &sh = shared();
    const int tid = threadIdx.x;
    if (gones) {
        if (tid < n)
            for (int g = 0; g < gones; ++g)
                if (sh.gone[g] == id_of_order(sh.list[tid].order)) sh.list[tid].w = 0;
        __syncthreads();
    }
    const Token t = ordered<true>(n);
    u64 all;
    const u64 upto = sum_up_to(t.w, &all);
    return upto - t.w <= goal && goal < upto ? id_of_order(t.order) : -1;
}

enum : int { ONE_TOKEN = 0, IN_LIST = 1, IN_ROW = 2 };        // what is left: l.tie alone; the first CTA's list; add_up's sums

// The bucket of a token of a run, BUCKETS for others: of equal width in the exponent, or (KEYS) in the bits of the keys from
// k_lo to k_hi. No branches, since a warp's tokens go all ways.
struct Places {
    float end, top, scale;
    int tie, shift;
    unsigned k_lo, k_hi;
    template <bool KEYS> __device__ __forceinline__ unsigned of(float x, int id) const {
        bool in = x > end | (x == end & id <= tie);
        unsigned b;
        if constexpr (KEYS) {
            const unsigned k = key_of(x);
            in = in & (k >= k_lo) & (k <= k_hi);
            b = (k_hi - k) >> shift;
        } else {
            b = __float_as_uint(fminf((top - x) * scale, (float)(BUCKETS - 1)) + 12582912.f) & (2 * BUCKETS - 1);
        }
        return in ? b : BUCKETS;
    }
};

// This CTA's histogram of counts or of masses (weights by `scale`).
template <typename T, bool KEYS, bool MASS>
__device__ __noinline__ void histogram(const Places p, const RowScale scale) {
    Shared &sh = shared();
    each<T>([&](float x, int id) {
        const unsigned b = p.of<KEYS>(x, id);
        if constexpr (MASS) {
            const u64 w = weight_in(scale, x, sh.table);
            if (b == BUCKETS) return;
            atomicAdd(&sh.hist[0][b], (unsigned)w & 0x7FFFu);
            atomicAdd(&sh.hist[1][b], (unsigned)(w >> 15) & 0x7FFFu);
            atomicAdd(&sh.hist[2][b], (unsigned)(w >> 30));
        } else {
            if (b != BUCKETS) atomicAdd(&sh.hist[0][b], 1u);
        }
    });
}

// Tokens of the places from `first` to `last` into the first CTA's list, or (all_lists) every CTA's; their number, which may
// be more than the list has. `which`: 0 or 1, the counters (zero before the last meeting).
template <typename T, bool KEYS>
__device__ __noinline__ unsigned gather(int which, const Places p, unsigned first, unsigned last, bool all_lists) {
    Shared &sh = shared();
    const int tid = threadIdx.x, lane = tid & 31, ctas = sh.ctas, id0 = sh.first - sh.mis + lane * 4, blocks = sh.blocks;
#pragma unroll 1
    for (int b = tid >> 5; b < blocks; b += WARPS) {
        float x[4];
        block_logits<T>(b, x);
        unsigned in = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            in |= (unsigned)(p.of<KEYS>(x[e], id0 + b * BLOCK + e) - first <= last - first) << e;       // (last < BUCKETS)
        }
        if (!__any_sync(0xffffffffu, in)) continue;
        if (in == 0 || *(volatile unsigned *)&sh.own_n[which] > LIST) continue;     // (too many already: how many does not matter)
        unsigned slot = atomicAdd(&sh.own_n[which], __popc(in));
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (in >> e & 1) {
                if (slot < LIST) sh.own[slot] = order_of(x[e], id0 + b * BLOCK + e);
                ++slot;
            }
    }
    __syncthreads();
    const unsigned own_n = sh.own_n[which];
    if (own_n && tid < ctas) sh.base[tid] = take(&sh.list_n[which], tid, own_n);
    __syncthreads();
    for (unsigned i = tid; i < min(own_n, (unsigned)LIST); i += ROW_THREADS)
        for (int r = 0; r < (all_lists ? ctas : 1); ++r) {
            const unsigned slot = sh.base[r] + i;
            if (slot < LIST) put(&sh.list[slot].order, r, sh.own[i]);
        }
    meet();
    return sh.list_n[which];
}

// Where the run of tokens of `l` ends whose count (mass false) reaches `goal`, or whose weight reaches the share `p` of
// theirs (mass true): a narrower l. x_end is about its smallest logit. Every CTA finds it by itself from the whole row's
// histogram and the bucket's tokens, which all are sent. Where few tokens lie before the bucket's end, they are gathered instead
// (*mode becomes IN_LIST, *n their number) and l.total is the weight that p is a share of; nothing else of l changes then.
// fresh: the first cut of the row.
template <typename T>
__device__ __noinline__ Left cut(Left l, bool mass, bool fresh, u64 goal, float p, float x_end, int *mode, unsigned *list_n) {
    Shared &sh = shared();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, ctas = sh.ctas;
    // buckets of equal width in the exponent between the largest logit and x_end; from the second round on, of the keys' bits
    const float y_end = fminf((l.scale.top - x_end) * l.scale.c_hi, Y_MOST);
    const float scale = y_end > 0.f ? (float)(BUCKETS - 1) / y_end * l.scale.c_hi : 0.f;
    u64 above = 0;
    Places places{l.end, l.scale.top, scale, l.tie, 0, 0, ~0u};
    for (int round = 0;; ++round) {
        if (round > 0 || !fresh) {
            for (int i = tid; i < (mass ? 3 : 1) * BUCKETS; i += ROW_THREADS) (&sh.hist[0][0])[i] = 0;
            if (tid < 2) sh.own_n[tid] = sh.list_n[tid] = 0;
            if (tid == 2) { sh.range_lo = ~0u; sh.range_hi = 0; }
            __syncthreads();
        }
        if (round == 0) mass ? histogram<T, false, true>(places, l.scale) : histogram<T, false, false>(places, l.scale);
        else mass ? histogram<T, true, true>(places, l.scale) : histogram<T, true, false>(places, l.scale);
        __syncthreads();
        for (int i = tid; i < BUCKETS; i += ROW_THREADS) {
            const u64 v = mass ? sh.hist[0][i] + ((u64)sh.hist[1][i] << 15) + ((u64)sh.hist[2][i] << 30) : sh.hist[0][i];
            if (ctas == 1) sh.all[i] = v;
            else if (v)
                for (int r = 0; r < ctas; ++r) add(&sh.all[i], r, v);
        }
        meet();
        // the bucket that the bound falls into
        constexpr int PER = BUCKETS / ROW_THREADS;
        u64 v[PER], run = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            v[i] = sh.all[tid * PER + i];
            sh.all[tid * PER + i] = 0;                                      // (the next time that it is added to lies behind a meeting)
            run += v[i];
        }
        const u64 own = run;
        u64 all;
        run = sum_up_to(run, &all);
        if (round == 0) {
            if (mass) goal = max(share_floor(p, all, true), 1ull);
            else if (all <= goal) {                                         // it has no more tokens than that
                meet();
                return l;
            }
        }
        u64 at = above + run - own;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (at < goal && goal <= at + v[i]) { sh.bucket = tid * PER + i; sh.above = at; sh.left = at + v[i]; }
            at += v[i];
        }
        __syncthreads();
        const unsigned bucket = sh.bucket;
        above = sh.above;
        // few tokens? (by mass: about as many as the buckets' masses are weights of their ends)
        bool few_before = round == 0 && sh.left <= LIST;
        if (round == 0 && mass) {
            float about = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (tid * PER + i <= bucket) about += (float)v[i] * exp2f((float)(tid * PER + i) * (y_end / (BUCKETS - 1)) - WEIGHT_BITS);
            u64 sum;
            sum_up_to((u64)fminf(16.f * about, 1e9f), &sum);
            few_before = sum < 16 * LIST;
        }
        if (few_before) {
            const unsigned n = gather<T, false>(0, places, 0, bucket, false);
            if (n <= LIST) {
                l.total = mass ? all : 0;
                *mode = IN_LIST;
                *list_n = n;
                return l;
            }
        }
        const unsigned n = round == 0 ? gather<T, false>(1, places, bucket, bucket, true) : gather<T, true>(1, places, bucket, bucket, true);
        const bool few = n <= LIST;
        if (!few) {                                                         // the range of their keys
            unsigned lo = ~0u, hi = 0;
            each<T>([&](float x, int id) {
                if ((round == 0 ? places.of<false>(x, id) : places.of<true>(x, id)) != bucket) return;
                lo = min(lo, key_of(x));
                hi = max(hi, key_of(x));
            });
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            if (hi && lane < ctas) { least(&sh.range_lo, lane, lo); most(&sh.range_hi, lane, hi); }
            meet();
            places.k_lo = sh.range_lo;
            places.k_hi = sh.range_hi;
        }
        if (!few && places.k_lo != places.k_hi) {
            places.shift = max(0, 22 - __clz(places.k_hi - places.k_lo));   // (k_hi - k_lo) >> shift < BUCKETS
            __syncthreads();                                                // all have read the list's length and the range
            continue;
        }
        if (few) {                                                          // each token's place among them
            const u64 order = ordered<false>((int)n).order;
            const u64 w = tid >= (int)n ? 0 : mass ? weight_in(l.scale, logit_of_order(order), sh.table) : 1;
            u64 sum;
            const u64 upto = above + sum_up_to(w, &sum);
            if (upto - w < goal && goal <= upto) { sh.end = logit_of_order(order); sh.tie = id_of_order(order); }
        } else {                                                            // equal logits: ids decide
            const float x = logit_of_order(sh.list[0].order);
            const u64 w = !mass ? 1 : max(weight_in(l.scale, x, sh.table), 1ull), need = (goal - above + w - 1) / w;
            if (l.end < x) l.tie = 0x7FFFFFFF;
            l.end = x;
            add_up<T>(l, true);
            const int id = locate<T>(l, true, need - 1, 0);
            if (id >= 0) {
                tell(&sh.end, x);
                tell(&sh.tie, id);
            }
            meet();
        }
        __syncthreads();
        l.end = sh.end;
        l.tie = sh.tie;
        return l;
    }
}

// What a row's settings leave of it: *mode, with IN_LIST in the first CTA alone (the others get a total of 0), *n
// tokens in its list. whole: every CTA gets to know l in that case too.
template <typename T>
__device__ __forceinline__ Left filter_row(const Extent &e, const RowSettings &f, bool whole, int *mode, unsigned *n) {
    Shared &sh = shared();
    Left l;
    l.total = 0;
    l.end = -INFINITY;
    l.tie = -1;
    l.least = 0;
    l.scale = RowScale{e.top, 0.f, 0.f};
    *mode = ONE_TOKEN;
    if (e.top == -INFINITY) return l;
    l.scale.c_hi = f.c_hi;
    l.scale.c_lo = f.c_lo;
    int k = f.top_k;
    const float p = f.top_p;
    if (k == 1) {                                                           // the first token alone
        unsigned id = ~0u;
        each<T>([&](float x, int i) {
            if (x == e.top) id = min(id, (unsigned)i);
        });
        id = __reduce_min_sync(0xffffffffu, id);
        const int lane = threadIdx.x & 31;
        if (lane < sh.ctas && id != ~0u) least(&sh.range_lo, lane, id);
        meet();
        l.end = e.top;
        l.tie = (int)sh.range_lo;
        l.total = 1ull << WEIGHT_BITS;
        return l;
    }
    *mode = IN_ROW;
    l.least = f.least;
    bool fresh = true;
    float x_end = e.low;
#pragma unroll 1
    for (int by = 0; by < 2 && *mode == IN_ROW; ++by) {                     // top-k, then top-p
        if (by == 0 ? k <= 0 : !(p < 1.f)) continue;
        l = cut<T>(l, by == 1, fresh, (u64)k, p, x_end, mode, n);
        fresh = false;
        if (*mode == IN_LIST && by == 1) k = 0;                             // (top-k is behind it already)
        if (l.end > -INFINITY) x_end = l.end;
    }
    if (*mode == IN_ROW) {
        l.total = add_up<T>(l, false);
        return l;
    }
    const u64 mass = l.total;
    l.total = 0;
    if (sh.rank == 0) l = rest_of_list(l, (int)*n, k, p, mass);
    if (whole && sh.ctas > 1) {
        if (sh.rank == 0 && threadIdx.x == 0) {
            tell(&sh.end, l.end);
            tell(&sh.tie, l.tie);
            tell(&sh.left, l.total);
        }
        meet();
        l.end = sh.end;
        l.tie = sh.tie;
        l.total = sh.left;
    }
    return l;
}

__device__ __forceinline__ float uniform(float u) { return fminf(u > 0.f ? u : 0.f, 0x1.fffffep-1f); }

template <typename T>
__global__ void __launch_bounds__(ROW_THREADS, 2)
sample_kernel(const T *__restrict__ logits, long ld, int V, int ctas, int slice, Settings f, const float *__restrict__ u,
              int *__restrict__ tokens, float *__restrict__ logp, float *__restrict__ probs, long ldp) {
    wait_prior();
    allow_dependents();
    Shared &sh = shared();
    const int r = blockIdx.x / ctas, rank = blockIdx.x % ctas;
    const T *row = logits + (long)r * ld;
    RowSettings settings;
    settings.request(f, r);
    const float own_u = u[r];
    const Extent e = load_row(row, V, ctas, rank, slice, [&] { settings.prepare(); });
    int mode;
    unsigned n = 0;
    const Left l = filter_row<T>(e, settings, probs != nullptr, &mode, &n);
    // the thread that knows the token writes it
    if (mode == IN_LIST && rank > 0 && !probs) return;
    if (logp && threadIdx.x == 32) sh.log_total = mode == ONE_TOKEN ? 0.0 : log2((double)l.total) - WEIGHT_BITS;     // (a warp that is free)
    const u64 goal = share_floor(uniform(own_u), l.total, false);
    int t = -1;
    if (mode == ONE_TOKEN) t = l.tie;
    else if (mode == IN_ROW) t = locate<T>(l, false, goal, 0);
    else if (rank == 0) t = locate_in_list((int)n, goal, 0);
    __syncthreads();
    if (mode == ONE_TOKEN ? rank == 0 && threadIdx.x == 0 : t >= 0) {
        tokens[r] = t;
        if (logp) {
            const float2 y = t < 0 ? make_float2(0.f, 0.f) : exponent_of(tame(logit_at(row, t), e.infinite), l.scale);
            logp[r] = t < 0 ? -INFINITY : (float)(-0.69314718055994530942 * ((double)y.x + (double)y.y + sh.log_total));
        }
    }
    if (probs) {
        const float scale = l.total ? (float)(0x1p44 / (double)l.total) : 0.f;
        const T *data = slice_data<T>() + sh.mis;
        float *to = probs + (long)r * ldp + sh.first;
        for (int i = threadIdx.x; i < sh.count; i += ROW_THREADS) {
            const float x = logit_at(data, i);
            float w = 0.f;
            if (l.has(x, sh.first + i)) {
                const float2 y = exponent_of(x, l.scale);
                if (y.x < 160.f && (l.least == 0 || weight_in(l.scale, x, sh.table) >= l.least)) w = exp2f(-y.x) * (1.f - 0.69314718f * y.y) * scale;
            }
            to[i] = w;
        }
    }
}

// Trees, and what becomes of their nodes: outcome[row] is the child that is accepted there, or -2 - the token drawn there.
struct TreeArgs {
    int n, rows, nodes, depth, children, ahead;
    const int *row_start, *tokens, *parent, *n_nodes;
    const float *u;
    int *outcome, *list;      // [rows]: see accept_plan_kernel
    int *path, *accept_len, *bonus;
};

__device__ __forceinline__ int nodes_of(const TreeArgs &a, int b) {
    const int start = a.row_start[b], rows = min(min(a.row_start[b + 1], a.rows) - start, a.nodes);
    return start < 0 ? 0 : a.n_nodes ? min(rows, a.n_nodes[b]) : rows;
}

struct Node {
    int b, node, n, d;        // its sequence, its index among n, drafts accepted there (more than depth: never reached)
};
__device__ __forceinline__ Node node_of(const TreeArgs &a, int r) {
    Node t{0, 0, 0, 0};
    for (int hi = a.n; hi - t.b > 1;) {                 // the last sequence that starts at or before the row
        const int mid = (t.b + hi) >> 1;
        if (a.row_start[mid] <= r) t.b = mid; else hi = mid;
    }
    t.node = r - a.row_start[t.b];
    t.n = nodes_of(a, t.b);
    if (t.node < 0 || t.node >= t.n) t.d = a.depth + 1;
    return t;
}
__device__ __forceinline__ void find_depth(const TreeArgs &a, Node &t) {
    const int *parent = a.parent + (long)t.b * a.nodes;
    for (int i = t.node; i > 0 && t.d <= a.depth; ++t.d) {
        const int up = parent[i];
        if (up < 0 || up >= i) { t.d = a.depth + 1; break; }
        i = up;
    }
}

// What becomes of a node whose parent is accepted.
template <typename T>
__device__ __forceinline__ void decide(const T *__restrict__ logits, long ld, int V, int ctas, int rank, int slice, const Settings &f,
                                       const TreeArgs &a, int r, const Node &t) {
    Shared &sh = shared();
    const int lane = threadIdx.x & 31, b = t.b, node = t.node, n = t.n, d = t.d;
    const int *parent = a.parent + (long)b * a.nodes, *tokens = a.tokens + (long)b * a.nodes;
    const T *row = logits + (long)r * ld;
    RowSettings settings;
    settings.request(f, b);
    const float *u = a.u + ((long)b * (a.depth + 1) + d) * (a.children + 1);
    const float last_u = u[a.children];
    int kids = 0;                                       // of the first CTA's first warp
    const Extent e = load_row(row, V, ctas, rank, slice, [&] {
        settings.prepare();
        // the first `children` children, in index order
        if (rank == 0 && threadIdx.x < 32 && d < a.depth)
            for (int j0 = node + 1; j0 < n && kids < a.children; j0 += 32) {
                const int j = j0 + lane;
                const bool is = j < n && parent[j] == node;
                const unsigned all = __ballot_sync(0xffffffffu, is);
                const int slot = kids + __popc(all & ((1u << lane) - 1u));
                if (is && slot < a.children) {
                    sh.kid[slot] = (unsigned short)j;
                    sh.kid_token[slot] = tokens[j];
                }
                kids = min(kids + __popc(all), a.children);
            }
    });
    int mode;
    unsigned in_list = 0;
    const Left l = filter_row<T>(e, settings, false, &mode, &in_list);
    if (mode == IN_LIST) {                              // the first CTA goes on alone
        if (rank > 0) return;
        __syncthreads();
        if (threadIdx.x == 0) sh.ctas = 1;
        __syncthreads();
    }
    const int ranks = sh.ctas;
    if (rank == 0 && threadIdx.x < 32) {
        // A child is tried when those before it are rejected, so its odds are known: 32 children at a time. A token that an
        // earlier child had has no weight left.
        u64 left = l.total;
        int gone = 0, next = -1;
        __syncwarp();
        for (int c0 = 0; c0 < kids && next < 0; c0 += 32) {
            const int c = c0 + lane, t = c < kids ? sh.kid_token[c] : -1 - lane;
            const float v = c < kids ? u[c] : 0.f;
            u64 w = t >= 0 && t < V && l.total ? weight_left(l, tame(logit_at(row, t), e.infinite), t, sh.table) : 0;
            if (__match_any_sync(0xffffffffu, t) & ((1u << lane) - 1u)) w = 0;
            for (int i = 0; i < gone; ++i)
                if (sh.gone[i] == t) w = 0;
            u64 upto = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 before = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += before;
            }
            const unsigned yes = __ballot_sync(0xffffffffu, c < kids && share_floor(uniform(v), left - (upto - w), false) < w);
            const unsigned tried = yes ? (1u << (__ffs(yes) - 1)) - 1u : 0xffffffffu;       // (and rejected)
            const unsigned less = __ballot_sync(0xffffffffu, w != 0) & tried;
            if (less >> lane & 1) sh.gone[gone + __popc(less & ((1u << lane) - 1u))] = t;
            gone += __popc(less);
            if (yes) next = sh.kid[c0 + __ffs(yes) - 1];
            left -= __shfl_sync(0xffffffffu, upto, 31);                                     // (not used any more if one is accepted)
            __syncwarp();
        }
        if (lane < ranks) {
            put(&sh.next, lane, next);
            put(&sh.gones, lane, gone);
            put(&sh.left, lane, left);
        }
        for (int p = 1; p < ranks; ++p)
            for (int i = lane; i < gone; i += 32) put(&sh.gone[i], p, sh.gone[i]);
    }
    meet();
    if (sh.next >= 0) {
        if (rank == 0 && threadIdx.x == 0) a.outcome[r] = sh.next;
        return;
    }
    const int gones = sh.gones;
    const u64 left = sh.left;
    if (mode == ONE_TOKEN || left == 0) {
        if (rank == 0 && threadIdx.x == 0) a.outcome[r] = left ? -2 - l.tie : -1;
        return;
    }
    const u64 goal = share_floor(uniform(last_u), left, false);
    if (mode == IN_ROW && gones) {                      // the sums without the rejected tokens
        if (threadIdx.x == 0) {
            u64 less = 0;
            for (int g = 0; g < gones; ++g) {
                const int i = sh.gone[g] - sh.first;
                if (i < 0 || i >= sh.count) continue;
                const u64 v = weight_left(l, logit_at(slice_data<T>(), sh.mis + i), sh.gone[g], sh.table);
                block_sums()[(sh.mis + i) / BLOCK] -= v;
                less += v;
            }
            if (less) tell(&sh.total[rank], sh.total[rank] - less);
        }
        meet();
    }
    const int id = mode == IN_ROW ? locate<T>(l, false, goal, gones) : locate_in_list((int)in_list, goal, gones);
    if (id >= 0) a.outcome[r] = -2 - id;
}

// A tree of 60 nodes, 32000 fp32 logits each, takes 27 us in one wave (and 5 the walk); 16 of them as staged below 53 us.
//
// Which rows: each of them, a cluster each; the first `ahead` ones of each sequence; those that the plan lists, in turns.
enum : int { EVERY = 0, AHEAD = 1, LISTED = 2 };

template <typename T>
__global__ void __launch_bounds__(ROW_THREADS, 2)
accept_rows_kernel(const T *__restrict__ logits, long ld, int V, int ctas, int slice, Settings f, TreeArgs a, int which) {
    wait_prior();
    allow_dependents();
    const int rank = blockIdx.x % ctas, count = which == LISTED ? a.list[a.rows - 1] : 0;
    for (int i = blockIdx.x / ctas;; i += gridDim.x / ctas) {               // (the whole cluster does the same)
        if (which == LISTED && i >= count) return;
        int r;
        Node t;
        if (which == AHEAD) {
            const int b = i % a.n;
            t = Node{b, i / a.n, nodes_of(a, b), 0};
            if (t.node >= t.n) return;
            r = a.row_start[b] + t.node;
        } else {
            r = which == EVERY ? i : a.list[i];
            t = node_of(a, r);
        }
        if (which == LISTED) t.d = a.outcome[r]; else find_depth(a, t);
        if (t.d > a.depth) return;
        decide(logits, ld, V, ctas, rank, slice, f, a, r, t);
        if (which != LISTED) return;
        __syncwarp();
        // shared memory is free again, and every CTA has read the depth that outcome held
        if (ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        else __syncthreads();
    }
}

// The rows that may still be reached once the first `ahead` ones of each sequence are decided: in list[0 ..), their number in its last
// element (a first node is not among them), and the drafts accepted there in outcome.
__global__ void __launch_bounds__(1024)
accept_plan_kernel(TreeArgs a) {
    __shared__ int count;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    wait_prior();
    allow_dependents();
    for (int r = threadIdx.x; r < a.rows; r += blockDim.x) {
        Node t = node_of(a, r);
        if (t.d > a.depth || t.node < a.ahead) continue;
        find_depth(a, t);
        bool may = t.d <= a.depth;
        for (int i = t.node; may && i > 0;) {
            const int up = a.parent[(long)t.b * a.nodes + i];
            may = up >= a.ahead || a.outcome[r - t.node + up] == i;
            i = up;
        }
        if (!may) continue;
        a.outcome[r] = t.d;
        a.list[atomicAdd(&count, 1)] = r;
    }
    __syncthreads();
    if (threadIdx.x == 0) a.list[a.rows - 1] = count;
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
        at = a.outcome[start + at];
        if (at < 0) bonus = -2 - at;
    }
    a.accept_len[b] = max(d - 1, 0);
    a.bonus[b] = max(bonus, -1);
    for (; d <= a.depth; ++d) path[d] = -1;
}

constexpr int RESIDENT = 2 * 152;               // CTAs that run at a time
constexpr int STAGED_ABOVE = 2 * RESIDENT;
static_assert(data_offset(most_blocks(MAX_VOCAB / 8, 4)) + (size_t)most_blocks(MAX_VOCAB / 8, 4) * BLOCK * 4 <= 227 * 1024, "the largest row fits");

// How many CTAs share a row, and the ids of each: as few as leave room for two CTAs on an SM, 4 where there are few
// rows (and 2048 ids for each; 8 are no faster: one row of 32000 in a graph takes 11.9 us in 4 parts, 12.0 in 8, 13.3 in 2, 15.7 in 1).
struct Cut {
    int ctas, slice;
    size_t smem;
};
static Cut cut_rows(int rows, int V, int size) {
    const auto smem = [&](int slice) { return data_offset(most_blocks(slice, size)) + (size_t)most_blocks(slice, size) * BLOCK * size; };
    const auto slice_of = [&](int ctas) { return ((V + ctas - 1) / ctas + 7) / 8 * 8; };
    int c = 1;
    while (c < 8 && smem(slice_of(c)) > 112 * 1024) c *= 2;
    while (c < 4 && (long)rows * c * 2 <= RESIDENT && slice_of(c * 2) >= 2048) c *= 2;
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

static Settings settings_of(const msd_filter *f) { return f ? Settings{f->temperature, f->top_k, f->top_p, f->min_p} : Settings{}; }

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
    const Settings s = settings_of(f);
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
    if (!batch || batch->n < 0 || batch->n > MAX_TREE_ROWS || batch->rows < 0 || batch->rows > MAX_TREE_ROWS) return MSD_ERR_INVALID;
    if (batch->n == 0) return MSD_OK;
    if (!batch->row_start || !tree || !tree->tokens || !tree->parent || tree_nodes < 1 || tree_nodes > MAX_TREE_NODES ||
        !u || depth < 0 || depth > MAX_DEPTH || children < 1 || children > MAX_CHILDREN || !path || !accept_len || !bonus)
        return MSD_ERR_INVALID;
    if (batch->rows > 0 && (bad_logits(logits, ld, dtype, vocab) || !scratch)) return MSD_ERR_INVALID;
    const Settings s = settings_of(f);
    const int size = dtype == MSD_F32 ? 4 : 2;
    const Cut c = batch->rows > 0 ? cut_rows(batch->rows, vocab, size) : Cut{1, 0, 0};
    const int ahead = std::max(1, std::min(tree_nodes, RESIDENT / c.ctas / batch->n));
    const TreeArgs a{batch->n, batch->rows, tree_nodes, depth, children, ahead, batch->row_start, tree->tokens, tree->parent, tree->n_nodes, u,
                     scratch, scratch + batch->rows, path, accept_len, bonus};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (batch->rows > 0) {
        if ((long)batch->rows * c.ctas > 0x7FFFFFFF || (long)batch->n * c.ctas > 0x7FFFFFFF) return MSD_ERR_INVALID;
        const auto rows = [&](int which, const Cut &cut, int count) {
            return dtype == MSD_F32 ? launch_rows(accept_rows_kernel<float>, count, cut, st, static_cast<const float *>(logits), (long)ld, vocab,
                                                  cut.ctas, cut.slice, s, a, which)
                                    : launch_rows(accept_rows_kernel<bf16>, count, cut, st, static_cast<const bf16 *>(logits), (long)ld, vocab,
                                                  cut.ctas, cut.slice, s, a, which);
        };
        // Where the rows are more than the GPU holds at a time (two CTAs an SM), the first nodes of each tree go ahead, as many as it
        // holds, and of the others only those that may be reached then follow. (16 trees of 60 nodes, 32000 tokens:
        // 53 us, 117 with every row, 80 with the roots alone ahead.)
        cudaError_t e;
        if ((long)batch->rows * c.ctas <= STAGED_ABOVE || depth == 0) {
            e = rows(EVERY, c, batch->rows);
        } else {
            const int first = batch->n * ahead;         // (at most n, or what the GPU holds)
            e = rows(AHEAD, cut_rows(first, vocab, size), first);
            if (e == cudaSuccess) {
                e = launch_chain(accept_plan_kernel, 1, 1024, 0, st, a);
                note_launch();
            }
            // (few are expected: the 16 trees with 4 CTAs a row 53 us, with 2 55)
            const Cut few = cut_rows(std::min(batch->rows, RESIDENT / 4), vocab, size);
            if (e == cudaSuccess) e = rows(LISTED, few, std::min(batch->rows, RESIDENT / few.ctas));
        }
        if (e != cudaSuccess) return MSD_ERR_CUDA;
    }
    if (launch_chain(accept_walk_kernel, (batch->n + 31) / 32, 32, 0, st, a) != cudaSuccess) return MSD_ERR_CUDA;
    note_launch();
    return MSD_OK;
}

}  // extern "C"
