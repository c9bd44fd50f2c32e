// Attention over pages on the 5th-generation tensor cores (bf16 pools).
//
// O = softmax(Q K^T) V over tiles of 128 packed rows and 128 keys (pages_attn.cuh: what an item
// is and how its steps are cut into CTAs). S = Q K^T reads both operands from shared memory;
// P goes back over S in tensor memory as the A operand of O += P V. A CTA keeps two softmax
// groups of four warps at work, so that one's S and P V run while the other takes exponentials:
//   two tiles of rows over the same keys (PAIR), where sequences have many packed rows
//   (each key tile is read once for 256 rows: the tensor cores bound it), or
//   one tile of rows over alternate key tiles, each group with a maximum, sum and O of its own,
//   joined at the end (bytes bound it: what counts is that the copies never pause). The groups
//   take the CTA's steps in turns across items too, so short items overlap.
// Measured, with the join (32 heads of 128, 8 K/V heads): one token each of 64 requests of up to 8192
// tokens 76 us, 5.1 TB/s; one token behind 131071 90 to 91 us, 5.9 TB/s; two chunks of up to 4096 rows behind
// 4096 299 us in a loop of their own, 1.43 PFLOP/s (the tensor pipe at work in 64% of the cycles), 315 us among other calls.
// Roles (384 threads, one warp without work; 216 registers for the softmax, 72 for the others):
//   warps 0-7   softmax groups 0 and 1, a row a thread: load the query rows into shared memory
//               (swizzled as the MMA reads them), then per key tile read S, hide what the row
//               does not see, online softmax in base 2, P as bf16 over S; at an item's end O
//   warp 8      TMA: a key tile is one box a page and 64 columns, K and V in slots of their own
//   warp 9      tensor memory and the MMAs
//   warp 10     what each segment of the CTA's run is, for the others, ahead of them
// P is rounded to bf16 (the V operand's type; the row's sum takes the weights unrounded): with
// the result's own rounding that is 2^-9 a value twice, not once. Maxima, sums, S and O are
// fp32. A row's reference maximum moves (and O is rescaled) only when a tile's exceeds it by
// more than 2^8, so P <= 256.
//
// Hidden keys: S is replaced before it is used, so what K holds there does not matter. V does,
// because 0 * NaN is a NaN: in a tile that some row does not see in full, the group looks
// through V in shared memory before P V, zeroes slots past the sequence's end, and zeroes values
// that are not finite after noting the step; the item's end then goes over the noted steps' keys and adds
// those that a row does see. Such tiles lie at the diagonal, at a window's edges and in a tree, so they are
// few however long the prompt is.
#include <cstring>
#include <type_traits>

#include "pages_attn.cuh"

namespace msd {
namespace {

constexpr int KT = 128, THREADS = 384, TILE = 128, SEGS = 8;
constexpr unsigned long long TIMEOUT_NS = 2000000000ull;
constexpr float RESCALE_LOG2 = 8.f;

// ROWS: packed rows of an item. 256: a pair of tiles. Fewer than 128: the MMA still takes 128 rows; what
// it reads past the ones there are gives rows of S that nobody looks at, and the shared memory that
// they would take holds key tiles instead.
template <int HD, int ROWS>
struct Lay {
    static constexpr int NB = HD / 64;                          // 64-column boxes of a row
    static constexpr int QROWS = ROWS < TILE ? ROWS : TILE;
    static constexpr uint32_t BOX = TILE * 128;                 // [128 keys][64 bf16]
    static constexpr uint32_t MAT = NB * BOX;                   // a K or V tile
    static constexpr uint32_t QBOX = QROWS * 128, QMAT = NB * QBOX;
    static constexpr uint32_t FIXED = 2 * QMAT + (sizeof(AttnSched) + 15) / 16 * 16 + 2 * TILE * 8;
    static constexpr uint32_t LIMIT = 227 * 1024 - 1024 - 1536; // less alignment and static shared memory
    static constexpr int SLOTS = (LIMIT - FIXED) / MAT < 12 ? (LIMIT - FIXED) / MAT : 12;
    static constexpr uint32_t Q = 0, RING = 2 * QMAT, SCHED = RING + SLOTS * MAT;
    static constexpr uint32_t ML = SCHED + (sizeof(AttnSched) + 15) / 16 * 16;      // [2][128] float2
    static constexpr uint32_t SMEM = ML + 2 * TILE * 8 + 1024;
    // tensor memory: two S (P over the first half), two O
    static constexpr uint32_t T_S = 0, T_O = 2 * KT, T_COLS = 512;
    static_assert(SMEM >= tmem_smem_floor((int)T_COLS) && SMEM <= 227 * 1024 - 1536 && SLOTS >= 4, "one CTA an SM, by its tensor memory");
    static_assert(SLOTS * MAT >= BOX + QBOX, "what the MMA reads past the query rows is shared memory");
};

__device__ __forceinline__ uint32_t su32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ unsigned long long gtime() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.b32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded wait: gives up when *abort is set, or after the limit (then sets it, and the status).
__device__ __forceinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, volatile int *abort, int *status) {
    const unsigned long long t0 = gtime();
    while (!bar_try(bar, parity)) {
        if (*abort) return false;
        if (gtime() - t0 > TIMEOUT_NS) {
            *abort = 1;
            set_status(status, ST_TIMEOUT);
            return false;
        }
    }
    return true;
}
// The whole warp waits; the answer is uniform.
__device__ __forceinline__ bool w_wait(uint32_t bar, uint32_t parity, volatile int *abort, int *status) {
    if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
    return __all_sync(0xffffffffu, bar_wait_slow(bar, parity, abort, status));
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Shared-memory matrix descriptor (128-byte swizzle): start address, leading byte offset (MN-major: between
// 64-element atoms along N) and stride byte offset (between 8-row groups).
__device__ __forceinline__ uint64_t sdesc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) |
           ((uint64_t)((sbo >> 4) & 0x3FFFu) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// Instruction descriptor, kind::f16: fp32 accumulate, bf16 A (K-major) and B (K-major, or MN-major: b_mn).
__device__ __forceinline__ uint32_t idesc(int M, int N, int b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(N >> 3) << 17) |
           ((uint32_t)(M >> 4) << 24);
}
// Issue loops run in whole warps; the lane that elect_one() names issues.
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t on;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(on));
    return on;
}
__device__ __forceinline__ void w_expect_tx(uint32_t on, uint32_t bar, uint32_t bytes) {
    asm volatile(
        "{\n.reg .pred q;\nsetp.ne.b32 q, %2, 0;\n"
        "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n}" ::"r"(bar),
        "r"(bytes), "r"(on)
        : "memory");
}
__device__ __forceinline__ void w_tma2d(uint32_t on, uint32_t dst, const CUtensorMap *m, int x, int y, uint32_t bar) {
    asm volatile(
        "{\n.reg .pred q;\nsetp.ne.b32 q, %5, 0;\n"
        "@q cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];\n}" ::"r"(dst),
        "l"(m), "r"(x), "r"(y), "r"(bar), "r"(on)
        : "memory");
}
// D (+)= A B^T, both from shared memory / A from tensor memory
__device__ __forceinline__ void w_mma_ss(uint32_t on, uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 q, %5, 0;\nsetp.ne.b32 p, %4, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(id), "r"(acc), "r"(on));
}
__device__ __forceinline__ void w_mma_ts(uint32_t on, uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t acc) {
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 q, %5, 0;\nsetp.ne.b32 p, %4, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
        "r"(a), "l"(b), "r"(id), "r"(acc), "r"(on));
}
__device__ __forceinline__ void w_commit(uint32_t on, uint32_t bar) {
    asm volatile(
        "{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"(on)
        : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 16 bytes into shared memory, zeros where `live` is false
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void store32(void *p, const uint32_t *u) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]),
                 "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
                 : "memory");
}
// packed pairs of fp32
__device__ __forceinline__ uint64_t pack2(uint32_t lo, uint32_t hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
    return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t pack2f(float lo, float hi) { return pack2(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ float lo2(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float hi2(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
// the largest of three, or NaN if one is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float ex2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 128 (or 32) columns of this warp's 32 lanes, waited for in the same statement: the registers
// are defined once the data has landed.
__device__ __forceinline__ void tmem_ld128(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x128.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%"
        "27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%"
        "52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63,%64,%65,%66,%67,%68,%69,%70,%71,%72,%73,%74,%75,%76,%"
        "77,%78,%79,%80,%81,%82,%83,%84,%85,%86,%87,%88,%89,%90,%91,%92,%93,%94,%95,%96,%97,%98,%99,%100,%101"
        ",%102,%103,%104,%105,%106,%107,%108,%109,%110,%111,%112,%113,%114,%115,%116,%117,%118,%119,%120,%121"
        ",%122,%123,%124,%125,%126,%127}, [%128];"
        "\ntcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]),
          "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]),
          "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]),
          "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]),
          "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63]), "=r"(r[64]),
          "=r"(r[65]), "=r"(r[66]), "=r"(r[67]), "=r"(r[68]), "=r"(r[69]), "=r"(r[70]), "=r"(r[71]), "=r"(r[72]),
          "=r"(r[73]), "=r"(r[74]), "=r"(r[75]), "=r"(r[76]), "=r"(r[77]), "=r"(r[78]), "=r"(r[79]), "=r"(r[80]),
          "=r"(r[81]), "=r"(r[82]), "=r"(r[83]), "=r"(r[84]), "=r"(r[85]), "=r"(r[86]), "=r"(r[87]), "=r"(r[88]),
          "=r"(r[89]), "=r"(r[90]), "=r"(r[91]), "=r"(r[92]), "=r"(r[93]), "=r"(r[94]), "=r"(r[95]), "=r"(r[96]),
          "=r"(r[97]), "=r"(r[98]), "=r"(r[99]), "=r"(r[100]), "=r"(r[101]), "=r"(r[102]), "=r"(r[103]), "=r"(r[104]),
          "=r"(r[105]), "=r"(r[106]), "=r"(r[107]), "=r"(r[108]), "=r"(r[109]), "=r"(r[110]), "=r"(r[111]),
          "=r"(r[112]), "=r"(r[113]), "=r"(r[114]), "=r"(r[115]), "=r"(r[116]), "=r"(r[117]), "=r"(r[118]),
          "=r"(r[119]), "=r"(r[120]), "=r"(r[121]), "=r"(r[122]), "=r"(r[123]), "=r"(r[124]), "=r"(r[125]),
          "=r"(r[126]), "=r"(r[127])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%"
        "27,%28,%29,%30,%31}, [%32];"
        "\ntcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,"
        "%28,%29,%30,%31,%32};"
        "\ntcgen05.wait::st.sync.aligned;" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// bits [a, b) of the 32 keys from `key` on
__device__ __forceinline__ uint32_t range_bits(int a, int b, int key) {
    const int lo = min(max(a - key, 0), 32), hi = min(max(b - key, 0), 32);
    const uint32_t below_hi = hi == 32 ? 0xffffffffu : (1u << hi) - 1u, below_lo = lo == 32 ? 0xffffffffu : (1u << lo) - 1u;
    return below_hi & ~below_lo;
}
// 32 mask bits from bit `at` on (at > -32)
__device__ __forceinline__ uint32_t mask_bits(const uint64_t *m, int words, int at) {
    if (at < 0) return words > 0 ? (uint32_t)m[0] << -at : 0u;
    const int w = at >> 6, o = at & 63;
    uint64_t x = w < words ? m[w] >> o : 0ull;
    if (o > 32 && w + 1 < words) x |= m[w + 1] << (64 - o);
    return (uint32_t)x;
}

// A segment as the roles need it: made by one warp ahead of them, in a ring in shared memory.
struct Seg {
    int i, h, seq, start;             // listed sequence, K/V head, table row, first row
    int len, base, rows, live;        // tokens, tokens before the rows, rows, rows that exist in its tree
    int m0, n, nx[2];                 // first packed row, steps (0: no more segments), steps of each group
    int u0;                           // the CTA's steps before it
    int full_start, full_end;         // a tile within these is seen in full by all rows that see anything
    unsigned odd;                     // bit t % 32: V of step t had values that are not finite, taken out
    int j0, sink_tiles, lo, whole;    // first step; which key tiles the steps are; the item's only segment
    long part;                        // its partial results' first row
    __device__ int key(int t) const {
        const int j = j0 + t;
        return (j < sink_tiles ? j : lo + j - sink_tiles) * KT;
    }
    __device__ bool full(const PagesAttn &a, int key0) const {
        return key0 + KT <= full_end && (key0 >= full_start || key0 + KT <= a.sinks);
    }
};

// A thread's row.
struct Row {
    int r, place;                     // -1: none that sees anything; its place
    const uint64_t *mask;
};

// The keys of a tile that a row sees.
__device__ __forceinline__ void seen_bits(const PagesAttn &a, const Seg &d, const Row &x, int key0, uint32_t *w) {
    if (x.r < 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = 0;
        return;
    }
    const int hi = a.mask ? d.base : d.base + x.r + 1, lo = a.window ? x.place - a.window + 1 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int key = key0 + 32 * i;
        w[i] = range_bits(lo, hi, key);
        if (a.sinks) w[i] |= range_bits(0, min(a.sinks, hi), key);
        if (a.mask && key + 32 > d.base && key < d.len) {
            uint32_t m = mask_bits(x.mask, a.words, key - d.base) & range_bits(d.base, d.len, key);
            if (a.window && x.place - d.base >= a.window) {       // (else all depths up to its own are inside)
                for (uint32_t left = m; left; left &= left - 1) {
                    const int bit = __ffs(left) - 1;
                    const int at = d.base + node_depth(a, d.i, key + bit - d.base);
                    if (x.place - at >= a.window && at >= a.sinks) m &= ~(1u << bit);
                }
            }
            w[i] |= m;
        }
    }
}

// Values of V that a tile's look-through took out, and that the row sees: added to eight of its columns.
// (A tile that one group of a pair sees in full may have been looked through by the other.)
__device__ __noinline__ void add_odd(const PagesAttn &a, const Seg &d, unsigned odd, Row x, int hd, int col, float *acc) {
    const PagesView &v = a.pv;
    for (int t = 0; t < d.n; ++t) {
        const int key0 = d.key(t);
        if (!(odd >> (t & 31) & 1u) || d.full(a, key0)) continue;
        uint32_t w[4];
        seen_bits(a, d, x, key0, w);
        for (int k = 0; k < KT; ++k) {
            const int slot = key0 + k;
            if (slot >= d.len || !((k < 64 ? k < 32 ? w[0] : w[1] : k < 96 ? w[2] : w[3]) >> (k & 31) & 1u)) continue;
            const int id = v.table[(long)d.seq * v.max_pages + (slot >> v.page_shift)];
            if ((unsigned)id >= (unsigned)v.n_pages) continue;
            const bf16 *src = static_cast<const bf16 *>(v.kv) + ((long)a.layer * v.n_pages + id) * v.page_elems() +
                              ((long)(v.kv_heads + d.h) * v.page + (slot & (v.page - 1))) * hd + col;
            for (int e = 0; e < 8; ++e) {
                const float y = __bfloat162float(src[e]);
                if (!isfinite(y)) acc[e] += y;
            }
        }
    }
}

// V as the MMA will read it: a thread's key row of a tile, zeros if no token is there (`held` false), and zeros for
// values that are not finite, which *odd's bit then tells. x * 0 is a NaN for those alone, so the look costs one
// multiply-add for two values.
template <int NB>
__device__ __forceinline__ void clean_row(uint8_t *row, uint32_t box, int lane, bool held, unsigned *odd, unsigned bit) {
    auto at = [&](int i) { return reinterpret_cast<uint4 *>(row + (i >> 3) * box + (((i + lane) & 7) << 4)); };
    if (!held) {
#pragma unroll
        for (int i = 0; i < 8 * NB; ++i) *at(i) = make_uint4(0, 0, 0, 0);
        return;
    }
    const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
    __nv_bfloat162 acc[4] = {zero, zero, zero, zero};
#pragma unroll
    for (int i = 0; i < 8 * NB; ++i) {
        const uint4 u = *at(i);
        acc[0] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u.x), zero, acc[0]);
        acc[1] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u.y), zero, acc[1]);
        acc[2] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u.z), zero, acc[2]);
        acc[3] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u.w), zero, acc[3]);
    }
    const __nv_bfloat162 all = __hadd2(__hadd2(acc[0], acc[1]), __hadd2(acc[2], acc[3]));
    if (__low2float(all) == 0.f && __high2float(all) == 0.f) return;
    atomicOr(odd, bit);
    __threadfence_block();
#pragma unroll 1
    for (int i = 0; i < 8 * NB; ++i) {
        uint32_t *q = reinterpret_cast<uint32_t *>(at(i));
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {
            uint32_t u = q[k];
            if ((u & 0x7f80u) == 0x7f80u) u &= 0xffff0000u;
            if ((u & 0x7f800000u) == 0x7f800000u) u &= 0x0000ffffu;
            q[k] = u;
        }
    }
}

// A place of the ring and the parity of its phase, counted.
template <int SLOTS>
struct Ticket {
    int slot = 0;
    uint32_t phase = 0;
    __device__ void next() {
        if (++slot == SLOTS) {
            slot = 0;
            phase ^= 1u;
        }
    }
};

// Where the ring holds the V tile of the CTA's step u: K tiles run LEAD steps ahead of V tiles (K0 K1 V0 K2 V1 ... for two; at
// the end of the run the places of K tiles that there are none of stay empty).
template <int LEAD>
__device__ __forceinline__ int ring_v(int u) { return 2 * u + LEAD; }

template <int HD, int ROWS>
__global__ void __launch_bounds__(THREADS, 1) pages_attn_tc_kernel(const __grid_constant__ CUtensorMap map, const PagesAttn a) {
    using L = Lay<HD, ROWS>;
    constexpr bool PAIR = ROWS == 2 * TILE;
    constexpr int LEAD = PAIR ? 1 : 2, SLOTS = L::SLOTS;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * SLOTS + 10 + 2 * SEGS];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    __shared__ Seg s_seg[SEGS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t raw = su32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *sm = smem_raw + (base - raw);
    AttnSched &sched = *reinterpret_cast<AttnSched *>(sm + L::SCHED);
    float2 *s_ml = reinterpret_cast<float2 *>(sm + L::ML);
    const uint32_t full0 = su32(bars), empty0 = full0 + 8 * SLOTS, s_full0 = empty0 + 8 * SLOTS, p_full0 = s_full0 + 16,
                   o_full0 = p_full0 + 16, q_full0 = o_full0 + 16, drain = q_full0 + 16, g_full0 = drain + 8,
                   g_empty0 = g_full0 + 8 * SEGS, both = g_empty0 + 8 * SEGS;
    if (threadIdx.x == 0) {
        for (int i = 0; i < SLOTS; ++i) {
            bar_init(full0 + 8 * i, 1);
            bar_init(empty0 + 8 * i, 1);
        }
        for (int x = 0; x < 2; ++x) {
            bar_init(s_full0 + 8 * x, 1);
            bar_init(p_full0 + 8 * x, 128);
            bar_init(o_full0 + 8 * x, 1);
            bar_init(q_full0 + 8 * x, 128);
        }
        bar_init(drain, 1);
        bar_init(both, 256);
        for (int i = 0; i < SEGS; ++i) {
            bar_init(g_full0 + 8 * i, 1);
            bar_init(g_empty0 + 8 * i, 2 + 256);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_abort = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(&s_tmem)),
                     "r"(L::T_COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    wait_prior();
    allow_dependents();
    attn_schedule<ROWS, KT, THREADS>(a, sched, blockIdx.x, gridDim.x);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = s_tmem;
    const PagesView &v = a.pv;
    const int G = a.group;
    int *status = v.status;
    auto seg_wait = [&](int i) { return w_wait(g_full0 + 8 * (i % SEGS), (uint32_t)(i / SEGS) & 1u, &s_abort, status); };
    // registers to where they are used: 216 a softmax thread, 72 the others (2 * 216 + 72 = 3 * 168)
    if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 10) {
        // ---- segments ------------------------------------------------------
        AttnWalk<ROWS, KT> walk(a, sched);
        Segment g;
        int u0 = 0;
        for (int i = 0;; ++i) {
            if (!w_wait(g_empty0 + 8 * (i % SEGS), (uint32_t)(i / SEGS + 1) & 1u, &s_abort, status)) break;
            const bool have = walk.next(g);
            if (lane == 0) {
                Seg &d = s_seg[i % SEGS];
                d.n = 0;
                if (have) {
                    d.i = g.i;
                    d.h = g.h;
                    d.seq = a.b.seqs[g.i];
                    d.start = a.b.row_start[g.i];
                    d.len = sched.len[g.i];
                    d.rows = sched.rows[g.i];
                    d.base = d.len - d.rows;
                    d.live = a.mask && a.n_nodes ? min(d.rows, a.n_nodes[g.i]) : d.rows;
                    d.m0 = g.tile * ROWS;
                    d.n = g.j1 - g.j0;
                    d.j0 = g.j0;
                    d.sink_tiles = g.range.sink_tiles;
                    d.lo = g.range.lo;
                    d.whole = segment_whole(g);
                    d.part = part_slot(g, blockIdx.x) * ROWS;
                    if (PAIR) {           // the first tile's rows may end before the last key tiles
                        const bool two = d.rows * G - d.m0 > TILE;
                        const int hi = d.base + group_div(a, d.m0 + TILE - 1) + 1;
                        d.nx[0] = two && !a.mask ? min(d.n, max(0, d.sink_tiles + (hi + KT - 1) / KT - d.lo - d.j0)) : d.n;
                        d.nx[1] = two ? d.n : 0;
                    } else {              // steps in turns
                        d.nx[u0 & 1] = (d.n + 1) / 2;
                        d.nx[(u0 & 1) ^ 1] = d.n / 2;
                    }
                    d.full_end = d.base + (a.mask ? 0 : group_div(a, d.m0) + 1);
                    d.full_start = !a.window ? 0
                                   : d.base + (a.mask ? a.nodes : group_div(a, min(d.m0 + ROWS, d.rows * G) - 1)) - a.window + 1;
                    d.odd = 0;
                    d.u0 = u0;
                    u0 += d.n;
                }
                bar_arrive(g_full0 + 8 * (i % SEGS));
            }
            __syncwarp();
            if (!have) break;
        }
        if (lane == 0) name_parts<ROWS, KT>(a, sched, blockIdx.x);
        __syncwarp();
        if (a.mask && a.window) check_depths<ROWS, KT>(a, sched, lane, 32);
        __syncwarp();
    } else if (warp == 8) {
        // ---- TMA -----------------------------------------------------------
        // A key tile costs this warp as little as can be: its page ids are asked for one tile ahead and kept for V, and
        // places of the ring are counted, not divided (with the ids loaded and the places computed where they are
        // needed, ragged chunks took 355 us; with shorter issue loops as well, 314).
        const uint32_t on = elect_one();
        const int per = KT >> v.page_shift, page_rows = v.kv_heads * v.page;          // rows of K, or V, of a page
        const uint32_t page_bytes = v.page * 128;                                     // of a box
        Ticket<SLOTS> at;
        int filled = 0;
        bool ok = true;
        struct Tile {
            int y, n;                     // the row of the lane's page where its K head begins; pages
        };
        auto load = [&](const Tile &x, int what) {
            if (!w_wait(empty0 + 8 * at.slot, at.phase ^ 1u, &s_abort, status)) return false;
            const uint32_t bar = full0 + 8 * at.slot;
            uint32_t dst = base + L::RING + at.slot * L::MAT;
            w_expect_tx(on, bar, (uint32_t)x.n * page_bytes * L::NB);
            for (int i = 0; i < x.n; ++i, dst += page_bytes) {
                const int y = __shfl_sync(0xffffffffu, x.y, i) + what * page_rows;
#pragma unroll
                for (int b = 0; b < L::NB; ++b) w_tma2d(on, dst + b * L::BOX, &map, 64 * b, y, bar);
            }
            at.next();
            ++filled;
            return true;
        };
        // the walk over K tiles, LEAD ahead of V's; V tiles' segments are only counted (for the ring of segments)
        int ks = 0, kt = 0, kn = 0, k_len = 0, k_y0 = 0, k_j0 = 0, k_sinks = 0, k_lo = 0, vs = 0, v_left = 0;
        const int *table = nullptr;
        Tile ahead{0, 0}, wait_v[LEAD + 1] = {};               // the next K tile; V tiles of the K tiles loaded
        auto fetch = [&]() {              // `ahead`: n 0 at the end
            ahead.n = 0;
            if (kt == kn) {
                if (!seg_wait(ks)) return false;
                const Seg &d = s_seg[ks % SEGS];
                kn = d.n;
                kt = 0;
                if (kn == 0) return true;
                ++ks;
                k_len = d.len;
                k_y0 = a.layer * v.n_pages * 2 * page_rows + d.h * v.page;
                k_j0 = d.j0;
                k_sinks = d.sink_tiles;
                k_lo = d.lo;
                table = v.table + (long)d.seq * v.max_pages;
            }
            const int j = k_j0 + kt++, key0 = (j < k_sinks ? j : k_lo + j - k_sinks) * KT, first = key0 >> v.page_shift;
            ahead.n = min(per, ((k_len - 1) >> v.page_shift) - first + 1);
            ahead.y = lane < ahead.n ? table[first + lane] : 0;       // (a page id as yet)
            return true;
        };
        auto next_k = [&](Tile &x) {      // loads `ahead` and asks for the one after it; x: its V
            x = ahead;
            if (x.n == 0) {               // no K tile: its place stays empty
                at.next();
                return true;
            }
            if ((unsigned)x.y < (unsigned)v.n_pages) {
                x.y = k_y0 + x.y * 2 * page_rows;       // (K's walk is still in its segment)
            } else {                      // no page: K and V from before the pool's first row, which are zeros
                x.y = -v.page - page_rows;
                set_status(status, ST_RANGE);
            }
            return load(x, 0) && fetch();
        };
        ok = fetch();
        for (int u = -LEAD; ok; ++u) {
            if (u >= 0) {
                if (wait_v[0].n == 0) break;
                if (v_left == 0) v_left = s_seg[vs % SEGS].n;     // (K's walk has been there)
                ok = load(wait_v[0], 1);
                if (--v_left == 0) {
                    __syncwarp();
                    if (lane == 0) bar_arrive(g_empty0 + 8 * (vs % SEGS));
                    ++vs;
                }
            }
            ok = ok && next_k(wait_v[LEAD]);
#pragma unroll
            for (int i = 0; i < LEAD; ++i) wait_v[i] = wait_v[i + 1];
        }
        if (s_abort) {            // the copies still in flight land before the CTA exits
            volatile int never = 0;
            Ticket<SLOTS> p;
            for (int i = 0; i < filled; ++i, p.next())
                if (i >= filled - SLOTS) bar_wait_slow(full0 + 8 * p.slot, p.phase, &never, status);
        }
        __syncwarp();
    } else if (warp == 9) {
        // ---- MMA -----------------------------------------------------------
        // (code that is short: every call of these is inlined once a loop. Unrolled over the groups, the loop below made 64
        // ragged requests take 112 us, not 97: its instructions did not stay beside the softmax's)
        const uint32_t on = elect_one();
        const uint32_t id_s = idesc(TILE, KT, 0), id_o = idesc(TILE, HD, 1);
        uint32_t p_ph = 0, q_ph = 0;      // a bit a group, a buffer
        bool ok = true;
        auto wait_slot = [&](const Ticket<SLOTS> &p) {
            const bool r = w_wait(full0 + 8 * p.slot, p.phase, &s_abort, status);
            fence_after();
            return r;
        };
        const uint64_t d_q = sdesc(base + L::Q, 16, 1024), d_k = sdesc(base + L::RING, 16, 1024),
                       d_v = sdesc(base + L::RING, L::BOX, 1024);
        auto s_mma = [&](int x, int slot, int qbuf) {
            const uint64_t k = d_k + (uint32_t)slot * (L::MAT >> 4), q = d_q + (uint32_t)qbuf * (L::QMAT >> 4);
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk)
                w_mma_ss(on, tmem + L::T_S + x * KT, q + (((kk >> 2) * L::QBOX + (kk & 3) * 32) >> 4),
                         k + (((kk >> 2) * L::BOX + (kk & 3) * 32) >> 4), id_s, kk > 0);
            w_commit(on, s_full0 + 8 * x);
        };
        auto o_mma = [&](int x, int slot, bool acc) {
            const uint64_t w = d_v + (uint32_t)slot * (L::MAT >> 4);
#pragma unroll
            for (int kk = 0; kk < KT / 16; ++kk)
                w_mma_ts(on, tmem + L::T_O + x * HD, tmem + L::T_S + x * KT + kk * 8, w + (kk * 2048 >> 4), id_o, kk > 0 || acc);
        };
        auto free_slot = [&](int slot) { w_commit(on, empty0 + 8 * slot); };
        auto wait_p = [&](int x) {
            const bool r = w_wait(p_full0 + 8 * x, p_ph >> x & 1u, &s_abort, status);
            p_ph ^= 1u << x;
            fence_after();
            return r;
        };
        auto wait_q = [&](int x) {
            const bool r = w_wait(q_full0 + 8 * x, q_ph >> x & 1u, &s_abort, status);
            q_ph ^= 1u << x;
            fence_after();
            return r;
        };
        int seg = 0;
        Ticket<SLOTS> at;                 // the ring's tiles in the order of their use
        if constexpr (PAIR) {
            for (;; ++seg) {
                ok = seg_wait(seg);
                if (!ok) break;
                const Seg &d = s_seg[seg % SEGS];
                const int n = d.n, nx0 = d.nx[0], nx1 = d.nx[1], last = nx1 > 0;
                if (n == 0) break;
                __syncwarp();
                if (lane == 0) bar_arrive(g_empty0 + 8 * (seg % SEGS));
                for (int t = -1; ok && t < n; ++t) {
                    Ticket<SLOTS> tv = at, tk = at;
                    if (t >= 0) tk.next();
#pragma unroll 1
                    for (int x = 0; x < 2; ++x) {
                        const int nx = x ? nx1 : nx0;
                        if (!ok) break;
                        if (t >= 0 && t < nx) {
                            ok = wait_p(x) && wait_slot(tv);
                            if (!ok) break;
                            o_mma(x, tv.slot, t > 0);
                            if (x == last) free_slot(tv.slot);
                            if (t == nx - 1) w_commit(on, o_full0 + 8 * x);
                        }
                        if (t + 1 < nx) {
                            if (t < 0) ok = wait_q(x);
                            ok = ok && wait_slot(tk);
                            if (!ok) break;
                            s_mma(x, tk.slot, x);
                            if (x == last) free_slot(tk.slot);
                        }
                    }
                    if (t >= 0) at.next();
                    if (t + 1 < n) at.next();
                }
                if (!ok) break;
            }
        } else {
            // S two steps ahead of P V, across segments: what P V of a step needs to know of its segment waits in three bits
            // a step (1: not its group's first there, 2: its group's last there, 4: there is such a step)
            int left = 0, t = 0, qbuf = 1;                        // steps left, and done, of the segment that S is in
            uint32_t flags = 0;                                   // of the step that P V is at, and the next ones
            bool more = true;
            auto next_s = [&](int x, int shift) {
                if (!more) return true;
                if (left == 0) {
                    if (!seg_wait(seg)) return false;
                    left = s_seg[seg % SEGS].n;
                    if (left == 0) {
                        more = false;
                        return true;
                    }
                    __syncwarp();
                    if (lane == 0) bar_arrive(g_empty0 + 8 * (seg % SEGS));
                    t = 0;
                    qbuf ^= 1;
                    if (!wait_q(qbuf)) return false;
                    ++seg;
                }
                if (!wait_slot(at)) return false;
                s_mma(x, at.slot, qbuf);
                free_slot(at.slot);
                flags |= ((t > 1 ? 1u : 0u) | (left <= 2 ? 2u : 0u) | 4u) << shift;
                ++t;
                --left;
                return true;
            };
            for (int u = -2; ok; ++u) {
                const int x = u & 1;
                if (u >= 0) {
                    if (!(flags & 4u)) break;
                    ok = wait_p(x) && wait_slot(at);
                    if (!ok) break;
                    o_mma(x, at.slot, flags & 1u);
                    free_slot(at.slot);
                    if (flags & 2u) w_commit(on, o_full0 + 8 * x);
                    at.next();
                    flags >>= 3;
                }
                ok = next_s(x, u == -2 ? 0 : 3);
                at.next();
            }
        }
        if (seg > 0 || !ok) {     // no MMA outlives the CTA's tensor memory
            w_commit(on, drain);
            volatile int never = 0;
            bar_wait_slow(drain, 0, &never, status);
        }
        __syncwarp();
    }
    } else {
        // ---- softmax -------------------------------------------------------
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int x = warp >> 2, m = threadIdx.x & 127;
        const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        const uint32_t t_s = lanes + L::T_S + x * KT, t_o = lanes + L::T_O;
        uint32_t s_ph = 0, o_ph[2] = {0, 0};
        bool dead = false;            // a wait ran out, here or in another role
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (!dead && !w_wait(bar, parity, &s_abort, status)) dead = true;
        };
        // both groups are here (twice a segment)
        auto groups_sync = [&](uint32_t parity) {
            fence_before();
            bar_arrive(both);
            wait(both, parity);
            fence_after();
        };
        // the query rows of a segment into a buffer (swizzled as the MMA reads them) by one group: a pair's groups load
        // their own tiles, else see below. Asked for while there is other work, handed over by give_q.
        auto load_q = [&](const Seg &d, int buf) {
            constexpr int PIECES = L::QROWS * HD / 8;             // of 16 bytes
            const int pm0 = d.m0 + (PAIR ? x * TILE : 0), left = d.rows * G - pm0;
            const bf16 *src = static_cast<const bf16 *>(a.q) + d.start * a.ldq + (long)d.h * G * HD;
            const uint32_t dst = base + L::Q + buf * L::QMAT;
#pragma unroll 4
            for (int p0 = 0; p0 < PIECES; p0 += 128) {
                const int p = p0 + m, row = p / (HD / 8), c = p % (HD / 8);
                const int pm = pm0 + row, r = group_div(a, pm);
                copy16(dst + (c >> 3) * L::QBOX + row * 128 + (((c & 7) ^ (row & 7)) << 4),
                       row < left ? src + r * a.ldq + (pm - r * G) * HD + 8 * c : src, row < left);
            }
        };
        auto give_q = [&](int buf) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy();
            bar_arrive(q_full0 + 8 * buf);
        };
        // segment i, if there is one (each segment but the first follows one that is there)
        auto has = [&](int i) {
            wait(g_full0 + 8 * (i % SEGS), (uint32_t)(i / SEGS) & 1u);
            return !dead && s_seg[i % SEGS].n > 0;
        };
        // the first segments' queries: a pair's groups their own tile of the first, else group x that of segment x
        if (has(0) && (PAIR ? s_seg[0].nx[x] > 0 : x == 0 || has(1))) {
            load_q(s_seg[PAIR ? 0 : x], x);
            give_q(x);
        }
        for (int seg = 0; !dead; ++seg) {
            const Seg &d = s_seg[seg % SEGS];
            const int n = d.n, nx = d.nx[x];
            if (n == 0) break;
            const int first = PAIR ? 0 : (d.u0 ^ x) & 1;          // the group's first step of the segment
            const int pm0 = d.m0 + (PAIR ? x * TILE : 0), pm = pm0 + m, r = group_div(a, pm);
            const bool valid = m < L::QROWS && pm < d.rows * G;
            Row rw;
            rw.r = valid && r < d.live ? r : -1;
            rw.place = d.base + r;
            rw.mask = nullptr;
            if (a.mask && rw.r >= 0) {
                rw.mask = a.mask + ((long)d.i * a.nodes + r) * a.words;
                if (a.window) rw.place = d.base + node_depth(a, d.i, r);
            }
            // every row that sees anything sees a whole tile that ends here at the latest, and starts here at the earliest
            const int full_end = d.base + (a.mask ? 0 : group_div(a, pm0) + 1);
            const int full_start = !a.window ? 0
                                   : d.base + (a.mask ? a.nodes : group_div(a, min(pm0 + L::QROWS, d.rows * G) - 1)) - a.window + 1;
            const bool any = __any_sync(0xffffffffu, rw.r >= 0), blind = __any_sync(0xffffffffu, valid && rw.r < 0);
            float m_ref = -INFINITY, sum = 0.f;
            // The queries to load once this segment's S are done, seen by the group that gets the last of them: the next
            // segment's (a pair: each group its own tile), or those of the one after it, into this one's buffer.
            bool q_next = false;
            auto next_q = [&]() {
                if constexpr (PAIR) {
                    q_next = has(seg + 1) && s_seg[(seg + 1) % SEGS].nx[x] > 0;
                    if (q_next) load_q(s_seg[(seg + 1) % SEGS], x);
                } else {
                    q_next = has(seg + 1) && has(seg + 2);
                    if (q_next) load_q(s_seg[(seg + 2) % SEGS], seg & 1);
                }
            };
            for (int t = 0; t < nx; ++t) {
                const int tt = PAIR ? t : 2 * t + first, key0 = d.key(tt);
                wait(s_full0 + 8 * x, s_ph);
                s_ph ^= 1u;
                fence_after();
                const bool full = key0 + KT <= full_end && (key0 >= full_start || key0 + KT <= a.sinks);
                if (any) {
                    uint32_t s[128];
                    if (!full || blind) {            // (a loop over tensor memory: short beside what every tile runs)
                        uint32_t w[4];
                        seen_bits(a, d, rw, key0, w);
#pragma unroll 1
                        for (int c = 0; c < 128; c += 32) {
                            tmem_ld32(t_s + c, s);
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (!(w[0] >> k & 1u)) s[k] = 0xff800000u;
                            tmem_st32(t_s + c, s);
                            w[0] = w[1];
                            w[1] = w[2];
                            w[2] = w[3];
                        }
                    }
                    tmem_ld128(t_s, s);
                    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 128; c += 8) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            top[k] = max3_nan(top[k], __uint_as_float(s[c + k]), __uint_as_float(s[c + 4 + k]));
                    }
                    const float now = max3_nan(max3_nan(top[0], top[1], top[2]), top[3], top[3]) * a.scale_log2;
                    const bool move = m_ref != -INFINITY && now > m_ref + RESCALE_LOG2;
                    if (__any_sync(0xffffffffu, move)) {
                        // (S of this tile has landed, so has the P V issued before it)
                        const float f = move ? ex2_fast(m_ref - now) : 1.f;
                        sum *= f;
                        if (move) m_ref = now;
#pragma unroll 1
                        for (int c = 0; c < HD; c += 32) {
                            uint32_t o[32];
                            tmem_ld32(t_o + x * HD + c, o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            tmem_st32(t_o + x * HD + c, o);
                        }
                    }
                    if (m_ref == -INFINITY || now != now) m_ref = now;       // (not a number: so are the row's weights)
                    const float use = m_ref == -INFINITY ? 0.f : m_ref;
                    uint64_t part[4] = {0, 0, 0, 0};
                    const uint64_t scale2 = pack2f(a.scale_log2, a.scale_log2), use2 = pack2f(-use, -use);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t p[32];
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            const uint64_t z = fma2(pack2(s[64 * h + 2 * c], s[64 * h + 2 * c + 1]), scale2, use2);
                            const float e0 = ex2_fast(lo2(z)), e1 = ex2_fast(hi2(z));
                            part[c & 3] = add2(part[c & 3], pack2f(e0, e1));
                            const __nv_bfloat162 b = __floats2bfloat162_rn(e0, e1);
                            p[c] = *reinterpret_cast<const uint32_t *>(&b);
                        }
                        tmem_st32(t_s + 32 * h, p);
                    }
                    const uint64_t all = add2(add2(part[0], part[1]), add2(part[2], part[3]));
                    sum += lo2(all) + hi2(all);
                }
                if (!full) {
                    const int pos = ring_v<LEAD>(d.u0 + tt);
                    wait(full0 + 8 * (pos % SLOTS), (uint32_t)(pos / SLOTS) & 1u);
                    clean_row<L::NB>(sm + L::RING + (pos % SLOTS) * L::MAT + m * 128, L::BOX, lane, key0 + m < d.len,
                                     &s_seg[seg % SEGS].odd, 1u << (tt & 31));
                    fence_proxy();
                }
                fence_before();
                bar_arrive(p_full0 + 8 * x);
                if (PAIR ? t == nx - 1 : tt == n - 1) next_q();
            }
            if (PAIR && nx == 0) next_q();
            if (!PAIR && nx == 0) {                  // the other group's alone
                o_ph[x ^ 1] ^= 1u;
                bar_arrive(g_empty0 + 8 * (seg % SEGS));
                if (!dead) wait(g_full0 + 8 * ((seg + 1) % SEGS), (uint32_t)((seg + 1) / SEGS) & 1u);
                continue;
            }

            // the item's end: this group's O, or half the columns of both groups' O joined
            float f0 = 1.f, f1 = 0.f;
            if (nx > 0) {
                wait(o_full0 + 8 * x, o_ph[x]);
                o_ph[x] ^= 1u;
            }
            if (q_next) give_q(PAIR ? x : seg & 1);
            if constexpr (!PAIR) {
                float2 a0 = make_float2(m_ref, sum), a1 = make_float2(-INFINITY, 0.f);
                if (n > 1) {
                    wait(o_full0 + 8 * (x ^ 1), o_ph[x ^ 1]);
                    o_ph[x ^ 1] ^= 1u;
                    s_ml[x * TILE + m] = a0;
                    groups_sync(0);
                    a0 = s_ml[m];
                    a1 = s_ml[TILE + m];
                }
                const float top = fmaxf(a0.x, a1.x), use = top == -INFINITY ? 0.f : top;
                f0 = a0.y == 0.f ? 0.f : a0.x == top ? 1.f : ex2_fast(a0.x - use);       // (nothing seen: 0 times nothing)
                f1 = a1.y == 0.f ? 0.f : a1.x == top ? 1.f : ex2_fast(a1.x - use);
                m_ref = top;
                sum = (a0.y == 0.f ? 0.f : a0.y * f0) + (a1.y == 0.f ? 0.f : a1.y * f1);
            }
            fence_after();
            // two groups' results: each half of the columns; one's: all of them
            const bool two = !PAIR && n > 1;
            const int cols = two ? HD / 2 : HD, col0 = two ? x * (HD / 2) : 0;
            const bool none = sum == 0.f;            // the row sees nothing: zeros, whatever O holds
            const bool whole = d.whole;
            const unsigned odd = d.odd;
            const int head = d.h * G + pm - r * G;
            const long row = d.start + r, part = d.part + (PAIR ? x * TILE : 0) + m;
            if (nx > 0) {
                const float inv = whole ? none ? 0.f : 1.f / sum : 1.f;
                const uint64_t g0 = pack2f(f0 * inv, f0 * inv), g1 = pack2f(f1 * inv, f1 * inv);
                bf16 *dst = static_cast<bf16 *>(a.out) + row * a.ldo + (long)head * HD + col0;
                float *pdst = a.part_o + part * HD + col0;
                const bool store = valid && !dead;
#pragma unroll 1
                for (int c = 0; c < cols; c += 32) {
                    uint32_t o[32];
                    uint64_t acc[16];
                    tmem_ld32(t_o + (two ? 0 : x * HD) + col0 + c, o);
#pragma unroll
                    for (int k = 0; k < 16; ++k) acc[k] = f0 == 0.f || none ? 0ull : fma2(pack2(o[2 * k], o[2 * k + 1]), g0, 0ull);
                    if (two) {
                        tmem_ld32(t_o + HD + col0 + c, o);
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (f1 != 0.f) acc[k] = fma2(pack2(o[2 * k], o[2 * k + 1]), g1, acc[k]);
                    }
                    if (odd && rw.r >= 0) {
#pragma unroll 1
                        for (int e = 0; e < 32; e += 8) {
                            float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                            add_odd(a, d, odd, rw, HD, col0 + c + e, y);
#pragma unroll
                            for (int k = 0; k < 16; ++k)
                                if (k / 4 == e / 8) acc[k] = add2(acc[k], pack2f(y[2 * (k & 3)], y[2 * (k & 3) + 1]));
                        }
                    }
                    if (!store) continue;
                    // (a lane's row is a line of its own: 32 bytes a store where the rows allow it)
                    if (whole) {
                        uint32_t u[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const __nv_bfloat162 b = __floats2bfloat162_rn(lo2(acc[k]), hi2(acc[k]));
                            u[k] = *reinterpret_cast<const uint32_t *>(&b);
                        }
                        if (a.wide) {
                            store32(dst + c, u);
                            store32(dst + c + 16, u + 8);
                        } else {
#pragma unroll
                            for (int k = 0; k < 16; k += 4)
                                *reinterpret_cast<uint4 *>(dst + c + 2 * k) = make_uint4(u[k], u[k + 1], u[k + 2], u[k + 3]);
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 16; k += 4) {
                            const uint32_t u[8] = {(uint32_t)acc[k], (uint32_t)(acc[k] >> 32), (uint32_t)acc[k + 1], (uint32_t)(acc[k + 1] >> 32),
                                                   (uint32_t)acc[k + 2], (uint32_t)(acc[k + 2] >> 32), (uint32_t)acc[k + 3],
                                                   (uint32_t)(acc[k + 3] >> 32)};
                            store32(pdst + c + 2 * k, u);
                        }
                    }
                }
            }
            if (valid && !dead && (!two || x == 0)) {
                if (!whole) *reinterpret_cast<float2 *>(a.part_ml + 2 * part) = make_float2(m_ref, sum);
                else if (a.lse) a.lse[row * v.heads + head] = none ? -INFINITY : (m_ref + log2f(sum)) * 0.6931471805599453f;
            }
            // the next segment is known before this one's place may go to a later one
            if (!dead) wait(g_full0 + 8 * ((seg + 1) % SEGS), (uint32_t)((seg + 1) / SEGS) & 1u);
            // the other group's O is not overwritten before this one has read it
            if (two) groups_sync(1);
            bar_arrive(g_empty0 + 8 * (seg % SEGS));
        }
    }
    fence_before();
    __syncthreads();
    if (warp == 9) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::T_COLS) : "memory");
    }
}

template <int HD, int ROWS>
cudaError_t launch(const CUtensorMap &map, const PagesAttn &a, int sms, cudaStream_t s) {
    cudaError_t e = launch_chain(pages_attn_tc_kernel<HD, ROWS>, dim3(sms), dim3(THREADS), Lay<HD, ROWS>::SMEM, s, map, a);
    note_launch();
    return e != cudaSuccess ? e : launch_pages_attn_join(a, MSD_BF16, sms, ROWS, s);
}

template <int HD, int ROWS>
bool setup() {
    return cudaFuncSetAttribute(pages_attn_tc_kernel<HD, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)Lay<HD, ROWS>::SMEM) == cudaSuccess;
}

// A tile as large as the sequences' packed rows: a small one leaves room for more key tiles in flight. One shape serves
// the whole call, by the mean: a chunk among many single tokens then runs in small tiles (of 32 rows for one of 512 rows and
// 127 tokens, four heads to a K/V head: 64 tiles where 8 would do), and tokens beside a long chunk in large ones.
template <int HD>
cudaError_t launch_rows(const CUtensorMap &map, const PagesAttn &a, int sms, cudaStream_t s) {
    return a.packed <= 32    ? launch<HD, 32>(map, a, sms, s)
           : a.packed <= 64  ? launch<HD, 64>(map, a, sms, s)
           : a.packed <= 128 ? launch<HD, 128>(map, a, sms, s)
                             : launch<HD, 256>(map, a, sms, s);
}

}  // namespace

bool pages_attn_tc_setup() {
    return setup<64, 32>() && setup<64, 64>() && setup<64, 128>() && setup<64, 256>() && setup<128, 32>() &&
           setup<128, 64>() && setup<128, 128>() && setup<128, 256>();
}

// The pool as rows of head_dim elements, in boxes of a page's tokens and 64 columns.
bool pages_attn_map(const PagesView &v, CUtensorMap *map) {
    cudaDriverEntryPointQueryResult q;
    void *fn = nullptr;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess || !fn)
        return false;
    memset(map, 0, sizeof *map);
    cuuint64_t dims[2] = {(cuuint64_t)v.head_dim, (cuuint64_t)v.layers * v.n_pages * 2 * v.kv_heads * v.page};
    cuuint64_t strides[1] = {(cuuint64_t)v.head_dim * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)v.page};
    cuuint32_t estr[2] = {1, 1};
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn)(
               map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, v.kv, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_pages_attn_tc(const CUtensorMap &map, const PagesAttn &a, int sms, cudaStream_t s) {
    return a.pv.head_dim == 64 ? launch_rows<64>(map, a, sms, s) : launch_rows<128>(map, a, sms, s);
}

}  // namespace msd
