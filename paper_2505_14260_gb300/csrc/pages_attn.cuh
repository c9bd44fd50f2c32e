// How the attention over pages is cut into CTAs (shared by its two kernels).
//
// An item is a tile of packed rows of one sequence and one K/V head: packed row m is head
// h * G + m % G of row m / G, so the G query heads that share a K/V head read it together. An
// item has as many steps as its rows see key tiles: those of the first tokens that stay
// visible, then those from the window's edge to the last key. All items' steps, sequence by
// sequence, head by head, tile by tile, form one line that the CTAs cut into equal runs: a
// ragged batch, a causal triangle and one long sequence all load the SMs alike. Where a run
// ends inside an item, its CTAs leave partial results (O, max, sum) that a second launch
// joins in order. Lengths are read on the device; the cut depends on them alone. An item also
// costs what it takes to begin and end (queries, output): ITEM_STEPS steps of the line before
// its own (what the times of CTAs with many and with few items come to), so that many short
// sequences spread over the SMs like a few long ones.
#pragma once

#include "pages.h"

namespace msd {

// (the tensor cores' kernel, key tiles of 128: a pair of row tiles, or one; the other kernel's items begin and end quickly)
template <int KT, int ROWS>
constexpr int ITEM_STEPS = KT != 128 ? 0 : ROWS == 256 ? 4 : 3;

struct AttnSched {
    long long pre[ATTN_MAX_SEQS + 1];     // steps before each sequence
    int len[ATTN_MAX_SEQS], rows[ATTN_MAX_SEQS];
    int4 first;                           // this CTA's first item: sequence, head, tile, place in it
    long long per;                        // steps of a CTA
};

// The depth of node j of listed sequence i. Which tiles a window shows in full follows from depths being 0 .. nodes - 1;
// one that is not counts as the nearest (and is reported: check_depths).
__device__ __forceinline__ int node_depth(const PagesAttn &a, int i, int j) {
    return min(max(a.depth[(long)i * a.nodes + j], 0), a.nodes - 1);
}

// the steps of a tile of rows
struct TileRange {
    int sink_tiles, lo, steps;            // key tile of step j: j < sink_tiles ? j : lo + j - sink_tiles
};

template <int ROWS, int KT>
__device__ __forceinline__ TileRange tile_range(const PagesAttn &a, int len, int rows, int tile) {
    const int L = len - rows, m0 = tile * ROWS, m1 = min(rows * a.group, m0 + ROWS);
    const int hi = a.mask ? len : L + group_div(a, m1 - 1) + 1;
    TileRange t;
    int lo = 0, sink = 0;
    if (a.window) {
        lo = max(0, (a.mask ? L : L + group_div(a, m0)) - a.window + 1);
        sink = min(a.sinks, lo);
    }
    t.lo = lo / KT;
    t.sink_tiles = min((sink + KT - 1) / KT, t.lo);
    t.steps = t.sink_tiles + (hi + KT - 1) / KT - t.lo;
    return t;
}

// A run of steps of one item.
struct Segment {
    int i, h, tile;           // listed sequence, K/V head, tile of rows
    int j0, j1;               // steps [j0, j1)
    TileRange range;
};

// Fills s (whole CTA, THREADS threads; ends with a barrier). Sequences that cannot be read
// (ids, lengths or row counts out of range) get no steps and set the status word; behind a page
// operation that was not carried out no sequence gets any.
template <int ROWS, int KT, int THREADS>
__device__ void attn_schedule(const PagesAttn &a, AttnSched &s, int cta, int ctas) {
    __shared__ long long s_sum[THREADS / 32];
    const PagesView &v = a.pv;
    const int G = a.group, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int NW = THREADS / 32;
    // steps of each sequence: a thread's own loop over few tiles, a warp's over many
    bool many = false;
    for (int i = tid; i < a.b.n; i += THREADS) {
        const int seq = a.b.seqs[i], r0 = a.b.row_start[i], r1 = a.b.row_start[i + 1];
        const int held = *static_cast<volatile const int *>(v.refused);      // (asked for with the others, not before them)
        int len = 0, rows = r1 - r0;
        bool ok = (unsigned)seq < (unsigned)v.max_seqs && r0 >= 0 && rows >= 0 && r1 <= a.b.rows;
        if (ok) {
            len = v.len[seq];
            ok = len >= rows && len <= (long)v.max_pages * v.page && (!a.mask || rows <= a.nodes);
        }
        if (!ok && !held) set_status(v.status, ST_BAD_BATCH);
        if (!ok || held) rows = 0;
        s.len[i] = len;
        s.rows[i] = rows;
        const int tiles = (rows * G + ROWS - 1) / ROWS;
        long long w = 0;
        if (tiles > 4) many = true;
        else
            for (int t = 0; t < tiles; ++t) w += ITEM_STEPS<KT, ROWS> + tile_range<ROWS, KT>(a, len, rows, t).steps;
        s.pre[i + 1] = w * v.kv_heads;
    }
    if (__syncthreads_or(many)) {
        for (int i = warp; i < a.b.n; i += NW) {
            const int tiles = (s.rows[i] * G + ROWS - 1) / ROWS;
            if (tiles <= 4) continue;
            long long w = 0;
            for (int t = lane; t < tiles; t += 32) w += ITEM_STEPS<KT, ROWS> + tile_range<ROWS, KT>(a, s.len[i], s.rows[i], t).steps;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
            if (lane == 0) s.pre[i + 1] = w * v.kv_heads;
        }
        __syncthreads();
    }
    // inclusive sums
    long long carry = 0;
    for (int i0 = 0; i0 < a.b.n; i0 += THREADS) {
        const int i = i0 + tid;
        long long x = i < a.b.n ? s.pre[i + 1] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (i0) __syncthreads();
        if (lane == 31) s_sum[warp] = x;
        __syncthreads();
        long long before = carry;
        for (int w = 0; w < NW; ++w) {
            if (w < warp) before += s_sum[w];
            carry += s_sum[w];
        }
        if (i < a.b.n) s.pre[i + 1] = before + x;
    }
    if (tid == 0) s.pre[0] = 0;
    const long long per = max(1ll, (carry + ctas - 1) / ctas), x0 = per * cta;
    __syncthreads();
    if (warp == 0) {
        int4 f = make_int4(-1, 0, 0, 0);
        if (x0 < carry) {
            int lo = 0, hi = a.b.n;               // pre[lo] <= x0 < pre[hi], and pre[lo + 1] > x0
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s.pre[mid] <= x0) lo = mid;
                else hi = mid;
            }
            const long long w = (s.pre[lo + 1] - s.pre[lo]) / v.kv_heads;
            long long x = x0 - s.pre[lo];
            const int h = (int)(x / w);
            x -= h * w;
            const int tiles = (s.rows[lo] * G + ROWS - 1) / ROWS;
            int t0 = 0;
            for (; t0 < tiles; t0 += 32) {        // 32 tiles at a time
                const int t = t0 + lane;
                int inc = t < tiles ? ITEM_STEPS<KT, ROWS> + tile_range<ROWS, KT>(a, s.len[lo], s.rows[lo], t).steps : 0;
                const int own = inc;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, inc, o);
                    if (lane >= o) inc += y;
                }
                const unsigned past = __ballot_sync(0xffffffffu, inc > x);
                if (past) {
                    const int at = __ffs(past) - 1;
                    f = make_int4(lo, h, t0 + at, (int)(x - __shfl_sync(0xffffffffu, inc - own, at)));
                    break;
                }
                x -= __shfl_sync(0xffffffffu, inc, 31);
            }
        }
        if (lane == 0) {
            s.first = f;
            s.per = per;
        }
    }
    __syncthreads();
}

// The segments of a CTA's run, in order: every role of the CTA walks them by itself.
template <int ROWS, int KT>
struct AttnWalk {
    const PagesAttn &a;
    const AttnSched &s;
    int G, i, h, tile, place;             // place: of the line, within the item
    long long left;
    __device__ AttnWalk(const PagesAttn &a_, const AttnSched &s_) : a(a_), s(s_) {
        G = a.group;
        i = s.first.x;
        h = s.first.y;
        tile = s.first.z;
        place = s.first.w;
        left = i < 0 ? 0 : s.per;
    }
    __device__ bool next(Segment &g) {
        while (left > 0 && i < a.b.n) {
            g.i = i;
            g.h = h;
            g.tile = tile;
            g.range = tile_range<ROWS, KT>(a, s.len[i], s.rows[i], tile);
            const int end = ITEM_STEPS<KT, ROWS> + g.range.steps, stop = (int)min((long long)end, place + left);
            g.j0 = max(place - ITEM_STEPS<KT, ROWS>, 0);
            g.j1 = max(stop - ITEM_STEPS<KT, ROWS>, 0);
            left -= stop - place;
            place = 0;
            if (stop == end && ++tile * ROWS >= s.rows[i] * G) {
                tile = 0;
                if (++h == a.pv.kv_heads) {
                    h = 0;
                    do ++i;
                    while (i < a.b.n && s.rows[i] == 0);
                }
            }
            if (g.j1 > g.j0) return true;         // (else the run ends before the item's first step)
        }
        return false;
    }
};

// Where a segment's partial results go, if it is not a whole item: of a CTA's two places, the
// first for one that began in an earlier CTA.
__device__ __forceinline__ bool segment_whole(const Segment &g) { return g.j0 == 0 && g.j1 == g.range.steps; }
__device__ __forceinline__ long part_slot(const Segment &g, int cta) { return 2l * cta + (g.j0 > 0 ? 0 : 1); }

// The CTA that ends an item begun elsewhere names it for the joining launch (rows 0: none).
template <int ROWS, int KT>
__device__ void name_parts(const PagesAttn &a, const AttnSched &s, int cta) {
    AttnWalk<ROWS, KT> walk(a, s);
    Segment g;
    PartItem item{0, 0, 0, 0, 0};
    if (walk.next(g) && g.j0 > 0 && g.j1 == g.range.steps)
        item = PartItem{a.b.row_start[g.i], g.h, g.tile * ROWS, min(s.rows[g.i] * a.group - g.tile * ROWS, ROWS),
                        (int)((s.per * cta - g.j0) / s.per)};
    a.part_item[cta] = item;
}

// Reports depths out of range of the rows in the CTA's run, a thread every `step`-th of a segment's. (A call of its own,
// away from the loops: with the report where depths are used, in the bf16 kernel a tree took 24.1 us for 23.4 and 64 ragged
// tokens 77.3 for 76.2, without any depth to read.)
template <int ROWS, int KT>
__device__ __noinline__ void check_depths(const PagesAttn &a, const AttnSched &s, int first, int step) {
    AttnWalk<ROWS, KT> walk(a, s);
    Segment g;
    while (walk.next(g)) {
        const int live = a.n_nodes ? min(s.rows[g.i], a.n_nodes[g.i]) : s.rows[g.i];
        for (int r = group_div(a, g.tile * ROWS) + first; r < live && r * a.group < (g.tile + 1) * ROWS; r += step)
            if ((unsigned)a.depth[(long)g.i * a.nodes + r] >= (unsigned)a.nodes) set_status(a.pv.status, ST_BAD_BATCH);
    }
}

}  // namespace msd
