// The paged cache (include/msd.h, msd_pages_*): the pool's page operations, rotary
// positions on three axes, and the rotation of q and k with K and V into the pages.
//
// Page operations run on device state, without a host round trip: lengths, tables and
// reference counts live in the caller's arrays, and the free pages in a bitmap of the
// pool. A page that is not full belongs to one sequence, so appending never copies; forks
// share full pages only. Allocation takes the lowest free page ids in the order of the
// call's list, so a sequence of calls always gives the same tables. A call that cannot be
// carried out (too few pages, bad lists) changes nothing, sets the status word, and keeps the
// calls behind it from running until the host has seen that (refuse, in pages.h).
// Round trips bound the lists (launches by themselves, cold): freeing takes 4.5 to 6 us, planning
// 64 forks 8.7, reserving for 16 sequences 7.6, planning 16 compactions of 1027 tokens 14.6,
// positions of 20544 rows 6.0; bytes bound the moves (68 us there).
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>

#include "pages.h"

namespace msd {
namespace {

constexpr int PLAN_THREADS = 1024;     // of a planning CTA, at most
constexpr int PLAN_INTS = 6;           // per listed sequence: id, base, new length, first page that changes,
                                       // pages before, pages after

__device__ __forceinline__ bool seq_ok(const PagesView &v, int s) { return (unsigned)s < (unsigned)v.max_seqs; }

// a length that the table can hold (the caller's array, read before it bounds anything)
__device__ __forceinline__ bool len_ok(const PagesView &v, int len) { return len >= 0 && len <= (long)v.max_pages * v.page; }

__device__ __forceinline__ int *row_of(const PagesView &v, int s) { return v.table + (long)s * v.max_pages; }

// A reference to page `id` less; the last one frees it. (Adds and ors of whole numbers: the
// outcome does not depend on their order.)
__device__ __forceinline__ void drop_ref(const PagesView &v, int id) {
    if ((unsigned)id < (unsigned)v.n_pages && atomicSub(v.refs + id, 1) == 1)
        atomicOr(v.bits + (id >> 5), 1u << (id & 31));
}

// Exclusive prefix sum over the CTA; *total gets the sum. s: 33 ints of shared memory.
// cap > 0: no sum passes it (for x in 0 .. cap; where the total reaches it the prefixes are of no use).
__device__ __forceinline__ int block_scan(int x, int *s, int *total, int cap = 0) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    auto add = [&](int a, int b) { return cap ? min(a + b, cap) : a + b; };
    int inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc = add(inc, y);
    }
    __syncthreads();                    // (the previous scan's readers are done)
    if (lane == 31) s[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        int t = lane < nw ? s[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, t, o);
            if (lane >= o) t = add(t, y);
        }
        s[lane] = t;
    }
    __syncthreads();
    *total = s[nw - 1];
    return inc - x + (warp ? s[warp - 1] : 0);
}

// The same of pages that each of a list's sequences needs: sums stop at one more than there are (32 sequences may need
// 2^31 pages), which the callers refuse.
__device__ __forceinline__ int pages_scan(const PagesView &v, int need, int *s, int *total) {
    return block_scan(min(need, v.n_pages + 1), s, total, v.n_pages + 1);
}

// The `total` lowest free pages, ascending, into fresh[]; their bits cleared. Returns
// false, with nothing changed, where there are fewer. One CTA; s: 33 ints.
__device__ bool take_pages(const PagesView &v, int total, int *fresh, int *s) {
    const int nw = (v.n_pages + 31) >> 5;          // (the bitmap is padded to 16 bytes with zeros)
    int got = 0;
    for (int w0 = 0; got < total && w0 < nw; w0 += 4 * blockDim.x) {
        const int w = w0 + 4 * threadIdx.x;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (w < nw) u = *reinterpret_cast<const uint4 *>(v.bits + w);
        int sum;
        int at = got + block_scan(__popc(u.x) + __popc(u.y) + __popc(u.z) + __popc(u.w), s, &sum);
        unsigned x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned before = x[k];
            while (x[k] && at < total) {
                fresh[at++] = 32 * (w + k) + __ffs(x[k]) - 1;
                x[k] &= x[k] - 1;
            }
            if (x[k] != before) v.bits[w + k] = x[k];
        }
        got += sum;
    }
    __syncthreads();
    if (got >= total) return true;
    for (int i = threadIdx.x; i < got; i += blockDim.x) atomicOr(v.bits + (fresh[i] >> 5), 1u << (fresh[i] & 31));
    return false;
}

// ---- restore ---------------------------------------------------------------

__global__ void restore_clear_kernel(const PagesView v) {
    wait_prior();
    allow_dependents();
    for (int p = blockIdx.x * blockDim.x + threadIdx.x; p < v.n_pages; p += gridDim.x * blockDim.x) v.refs[p] = 0;
}

// One CTA a sequence: counts its pages, marks the rest of its row as none.
__global__ void restore_count_kernel(const PagesView v) {
    wait_prior();
    allow_dependents();
    const int s = blockIdx.x;
    const int len = v.len[s];
    const bool ok = len_ok(v, len);
    const int n = ok ? pages_of(len, v.page_shift, v.page) : 0;
    __syncthreads();
    if (!ok && threadIdx.x == 0) {
        v.len[s] = 0;
        set_status(v.status, ST_RANGE);
    }
    int *row = row_of(v, s);
    bool bad = false;
    for (int k = threadIdx.x; k < v.max_pages; k += blockDim.x) {
        const int id = row[k];
        if (k >= n) row[k] = -1;
        else if ((unsigned)id >= (unsigned)v.n_pages) bad = true;
        else atomicAdd(v.refs + id, 1);
    }
    if (bad) set_status(v.status, ST_RANGE);
}

// The free pages; a page that is not full and held by several sequences is reported.
__global__ void restore_bits_kernel(const PagesView v) {
    wait_prior();
    allow_dependents();
    for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < v.max_seqs; s += gridDim.x * blockDim.x) {
        const int len = v.len[s], id = len & (v.page - 1) ? row_of(v, s)[len >> v.page_shift] : -1;
        if ((unsigned)id < (unsigned)v.n_pages && v.refs[id] > 1) set_status(v.status, ST_RANGE);
    }
    const int words = (v.n_pages + 31) / 32;
    for (int w = (blockIdx.x * blockDim.x + threadIdx.x) >> 5; w < words; w += (gridDim.x * blockDim.x) >> 5) {
        const int p = 32 * w + (threadIdx.x & 31);
        const unsigned b = __ballot_sync(0xffffffffu, p < v.n_pages && v.refs[p] == 0);
        if ((threadIdx.x & 31) == 0) v.bits[w] = b;
    }
}

// ---- after an error --------------------------------------------------------

// (The operations read the mark beside their lists and look at it once those are there, so that it costs no round trip
// of its own.)

// Behind what the host had queued when it took `code` from the status word. The calls that were held back may run again
// if that was the refused operation's error. If it was another one's, the refusal is put where the host sees it next.
__global__ void resume_kernel(const PagesView v, int code) {
    wait_prior();
    allow_dependents();
    const int held = *v.refused;
    if (held && code == held) *v.refused = 0;
    else if (held) set_status(v.status, held);
}

// ---- free ------------------------------------------------------------------

// Every CTA looks through the whole list first, so that it is freed whole or not at all (a length that another CTA has
// set to 0 by then is as good as the one it was), then frees its share of it. A sequence listed twice is freed once
// (the exchange).
__global__ void __launch_bounds__(128) free_kernel(const PagesView v, int n, const int *seqs) {
    __shared__ int s_len;
    wait_prior();
    allow_dependents();
    const int held = *v.refused;          // (or by CTA 0 of this launch: then the others find the same)
    int code = 0;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int s = seqs[i];
        if (!seq_ok(v, s)) code = ST_BAD_BATCH;
        else if (!len_ok(v, v.len[s])) code = ST_RANGE;
    }
    if (code && !held && blockIdx.x == 0) refuse(v, code);
    if (__syncthreads_or(code | held)) return;
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        const int s = seqs[i];
        if (threadIdx.x == 0) s_len = atomicExch(v.len + s, 0);
        __syncthreads();
        const int pages = pages_of(s_len, v.page_shift, v.page);
        int *row = row_of(v, s);
        for (int k = threadIdx.x; k < pages; k += blockDim.x) {
            const int id = row[k];
            row[k] = -1;
            drop_ref(v, id);
        }
        __syncthreads();
    }
}

// ---- reserve ---------------------------------------------------------------

// One CTA. Per listed sequence the pages that its new rows need, a prefix sum over the
// list, the lowest free pages, and the tables' new entries.
__global__ void __launch_bounds__(PLAN_THREADS) reserve_kernel(const PagesView v, const BatchView b, int *mark, int *off,
                                                               int *fresh) {
    __shared__ int s_scan[33], s_bad;
    wait_prior();
    allow_dependents();
    const int held = *v.refused;
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
    int total = 0;
    for (int i0 = 0; i0 < b.n; i0 += blockDim.x) {
        const int i = i0 + threadIdx.x;
        int need = 0;
        if (i < b.n) {
            const int s = b.seqs[i];
            const int add = b.row_start[i + 1] - b.row_start[i];
            bool ok = seq_ok(v, s) && add >= 0;
            if (ok && atomicExch(mark + s, 1) != 0) ok = false;
            if (ok) {
                const int len = v.len[s];
                const long after = (long)len + add;
                ok = len_ok(v, len) && after <= (long)v.max_pages * v.page;
                if (ok) need = pages_of((int)after, v.page_shift, v.page) - pages_of(len, v.page_shift, v.page);
            }
            if (!ok) s_bad = 1;
        }
        int sum;
        const int at = pages_scan(v, need, s_scan, &sum);
        if (i < b.n) off[i] = total + at;
        total = min(total + sum, v.n_pages + 1);         // (more than there are: refused below)
    }
    __syncthreads();
    for (int i = threadIdx.x; i < b.n; i += blockDim.x)
        if (seq_ok(v, b.seqs[i])) mark[b.seqs[i]] = 0;
    if (held) return;
    if (s_bad) {
        if (threadIdx.x == 0) refuse(v, ST_BAD_BATCH);
        return;
    }
    if (total > v.n_pages || !take_pages(v, total, fresh, s_scan)) {
        if (threadIdx.x == 0) refuse(v, ST_NO_PAGES);
        return;
    }
    for (int x = threadIdx.x; x < total; x += blockDim.x) {
        int lo = 0, hi = b.n;                            // the last i with off[i] <= x
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (off[mid] <= x) lo = mid;
            else hi = mid;
        }
        const int s = b.seqs[lo], id = fresh[x];
        row_of(v, s)[pages_of(v.len[s], v.page_shift, v.page) + x - off[lo]] = id;
        v.refs[id] = 1;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < b.n; i += blockDim.x) v.len[b.seqs[i]] += b.row_start[i + 1] - b.row_start[i];
}

// ---- fork ------------------------------------------------------------------

// One CTA: checks the lists and takes the pages that each copy starts with (its partial
// last page; all of them for a deep one). ok_out: whether fork_apply_kernel may go on.
__global__ void __launch_bounds__(PLAN_THREADS) fork_plan_kernel(const PagesView v, int n, const int *src, const int *dst,
                                                                 int deep, int *mark, int *off, int *fresh, int *ok_out) {
    __shared__ int s_scan[33], s_bad;
    wait_prior();
    allow_dependents();
    const int held = *v.refused;
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
    int total = 0;
    for (int i0 = 0; i0 < n; i0 += blockDim.x) {
        const int i = i0 + threadIdx.x;
        int need = 0;
        if (i < n) {
            const int a = src[i], d = dst[i];
            bool ok = seq_ok(v, a) && seq_ok(v, d);
            if (ok && atomicExch(mark + d, 1) != 0) ok = false;
            if (ok && (v.len[d] != 0 || !len_ok(v, v.len[a]))) ok = false;
            if (ok) {
                const int len = v.len[a];
                need = deep ? pages_of(len, v.page_shift, v.page) : (len & (v.page - 1)) != 0;
            }
            if (!ok) s_bad = 1;
        }
        int sum;
        const int at = pages_scan(v, need, s_scan, &sum);
        if (i < n) off[i] = total + at;
        total = min(total + sum, v.n_pages + 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x)
        if (seq_ok(v, src[i]) && mark[src[i]] != 0) s_bad = 1;       // (a sequence is not copied while it is made)
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x)
        if (seq_ok(v, dst[i])) mark[dst[i]] = 0;
    const bool bad = s_bad != 0;
    const bool ok = !bad && !held && total <= v.n_pages && take_pages(v, total, fresh, s_scan);
    if (threadIdx.x == 0) {
        *ok_out = ok;
        if (!ok && !held) refuse(v, bad ? ST_BAD_BATCH : ST_NO_PAGES);
    }
}

// CTA (i, layer, z of gridDim.z): the copies' tables and counts (layer 0, z 0), and the tokens of the pages that are
// copied: the pieces of K and V of all heads, 16 bytes a thread and four requests in flight, the (page, head)s spread
// over z.
template <int ESZ>
__global__ void __launch_bounds__(256) fork_apply_kernel(const PagesView v, const int *src, const int *dst, int deep,
                                                         const int *off, const int *fresh, const int *ok) {
    wait_prior();
    allow_dependents();
    if (!*ok) return;
    const int i = blockIdx.x, layer = blockIdx.y;
    const int a = src[i], d = dst[i];
    const int len = v.len[a], n = pages_of(len, v.page_shift, v.page);
    const int first = deep ? 0 : len >> v.page_shift;         // pages before it are shared
    const int *from = row_of(v, a), *ids = fresh + off[i];
    if (layer == 0 && blockIdx.z == 0) {
        int *to = row_of(v, d);
        for (int k = threadIdx.x; k < n; k += blockDim.x) {
            if (k < first) {
                const int id = from[k];
                to[k] = id;
                if ((unsigned)id < (unsigned)v.n_pages) atomicAdd(v.refs + id, 1);
            } else {
                to[k] = ids[k - first];
                v.refs[ids[k - first]] = 1;
            }
        }
        if (threadIdx.x == 0) v.len[d] = len;
    }
    const int heads = 2 * v.kv_heads, run16 = v.head_dim * ESZ / 16;     // of a page; 16-byte pieces of a token's head
    const int stride16 = v.page * run16;                                 // pieces of a head's page
    const long pe16 = v.page_elems() * ESZ / 16;
    uint4 *kv = static_cast<uint4 *>(v.kv) + (long)layer * v.n_pages * pe16;
    const int per = (heads + (int)gridDim.z - 1) / (int)gridDim.z;       // heads of a CTA, or more than one page's
    const int splits = (heads + per - 1) / per;
    for (int w = blockIdx.z; w < (n - first) * splits; w += gridDim.z) {
        const int k = first + w / splits, h0 = w % splits * per, hn = min(per, heads - h0);
        if ((unsigned)from[k] >= (unsigned)v.n_pages) continue;
        const int live = min(v.page, len - (k << v.page_shift)) * run16, all = hn * live;
        const uint4 *s = kv + from[k] * pe16 + h0 * stride16;
        uint4 *t = kv + ids[k - first] * pe16 + h0 * stride16;
        for (int x0 = threadIdx.x; x0 < all; x0 += 4 * blockDim.x) {
            uint4 r[4];
            int at[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int x = x0 + u * blockDim.x;
                at[u] = x / live * stride16 + x % live;
                if (x < all) r[u] = s[at[u]];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (x0 + u * (int)blockDim.x < all) t[at[u]] = r[u];
        }
    }
}

// ---- compact ---------------------------------------------------------------

struct CompactArgs {
    const int *keep;         // [n][stride], or null: the first n_keep rows
    int stride;
    const int *n_keep;
    int *mark, *off, *fresh, *plan, *old_table, *rank;
    int *flags;              // 0: tickets, 1: a bad list, 2: the plan holds
};

// CTA i: checks its keep list, finds the first row that moves and the pages from there on
// that are shared with others (they are replaced); the last CTA takes the new pages.
__global__ void __launch_bounds__(PLAN_THREADS) compact_plan_kernel(const PagesView v, const BatchView b,
                                                                    const CompactArgs c) {
    __shared__ int s_scan[33], s_first, s_bad, s_last;
    wait_prior();
    allow_dependents();
    const int held = *v.refused;                      // (set by the launch's last CTA at the earliest, so the same for all)
    const int i = blockIdx.x;
    const int s = b.seqs[i];
    const int rows = b.row_start[i + 1] - b.row_start[i];
    const int nk = c.n_keep[i];
    if (threadIdx.x == 0) {
        s_bad = !seq_ok(v, s) || rows < 0 || nk < 0 || nk > rows || (c.keep && nk > c.stride);
        if (!s_bad) s_bad = v.len[s] < rows || !len_ok(v, v.len[s]) || atomicExch(c.mark + s, 1) != 0;
        s_first = nk;
    }
    __syncthreads();
    int need = 0;
    if (!s_bad) {                                     // (the same for the CTA: nobody writes it before the barrier below)
        int first = nk;
        bool bad = false;
        if (c.keep) {
            const int *keep = c.keep + (long)i * c.stride;
            for (int j = threadIdx.x; j < nk; j += blockDim.x) {
                const int k = keep[j];
                if (k >= rows || k <= (j ? keep[j - 1] : -1)) bad = true;
                if (k != j) first = min(first, j);
            }
        }
        __syncthreads();
        if (bad) s_bad = 1;
        if (first < nk) atomicMin(&s_first, first);
        __syncthreads();
        const int len = v.len[s], base = len - rows, after = base + nk;
        const int k0 = (base + s_first) >> v.page_shift;
        const int was = pages_of(len, v.page_shift, v.page), now = pages_of(after, v.page_shift, v.page);
        const int *row = row_of(v, s);
        int *old = c.old_table + (long)i * v.max_pages, *rank = c.rank + (long)i * v.max_pages;
        for (int p0 = k0; p0 < was; p0 += blockDim.x) {
            const int k = p0 + threadIdx.x;
            int shared = 0;
            if (k < was) {
                int id = row[k];
                if ((unsigned)id >= (unsigned)v.n_pages) {         // (no page: a table that restore reported)
                    id = 0;
                    s_bad = 1;
                }
                old[k] = id;
                shared = k < now && v.refs[id] > 1;
            }
            int sum;
            const int at = block_scan(shared, s_scan, &sum);
            if (k < was) rank[k] = shared ? need + at : -1;
            need += sum;
        }
        if (threadIdx.x == 0) {
            int *p = c.plan + PLAN_INTS * i;
            p[0] = s; p[1] = base; p[2] = after; p[3] = k0; p[4] = was; p[5] = now;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        c.off[i] = need;
        if (s_bad) atomicExch(c.flags + 1, 1);
        __threadfence();
        s_last = atomicAdd(c.flags, 1) == (int)gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    int total = 0;
    for (int i0 = 0; i0 < b.n; i0 += blockDim.x) {
        const int x = i0 + threadIdx.x;
        int sum;
        const int at = pages_scan(v, x < b.n ? __ldcg(c.off + x) : 0, s_scan, &sum);
        if (x < b.n) {
            c.off[x] = total + at;
            if (seq_ok(v, b.seqs[x])) c.mark[b.seqs[x]] = 0;
        }
        total = min(total + sum, v.n_pages + 1);
    }
    const bool bad = __ldcg(c.flags + 1) != 0;
    const bool ok = !bad && !held && total <= v.n_pages && take_pages(v, total, c.fresh, s_scan);
    __syncthreads();
    if (threadIdx.x == 0) {
        c.flags[0] = 0;
        c.flags[1] = 0;
        c.flags[2] = ok;
        if (!ok && !held) refuse(v, bad ? ST_BAD_BATCH : ST_NO_PAGES);
    }
}

constexpr int MOVE_TOKENS = 1024;      // whose places a CTA lays out at once

// The tables and counts, a CTA per sequence, and the moves. A CTA first lays out where the next MOVE_TOKENS kept tokens
// come from and go to (three round trips), then moves them: `lanes` threads hold one token's head of one (layer, K
// or V, head), 16 bytes each; `side` tokens go side by side and U follow one another, all requested before any is stored
// (side > 1: and the CTA's barrier between). keep[j] >= j, so a token's old place is not overwritten before the batch
// that holds it has been read, and later batches lie behind it. Wide lists (side 16: 128 tokens a batch) are bound by
// bytes; for an accepted path (side 1) a CTA takes 16 heads, and the round trips of the lookups bound it.
template <int ESZ, int U>
__global__ void __launch_bounds__(256) compact_apply_kernel(const PagesView v, const CompactArgs c, int groups, int side) {
    __shared__ long s_from[MOVE_TOKENS], s_to[MOVE_TOKENS];   // 16-byte pieces from the layer's first; s_from -1: stays
    wait_prior();
    allow_dependents();
    if (!c.flags[2]) return;
    const int i = blockIdx.y;
    const int *p = c.plan + PLAN_INTS * i;
    const int s = p[0], base = p[1], after = p[2], k0 = p[3], was = p[4], now = p[5];
    const int *old = c.old_table + (long)i * v.max_pages, *rank = c.rank + (long)i * v.max_pages;
    const int *ids = c.fresh + c.off[i];
    if (blockIdx.x == 0) {
        int *row = row_of(v, s);
        for (int k = k0 + threadIdx.x; k < was; k += blockDim.x) {
            const int r = rank[k];
            if (k >= now) {
                row[k] = -1;
                drop_ref(v, old[k]);
            } else if (r >= 0) {
                row[k] = ids[r];
                v.refs[ids[r]] = 1;
                drop_ref(v, old[k]);
            }
        }
        if (threadIdx.x == 0) v.len[s] = after;
    }
    const int lanes = v.head_dim * ESZ / 16, unit = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    const int group = blockIdx.x * (256 / lanes / side) + unit / side, tok = unit % side;
    const int layer = group / (2 * v.kv_heads), kvh = group - layer * 2 * v.kv_heads;
    const long pe16 = v.page_elems() * ESZ / 16;
    uint4 *kv = static_cast<uint4 *>(v.kv) + (long)layer * v.n_pages * pe16 + (long)kvh * v.page * lanes + lane;
    const int *keep = c.keep ? c.keep + (long)i * c.stride : nullptr;
    for (int c0 = k0 << v.page_shift; c0 < after; c0 += MOVE_TOKENS) {
        const int n = min(MOVE_TOKENS, after - c0);
        __syncthreads();
        for (int x = threadIdx.x; x < n; x += 256) {
            const int t = c0 + x, k = t >> v.page_shift, rk = rank[k];
            const int from = t < base || !keep ? t : base + keep[t - base];
            const int of = old[from >> v.page_shift], in = rk >= 0 ? ids[rk] : old[k];
            s_from[x] = of != in || from != t ? of * pe16 + (long)(from & (v.page - 1)) * lanes : -1;
            s_to[x] = in * pe16 + (long)(t & (v.page - 1)) * lanes;
        }
        __syncthreads();
        for (int t0 = 0; t0 < n; t0 += U * side) {
            uint4 r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = t0 + u * side + tok;
                if (t < n && group < groups && s_from[t] >= 0) r[u] = kv[s_from[t]];
            }
            if (side > 1) __syncthreads();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = t0 + u * side + tok;
                if (t < n && group < groups && s_from[t] >= 0) kv[s_to[t]] = r[u];
            }
        }
    }
}

// ---- rotary positions ------------------------------------------------------

constexpr int SPAN_TILE = 256;

// Positions of a sequence's rows on three axes: CTA (i, chunk of 256 rows), a row a thread.
// A span of t * h * w rows moves the position by its largest extent alone, so a row's
// position is its number less the sum of what the spans before it fall short. The spans
// come in tiles of 256, with a prefix sum of those shortfalls and a binary search.
__global__ void __launch_bounds__(SPAN_TILE) positions_kernel(const PagesView v, const BatchView b, const int *span_start,
                                                              const int *spans, int n_spans, const int *first, int *pos,
                                                              long pos_stride, int *next) {
    __shared__ int s_scan[33];
    __shared__ int s_row[SPAN_TILE], s_size[SPAN_TILE], s_less[SPAN_TILE], s_before[SPAN_TILE];
    wait_prior();
    allow_dependents();
    const int i = blockIdx.x;
    const int r0 = b.row_start[i], rows = b.row_start[i + 1] - r0;
    const int a = span_start ? span_start[i] : 0, z = span_start ? span_start[i + 1] : 0;
    const int start = first ? first[i] : 0;
    if (rows < 0 || r0 < 0 || (long)r0 + rows > b.rows || a < 0 || z < a || z > n_spans) {
        if (threadIdx.x == 0) set_status(v.status, ST_BAD_BATCH);
        return;
    }
    bool bad = false;
    int carry = 0;
    for (int c0 = blockIdx.y * SPAN_TILE; c0 == 0 || c0 < rows; c0 += gridDim.y * SPAN_TILE) {
        const int r = c0 + threadIdx.x;
        int span = -1, s_at = 0, size = 0, less = 0, before = 0;      // the last span that starts at or before the row
        carry = 0;
        for (int t0 = a; t0 < z; t0 += SPAN_TILE) {
            const int k = t0 + threadIdx.x;
            int my_row = 0x7fffffff, my_size = 0, my_less = 0;
            if (k < z) {
                const int *sp = spans + 5l * k;
                const long t = sp[1], h = sp[2], w = sp[3], step = sp[4];
                const long end = k + 1 < z ? sp[5] : rows;            // the next span's first row
                const bool ok = sp[0] >= 0 && end <= rows && t > 0 && h > 0 && w > 0 && t <= rows && h <= rows &&
                                w <= rows && t * h <= rows && t * h * w <= end - sp[0] && step > 0 &&
                                (t - 1) * step < (1l << 30);
                if (ok) {
                    my_row = sp[0];
                    my_size = (int)(t * h * w);
                    my_less = my_size - (int)max(max((t - 1) * step + 1, h), w);
                } else {
                    my_row = max(sp[0], 0);
                    bad = true;
                }
            }
            int sum;
            const int at = block_scan(my_less, s_scan, &sum);
            s_row[threadIdx.x] = my_row;
            s_size[threadIdx.x] = my_size;
            s_less[threadIdx.x] = my_less;
            s_before[threadIdx.x] = carry + at;
            __syncthreads();
            int lo = -1, hi = min(SPAN_TILE, z - t0);
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_row[mid] <= r) lo = mid;
                else hi = mid;
            }
            if (lo >= 0) {
                span = t0 + lo;
                s_at = s_row[lo];
                size = s_size[lo];
                less = s_less[lo];
                before = s_before[lo];
            }
            carry += sum;
            __syncthreads();
        }
        if (r < rows) {
            int p = start + r, x = 0, y = 0, u = 0;
            if (span >= 0 && r - s_at < size) {
                const int *sp = spans + 5l * span;
                const int k = r - s_at, hw = sp[2] * sp[3];
                p -= before + k;
                x = k / hw * sp[4];
                y = k / sp[3] % sp[2];
                u = k % sp[3];
            } else if (span >= 0) {
                p -= before + less;
            }
            pos[r0 + r] = p + x;
            pos[pos_stride + r0 + r] = p + y;
            pos[2 * pos_stride + r0 + r] = p + u;
        }
    }
    if (bad) set_status(v.status, ST_BAD_BATCH);
    if (next && blockIdx.y == 0 && threadIdx.x == 0) next[i] = start + rows - carry;
}

// ---- rotation and append ---------------------------------------------------

struct RopeArgs {
    const void *q, *k, *v;
    long ldq, ldk, ldv;
    const int *pos;
    long pos_stride;
    void *out;
    long ldo;
    int layer, half;         // half: rotated pairs of a head
};

// G elements as they are in memory
template <typename T, int G>
struct Run {
    uint4 w[G * sizeof(T) / 16];
    __device__ __forceinline__ void load(const T *g) {
#pragma unroll
        for (int i = 0; i < (int)(G * sizeof(T) / 16); ++i) w[i] = reinterpret_cast<const uint4 *>(g)[i];
    }
    __device__ __forceinline__ void to(float *x) const {
#pragma unroll
        for (int i = 0; i < (int)(G * sizeof(T) / 16); ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (sizeof(T) == 4) {
                    x[4 * i + k] = __uint_as_float(u[k]);
                } else {
                    x[8 * i + 2 * k] = __uint_as_float(u[k] << 16);
                    x[8 * i + 2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
                }
            }
        }
    }
};
template <typename T>
struct Run<T, 1> {
    T w;
    __device__ __forceinline__ void load(const T *g) { w = *g; }
    __device__ __forceinline__ void to(float *x) const { x[0] = (float)w; }
};

template <typename T, int G>
__device__ __forceinline__ void store_run(T *g, const float *x) {
    if constexpr (G == 1) {
        if constexpr (sizeof(T) == 4) *g = x[0];
        else *g = __float2bfloat16_rn(x[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < G; e += 4) *reinterpret_cast<float4 *>(g + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
    } else {
        uint32_t u[G / 2];
#pragma unroll
        for (int e = 0; e < G; e += 2) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[e], x[e + 1]);
            u[e / 2] = *reinterpret_cast<const uint32_t *>(&h);
        }
        static_assert(G == 8 || sizeof(T) == 4, "runs of 8 elements");
        *reinterpret_cast<uint4 *>(g) = make_uint4(u[0], u[1], u[2], u[3]);
    }
}

// The slot of a row: elements from the layer's first to its K of head 0, or -1 (none, or on a page that other sequences
// hold as well). Whole warp. Up to 32 sequences the lanes hold all of the list after one round trip (then the length, the
// page, its count); more are searched.
__device__ __forceinline__ long row_slot(const PagesView &v, const BatchView &b, int row) {
    const int lane = threadIdx.x & 31;
    int first, next, s;
    if (b.n <= 32) {
        const int start = lane < b.n ? b.row_start[lane] : 0x7fffffff, seq = lane < b.n ? b.seqs[lane] : -1;
        const int end = b.row_start[b.n];
        const int i = max(__popc(__ballot_sync(0xffffffffu, start <= row)) - 1, 0);
        first = __shfl_sync(0xffffffffu, start, i);
        next = i + 1 < b.n ? __shfl_sync(0xffffffffu, start, i + 1) : end;
        s = __shfl_sync(0xffffffffu, seq, i);
    } else {
        const int i = row_owner(b.row_start, b.n, row);
        first = b.row_start[i];
        next = b.row_start[i + 1];
        s = b.seqs[i];
    }
    if ((unsigned)s >= (unsigned)v.max_seqs || row < first || row >= next) return -1;
    const int slot = v.len[s] - next + row;
    if (slot < 0 || slot >= (long)v.max_pages * v.page) return -1;
    const int id = v.table[(long)s * v.max_pages + (slot >> v.page_shift)];
    return (unsigned)id < (unsigned)v.n_pages && v.refs[id] <= 1 ? id * v.page_elems() + (slot & (v.page - 1)) * v.head_dim : -1;
}

constexpr int ROPE_ROWS = 32, ROPE_THREADS = 256;      // of a CTA, at most

// CTA (P * side rows, a chunk of heads): a thread takes 2 G elements of one head, G of them and the G that they pair
// with (past the rotated part: 2 G in a row), of P rows, all requested first; where a row's heads do not fill the CTA,
// `side` rows lie side by side. Meanwhile a warp a row finds its slot (four round trips; only where the chunk has K or V
// heads) and the CTA the rows' sines. The angle in turns is the product of the position and a 64-bit fraction mod 1,
// which whole-number arithmetic gives exactly at any position; its upper 32 bits go to sincospi. Bytes bound it: the
// rows are read and written once.
template <typename TS, typename TD, int G, int P>
__global__ void __launch_bounds__(ROPE_THREADS) rope_append_kernel(const PagesView v, const BatchView b,
                                                                   const __grid_constant__ RopeTable rt, const RopeArgs a,
                                                                   int chunk, int side) {
    __shared__ float2 s_cs[ROPE_ROWS][MAX_ROT_PAIRS];
    __shared__ long s_slot[ROPE_ROWS];                        // elements from the layer's first to the row's K of head 0
    wait_prior();
    allow_dependents();
    const int hd = v.head_dim, units = hd / (2 * G), tid = threadIdx.x;
    const int h0 = blockIdx.y * chunk, hn = min(chunk, v.heads + 2 * v.kv_heads - h0);
    const int row0 = blockIdx.x * P * side, rows = min(P * side, b.rows - row0);
    const int at = tid / (chunk * units), rest = tid - at * chunk * units, head = h0 + rest / units, unit = rest % units;
    const int held = *v.refused;                              // (asked for first, looked at before anything is written)
    const bool live = at < side && head < h0 + hn;
    // first elements of the two runs
    const bool in = unit * G < a.half;
    const int e0 = in ? unit * G : 2 * a.half + 2 * (unit * G - a.half), e1 = in ? e0 + a.half : e0 + G;
    const bool is_q = head < v.heads, is_k = !is_q && head < v.heads + v.kv_heads;
    const TS *src = static_cast<const TS *>(is_q ? a.q : is_k ? a.k : a.v) +
                    (long)(is_q ? head : is_k ? head - v.heads : head - v.heads - v.kv_heads) * hd;
    const long ld = is_q ? a.ldq : is_k ? a.ldk : a.ldv;
    Run<TS, G> in0[P], in1[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int u = i * side + at;
        if (live && u < rows) {
            in0[i].load(src + (row0 + u) * ld + e0);
            in1[i].load(src + (row0 + u) * ld + e1);
        }
    }
    for (int e = tid; e < rows * a.half; e += blockDim.x) {
        const int u = e / a.half, pair = e - u * a.half;
        const long p = a.pos[rt.axis[pair] * a.pos_stride + row0 + u];
        const int angle = (int)(((unsigned long long)p * rt.turn[pair]) >> 32);
        float s, c;
        sincospif((float)angle * 0x1p-31f, &s, &c);
        s_cs[u][pair] = make_float2(c, s);
    }
    if (h0 + hn > v.heads) {
        for (int u = tid >> 5; u < rows; u += blockDim.x >> 5) {
            const long slot = row_slot(v, b, row0 + u);
            if ((tid & 31) == 0) {
                s_slot[u] = slot;
                if (slot < 0 && !held) set_status(v.status, ST_RANGE);
            }
        }
    }
    __syncthreads();
    if (!live || held) return;
    TD *dst = is_q ? static_cast<TD *>(a.out) + row0 * a.ldo + (long)head * hd
                   : static_cast<TD *>(v.kv) + (long)a.layer * v.n_pages * v.page_elems() + (long)(head - v.heads) * v.page * hd;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int u = i * side + at;
        if (u >= rows || (!is_q && s_slot[u] < 0)) continue;
        TD *to = dst + (is_q ? u * a.ldo : s_slot[u]);
        float f[G], w[G];
        in0[i].to(f);
        in1[i].to(w);
        if (in && (is_q || is_k)) {
#pragma unroll
            for (int e = 0; e < G; ++e) {
                const float2 cs = s_cs[u][e0 + e];
                const float y = f[e], z = w[e];
                f[e] = y * cs.x - z * cs.y;
                w[e] = z * cs.x + y * cs.y;
            }
        }
        store_run<TD, G>(to + e0, f);
        store_run<TD, G>(to + e1, w);
    }
}

template <typename TS, typename TD>
cudaError_t launch_rope(const msd_pages *p, const BatchView &b, const RopeArgs &a, cudaStream_t s) {
    const int heads = p->cfg.n_heads + 2 * p->cfg.n_kv_heads;
    auto go = [&](auto kernel, int run, int P) {
        // the heads in even chunks of up to 192 threads (large CTAs leave an SM's registers half used); rows side by
        // side where they are few
        const int units = p->cfg.head_dim / (2 * run), chunks = (heads * units + 191) / 192;
        const int chunk = (heads + chunks - 1) / chunks, side = std::max(1, std::min(192 / (chunk * units), ROPE_ROWS / P));
        const int threads = (side * chunk * units + 31) / 32 * 32, rows = P * side;
        const cudaError_t e = launch_chain(kernel, dim3((b.rows + rows - 1) / rows, (heads + chunk - 1) / chunk), dim3(threads), 0,
                                           s, p->v, b, p->rope, a, chunk, side);
        note_launch();
        return e;
    };
    // runs of 8 elements where the rotated part allows it, else pair by pair; two rows to a thread once that leaves every
    // SM some CTAs. One and two rows a thread from fp32 (from bf16) rows of 96 heads of 128, in a loop: 60 rows 3.7, 3.7 us
    // (3.5, 3.7), 124 rows 4.5, 4.3 (4.1, 4.1), 186 rows, where the rule turns, 4.7, 4.6 (4.5, 4.5), 240 rows 5.8, 5.0
    // (5.2, 4.9). 20544 bf16 rows of 48 heads take 93 us by themselves, 5.4 TB/s (one row a thread 121 where two took 90).
    if (a.half % 8) return go(rope_append_kernel<TS, TD, 1, 1>, 1, 1);
    const long each = (long)b.rows * heads * p->cfg.head_dim / p->sms;        // elements of an SM
    return each >= 15000 ? go(rope_append_kernel<TS, TD, 8, 2>, 8, 2) : go(rope_append_kernel<TS, TD, 8, 1>, 8, 1);
}

}  // namespace
}  // namespace msd

using namespace msd;

namespace {

msd_status pfail(msd_pages *p, msd_status st, const char *msg) {
    snprintf(p->err, sizeof p->err, "%s", msg);
    return st;
}

template <typename... KArgs, typename... Args>
cudaError_t chain(void (*kernel)(KArgs...), dim3 grid, int threads, cudaStream_t s, Args &&...args) {
    const cudaError_t e = launch_chain(kernel, grid, dim3(threads), 0, s, std::forward<Args>(args)...);
    note_launch();
    return e;
}

// What every call begins with: an error that was pending before it, the pool's device, and
// the status word of earlier calls. Reporting a refusal lets later calls run again: the mark that holds
// them back is cleared on the stream, behind the calls that it is for. A call that is being recorded
// cannot do that (it would be recorded too), so the word stays for the next one that is not.
msd_status enter(msd_pages *p, const char *call, cudaStream_t s) {
    p->err[0] = 0;
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) {
        fprintf(stderr, "msd: %s: found a pending CUDA error: %s\n", call, cudaGetErrorString(e));
        return pfail(p, MSD_ERR_CUDA, "a CUDA error was pending before the call");
    }
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != p->dev)
        return pfail(p, MSD_ERR_INVALID, "the pool belongs to another device than the current one");
    int code = *p->status_host;
    if (code != 0) {
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusActive;
        if (cudaStreamIsCapturing(s, &capture) != cudaSuccess) cudaGetLastError();       // (the default stream, while another records)
        if (capture == cudaStreamCaptureStatusNone) {
            *p->status_host = 0;
            const cudaError_t failed = chain(resume_kernel, dim3(1), 1, s, p->v, code);
            if (failed != cudaSuccess) {                // (still to be reported)
                *p->status_host = code;
                return pfail(p, MSD_ERR_CUDA, cudaGetErrorString(failed));
            }
        }
        code &= ~ST_REFUSED;
        if (code == ST_NO_PAGES)
            return pfail(p, MSD_ERR_CAPACITY, "an earlier call needed more free pages than there were; it changed nothing");
        snprintf(p->err, sizeof p->err, "an earlier call set the device status word (code %d: %s)", code,
                 code == ST_BAD_BATCH ? "sequences, row counts or lists out of range"
                 : code == ST_RANGE   ? "an index outside its buffer was skipped"
                 : code == ST_TIMEOUT ? "a bounded wait ran out"
                                      : "unknown");
        return MSD_ERR_DEVICE;
    }
    return MSD_OK;
}

msd_status leave(msd_pages *p, cudaError_t e) {
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) return MSD_OK;
    return pfail(p, MSD_ERR_CUDA, cudaGetErrorString(e));
}

bool batch_view(const msd_pages *p, const msd_batch *b, BatchView *out) {
    if (!b || b->n < 1 || b->n > p->cfg.max_seqs || !b->seqs || !b->row_start || b->rows < 0) return false;
    *out = BatchView{b->n, b->rows, b->seqs, b->row_start};
    return true;
}

// Threads of a planning CTA: a thread for each of n entries and each 128 pages of the free bitmap. (Its barriers cost
// more the more threads there are.)
int plan_threads(const msd_pages *p, int n) {
    return std::min(PLAN_THREADS, std::max(128, (std::max(n, p->cfg.n_pages / 128 + 1) + 31) / 32 * 32));
}

bool valid(const msd_pages_config *c) {
    if (c->dtype != MSD_F32 && c->dtype != MSD_BF16) return false;
    if (c->n_layers < 1 || c->n_layers > 65535 || c->n_kv_heads < 1 || c->n_heads < 1 || c->n_heads > 4096) return false;
    if (c->n_heads % c->n_kv_heads || c->n_heads / c->n_kv_heads > 64) return false;
    if (c->head_dim != 64 && c->head_dim != 128) return false;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return false;
    if (c->n_pages < 1 || c->max_seqs < 1 || c->max_seqs > 65535 || c->max_pages < 1) return false;
    if ((long)c->max_pages * c->page_size > 1l << 30 || c->n_pages > 1 << 30) return false;
    // rows of head_dim elements in the pool: what a tensor copy's signed coordinate reaches
    if ((long)c->n_layers * c->n_pages > (1l << 31) / (2l * c->n_kv_heads * c->page_size)) return false;
    if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 2) return false;
    const int half = c->rot_dim / 2, *s = c->rot_section;
    if (s[0] < 0 || s[1] < 0 || s[2] < 0 || (long)s[0] + s[1] + s[2] != half) return false;
    if (c->rot_interleaved != 0 && c->rot_interleaved != 1) return false;
    // taking turns, height and width have all their pairs before the last one
    if (c->rot_interleaved && ((s[1] && 3 * s[1] - 2 >= half) || (s[2] && 3 * s[2] - 1 >= half))) return false;
    return half == 0 || (c->rope_base >= 1.f && c->rope_base < INFINITY);
}

}  // namespace

extern "C" {

msd_status msd_pages_create(const msd_pages_config *cfg, const msd_pages_buffers *buf, msd_pages **out) {
    if (out) *out = nullptr;
    if (!cfg || !buf || !out || !valid(cfg)) return MSD_ERR_INVALID;
    if (!buf->kv || !buf->table || !buf->len || !buf->refs) return MSD_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(buf->kv) % 16) return MSD_ERR_INVALID;
    msd_pages *p = new (std::nothrow) msd_pages();
    if (!p) return MSD_ERR_OOM;
    p->cfg = *cfg;
    int shift = 0;
    while ((1 << shift) < cfg->page_size) ++shift;
    const int half = cfg->rot_dim / 2;
    for (int i = 0; i < half; ++i) {
        const double turns = std::pow((double)cfg->rope_base, -2.0 * i / cfg->rot_dim) / (2.0 * 3.14159265358979323846);
        p->rope.turn[i] = (unsigned long long)std::ldexp(turns, 64);       // (at most 1 / 2 pi of a turn)
        const int *s = cfg->rot_section;
        p->rope.axis[i] = !cfg->rot_interleaved ? (i >= s[0]) + (i >= s[0] + s[1])
                          : i % 3 == 1 && i < 3 * s[1] ? 1
                          : i % 3 == 2 && i < 3 * s[2] ? 2
                                                       : 0;
    }
    bool ok = cudaGetDevice(&p->dev) == cudaSuccess &&
              cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, p->dev) == cudaSuccess;
    // the workspace: the free bitmap, marks and offsets of sequences, page lists, plans of a
    // compaction, partial results of the attention
    size_t at = 0;
    auto room = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const size_t seqs = cfg->max_seqs, cells = seqs * cfg->max_pages, parts = pages_attn_part_rows(p->sms);
    const size_t o_bits = room(((size_t)cfg->n_pages + 127) / 128 * 16), o_mark = room(4 * seqs), o_flags = room(16);
    const size_t zeroed = at;
    const size_t o_off = room(4 * (seqs + 1)), o_fresh = room(4 * (size_t)cfg->n_pages),
                 o_plan = room(4 * PLAN_INTS * seqs), o_old = room(4 * cells), o_rank = room(4 * cells),
                 o_po = room(parts * cfg->head_dim * 4), o_pml = room(parts * 8), o_item = room(32 * 4096);
    void *mapped = nullptr, *host = nullptr, *ws = nullptr;
    bool oom = false;
    if (ok) {
        ok = cudaMalloc(&ws, at) == cudaSuccess;
        oom = !ok;
    }
    p->ws = static_cast<char *>(ws);
    ok = ok && cudaMemset(ws, 0, zeroed) == cudaSuccess && cudaStreamSynchronize(0) == cudaSuccess;
    ok = ok && cudaHostAlloc(&host, 64, cudaHostAllocMapped) == cudaSuccess;
    p->status_host = static_cast<volatile int *>(host);
    ok = ok && cudaHostGetDevicePointer(&mapped, host, 0) == cudaSuccess;
    ok = ok && pages_attn_simt_setup() && pages_attn_tc_setup();
    if (!ok) {
        cudaGetLastError();
        msd_pages_destroy(p);
        return oom ? MSD_ERR_OOM : MSD_ERR_CUDA;
    }
    *p->status_host = 0;
    p->v = PagesView{buf->kv, buf->table, buf->len, buf->refs, reinterpret_cast<unsigned *>(p->ws + o_bits),
                     static_cast<int *>(mapped), reinterpret_cast<int *>(p->ws + o_flags) + 3, cfg->n_layers, cfg->n_heads, cfg->n_kv_heads, cfg->head_dim,
                     cfg->page_size, shift, cfg->n_pages, cfg->max_seqs, cfg->max_pages};
    p->mark = reinterpret_cast<int *>(p->ws + o_mark);
    p->flags = reinterpret_cast<int *>(p->ws + o_flags);
    p->off = reinterpret_cast<int *>(p->ws + o_off);
    p->fresh = reinterpret_cast<int *>(p->ws + o_fresh);
    p->plan = reinterpret_cast<int *>(p->ws + o_plan);
    p->old_table = reinterpret_cast<int *>(p->ws + o_old);
    p->rank = reinterpret_cast<int *>(p->ws + o_rank);
    p->part_o = reinterpret_cast<float *>(p->ws + o_po);
    p->part_ml = reinterpret_cast<float *>(p->ws + o_pml);
    p->part_item = reinterpret_cast<PartItem *>(p->ws + o_item);
    if (cfg->dtype == MSD_BF16 && !pages_attn_map(p->v, &p->map)) {
        msd_pages_destroy(p);
        return MSD_ERR_CUDA;
    }
    *out = p;
    return MSD_OK;
}

msd_status msd_pages_destroy(msd_pages *p) {
    if (!p) return MSD_OK;
    if (p->ws) cudaFree(p->ws);
    if (p->status_host) cudaFreeHost(const_cast<int *>(p->status_host));
    delete p;
    return MSD_OK;
}

const char *msd_pages_last_error(const msd_pages *p) { return p ? p->err : "null pool"; }

msd_status msd_pages_restore(msd_pages *p, void *stream) {
    if (!p) return MSD_ERR_INVALID;
    msd_status st = enter(p, "msd_pages_restore", static_cast<cudaStream_t>(stream));
    if (st != MSD_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int blocks = std::min((p->cfg.n_pages + 255) / 256, 4 * p->sms);
    cudaError_t e = chain(restore_clear_kernel, dim3(blocks), 256, s, p->v);
    if (e == cudaSuccess) e = chain(restore_count_kernel, dim3(p->cfg.max_seqs), 256, s, p->v);
    if (e == cudaSuccess) e = chain(restore_bits_kernel, dim3(blocks), 256, s, p->v);
    return leave(p, e);
}

msd_status msd_pages_reserve(msd_pages *p, const msd_batch *batch, void *stream) {
    if (!p) return MSD_ERR_INVALID;
    msd_status st = enter(p, "msd_pages_reserve", static_cast<cudaStream_t>(stream));
    if (st != MSD_OK) return st;
    BatchView b;
    if (!batch_view(p, batch, &b)) return pfail(p, MSD_ERR_INVALID, "bad batch");
    return leave(p, chain(reserve_kernel, dim3(1), plan_threads(p, b.n), static_cast<cudaStream_t>(stream), p->v, b, p->mark,
                          p->off, p->fresh));
}

msd_status msd_pages_fork(msd_pages *p, int32_t n, const int32_t *src, const int32_t *dst, int32_t deep, void *stream) {
    if (!p) return MSD_ERR_INVALID;
    msd_status st = enter(p, "msd_pages_fork", static_cast<cudaStream_t>(stream));
    if (st != MSD_OK) return st;
    if (n < 1 || n > p->cfg.max_seqs || !src || !dst) return pfail(p, MSD_ERR_INVALID, "bad count or null list");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = chain(fork_plan_kernel, dim3(1), plan_threads(p, n), s, p->v, n, src, dst, deep != 0, p->mark, p->off,
                          p->fresh, p->flags + 2);
    if (e == cudaSuccess) {
        // enough CTAs for every SM's eight, by the heads (and pages) of a copy
        const long base = (long)n * p->cfg.n_layers, want = (8l * p->sms + base - 1) / base;
        const dim3 grid(n, p->cfg.n_layers, (unsigned)std::max(1l, std::min(want, deep ? 64l : 2l * p->cfg.n_kv_heads)));
        e = p->cfg.dtype == MSD_F32
                ? chain(fork_apply_kernel<4>, grid, 256, s, p->v, src, dst, deep != 0, p->off, p->fresh, p->flags + 2)
                : chain(fork_apply_kernel<2>, grid, 256, s, p->v, src, dst, deep != 0, p->off, p->fresh, p->flags + 2);
    }
    return leave(p, e);
}

msd_status msd_pages_compact(msd_pages *p, const msd_batch *batch, const int32_t *keep, int32_t keep_stride,
                             const int32_t *n_keep, void *stream) {
    if (!p) return MSD_ERR_INVALID;
    msd_status st = enter(p, "msd_pages_compact", static_cast<cudaStream_t>(stream));
    if (st != MSD_OK) return st;
    BatchView b;
    if (!batch_view(p, batch, &b) || !n_keep || (keep && keep_stride < 1))
        return pfail(p, MSD_ERR_INVALID, "bad batch, stride or null count");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const CompactArgs c{keep, keep_stride, n_keep, p->mark, p->off, p->fresh, p->plan, p->old_table, p->rank, p->flags};
    cudaError_t e = chain(compact_plan_kernel, dim3(b.n), plan_threads(p, std::max(b.n, keep ? keep_stride / 4 : 0)), s, p->v, b, c);
    if (e == cudaSuccess) {
        const int groups = p->cfg.n_layers * 2 * p->cfg.n_kv_heads;
        const int units = 256 / (p->cfg.head_dim * (p->cfg.dtype == MSD_F32 ? 4 : 2) / 16);
        // Lists of 64 and more side by side: 16 lists of 1027 tokens, 8 layers of 8 heads, with the fork before them, take 100 us,
        // and 227 one by one. Near 64 the two cross, later the more layers there are (room, lists of every other row, cut
        // again; side by side and one by one): 32 layers of 8 heads 80, 63 us at 32 tokens, 100, 96 at 64, 116, 120 at 96;
        // 8 layers of 8 heads 37, 39 at 32, 39, 43 at 64, 51, 64 at 128; 4 layers of 4 heads 25, 31 at 32.
        const int side = keep && keep_stride < 64 ? 1 : std::min(units, 16);
        const dim3 grid((groups + units / side - 1) / (units / side), b.n);        // (sequences are few enough for y, groups need not be)
        e = p->cfg.dtype == MSD_F32 ? chain(compact_apply_kernel<4, 8>, grid, 256, s, p->v, c, groups, side)
                                    : chain(compact_apply_kernel<2, 8>, grid, 256, s, p->v, c, groups, side);
    }
    return leave(p, e);
}

msd_status msd_pages_free(msd_pages *p, int32_t n, const int32_t *seqs, void *stream) {
    if (!p) return MSD_ERR_INVALID;
    msd_status st = enter(p, "msd_pages_free", static_cast<cudaStream_t>(stream));
    if (st != MSD_OK) return st;
    if (n < 1 || n > p->cfg.max_seqs || !seqs) return pfail(p, MSD_ERR_INVALID, "bad count or null list");
    return leave(p, chain(free_kernel, dim3(std::min(n, 8 * p->sms)), 128, static_cast<cudaStream_t>(stream), p->v, n, seqs));
}

msd_status msd_rope_positions(msd_pages *p, const msd_batch *batch, const int32_t *span_start, const int32_t *spans,
                              int32_t n_spans, const int32_t *first, int32_t *pos, int64_t pos_stride, int32_t *next,
                              void *stream) {
    if (!p) return MSD_ERR_INVALID;
    msd_status st = enter(p, "msd_rope_positions", static_cast<cudaStream_t>(stream));
    if (st != MSD_OK) return st;
    BatchView b;
    if (!batch_view(p, batch, &b) || !pos || (span_start && (!spans || n_spans < 0)) || pos_stride < b.rows)
        return pfail(p, MSD_ERR_INVALID, "bad batch, stride or null array");
    // CTAs of a sequence, by an even batch's (16 sequences of 1260 rows 1.5 us warm, one of 20000 among 15 short ones 3.1,
    // among 255 of one row 9.2)
    const int chunks = std::max(1, std::min((b.rows / b.n + SPAN_TILE - 1) / SPAN_TILE, 64));
    return leave(p, chain(positions_kernel, dim3(b.n, chunks), SPAN_TILE, static_cast<cudaStream_t>(stream), p->v, b,
                          span_start, spans, span_start ? n_spans : 0, first, pos, (long)pos_stride, next));
}

msd_status msd_rope_append(msd_pages *p, int32_t layer, const msd_batch *batch, const void *q, int64_t ldq,
                           const void *k, int64_t ldk, const void *v, int64_t ldv, int32_t src_dtype,
                           const int32_t *pos, int64_t pos_stride, void *out, int64_t ldo, void *stream) {
    if (!p) return MSD_ERR_INVALID;
    msd_status st = enter(p, "msd_rope_append", static_cast<cudaStream_t>(stream));
    if (st != MSD_OK) return st;
    BatchView b;
    const msd_pages_config &c = p->cfg;
    if (!batch_view(p, batch, &b) || layer < 0 || layer >= c.n_layers || !q || !k || !v || !out || !pos)
        return pfail(p, MSD_ERR_INVALID, "bad batch, layer or null array");
    if (src_dtype != MSD_F32 && src_dtype != c.dtype) return pfail(p, MSD_ERR_INVALID, "source is neither fp32 nor the cache's type");
    const long hd = c.head_dim;
    if (ldq < c.n_heads * hd || ldo < c.n_heads * hd || ldk < c.n_kv_heads * hd || ldv < c.n_kv_heads * hd ||
        (pos_stride != 0 && pos_stride < b.rows))
        return pfail(p, MSD_ERR_INVALID, "a stride is shorter than its row");
    const size_t se = src_dtype == MSD_F32 ? 4 : 2, de = c.dtype == MSD_F32 ? 4 : 2;
    auto off16 = [](const void *x, int64_t ld, size_t e) { return reinterpret_cast<uintptr_t>(x) % 16 || ld * e % 16; };
    if (off16(q, ldq, se) || off16(k, ldk, se) || off16(v, ldv, se) || off16(out, ldo, de))
        return pfail(p, MSD_ERR_INVALID, "pointers and rows must be 16-byte aligned");
    if (b.rows == 0) return MSD_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const RopeArgs a{q, k, v, (long)ldq, (long)ldk, (long)ldv, pos, (long)pos_stride, out, (long)ldo, layer, c.rot_dim / 2};
    return leave(p, c.dtype == MSD_F32       ? launch_rope<float, float>(p, b, a, s)
                    : src_dtype == MSD_F32 ? launch_rope<float, bf16>(p, b, a, s)
                                           : launch_rope<bf16, bf16>(p, b, a, s));
}

msd_status msd_pages_attention(msd_pages *p, int32_t layer, const msd_batch *batch, const msd_tree *tree,
                               int32_t tree_nodes, int32_t window, int32_t sinks, const void *q, int64_t ldq, void *out,
                               int64_t ldo, float *lse, void *stream) {
    if (!p) return MSD_ERR_INVALID;
    msd_status st = enter(p, "msd_pages_attention", static_cast<cudaStream_t>(stream));
    if (st != MSD_OK) return st;
    BatchView b;
    const msd_pages_config &c = p->cfg;
    if (!batch_view(p, batch, &b) || layer < 0 || layer >= c.n_layers || !q || !out)
        return pfail(p, MSD_ERR_INVALID, "bad batch, layer or null array");
    if (window < 0 || sinks < 0) return pfail(p, MSD_ERR_INVALID, "negative window or sinks");
    if (tree && (!tree->mask || !tree->depth || tree_nodes < 1 || tree_nodes > 1024))
        return pfail(p, MSD_ERR_INVALID, "a tree needs its mask and depths, and 1 to 1024 nodes");
    if ((long)b.rows * (c.n_heads / c.n_kv_heads) >= 1l << 26)
        return pfail(p, MSD_ERR_INVALID, "rows times query heads of a K/V head reach 2^26");
    if (tree && (long)b.rows > (long)b.n * tree_nodes) return pfail(p, MSD_ERR_INVALID, "more rows than tree nodes");
    const long hd = c.head_dim;
    const size_t de = c.dtype == MSD_F32 ? 4 : 2;
    if (ldq < c.n_heads * hd || ldo < c.n_heads * hd) return pfail(p, MSD_ERR_INVALID, "a stride is shorter than its row");
    if (reinterpret_cast<uintptr_t>(q) % 16 || reinterpret_cast<uintptr_t>(out) % 16 || ldq * de % 16 || ldo * de % 16)
        return pfail(p, MSD_ERR_INVALID, "pointers and rows must be 16-byte aligned");
    if (b.rows == 0) return MSD_OK;
    PagesAttn a{};
    a.pv = p->v;
    a.b = b;
    a.layer = layer;
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.ldq = ldq;
    a.ldo = ldo;
    if (tree) {
        a.mask = tree->mask;
        a.depth = tree->depth;
        a.n_nodes = tree->n_nodes;
        a.nodes = tree_nodes;
        a.words = (tree_nodes + 63) / 64;
    }
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.group = c.n_heads / c.n_kv_heads;
    a.packed = (int)(((long)b.rows * a.group + b.n - 1) / b.n);
    a.group_magic = ((1ull << 32) + a.group - 1) / a.group;
    a.scale_log2 = 1.4426950408889634f / std::sqrt((float)hd);
    a.part_o = p->part_o;
    a.part_ml = p->part_ml;
    a.part_item = p->part_item;
    a.wide = reinterpret_cast<uintptr_t>(out) % 32 == 0 && ldo * de % 32 == 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < b.n && e == cudaSuccess; i += ATTN_MAX_SEQS) {
        a.b = BatchView{std::min(b.n - i, ATTN_MAX_SEQS), b.rows, b.seqs + i, b.row_start + i};
        if (tree) {
            a.mask = tree->mask + (long)i * tree_nodes * a.words;
            a.depth = tree->depth + (long)i * tree_nodes;
            a.n_nodes = tree->n_nodes ? tree->n_nodes + i : nullptr;
        }
        e = c.dtype == MSD_BF16 ? launch_pages_attn_tc(p->map, a, p->sms, s) : launch_pages_attn_simt(a, p->sms, s);
    }
    return leave(p, e);
}

}  // extern "C"
