// The paged cache: what its operators share on the host and on the device.
#pragma once

#include <algorithm>
#include <cuda.h>
#include <cudaTypedefs.h>

#include "common.cuh"
#include "msd.h"

namespace msd {

// Device status codes of the paged cache (after common.cuh's).
enum : int {
    ST_NO_PAGES = 5,      // fewer free pages than a call needed: the call changed nothing
    ST_BAD_BATCH = 6,     // sequence ids, row counts or lists that the call cannot take
    ST_REFUSED = 0x100,   // with one of the others: a page operation was not carried out
};

constexpr int MAX_ROT_PAIRS = 64;

// Turns per position of each rotated pair as a 64-bit fraction (base^(-2i/rot) / 2 pi,
// scaled by 2^64), and the axis (0 time, 1 height, 2 width) that the pair turns by.
struct RopeTable {
    unsigned long long turn[MAX_ROT_PAIRS];
    unsigned char axis[MAX_ROT_PAIRS];
};

struct PagesView {
    void *kv;                 // [layers][n_pages][2][kv_heads][page][head_dim]
    int *table;               // [max_seqs][max_pages]
    int *len, *refs;
    unsigned *bits;           // bit p % 32 of word p / 32: page p is free
    int *status;
    int *refused;             // not 0: the code of a page operation that was not carried out, which the host has not reported
    int layers, heads, kv_heads, head_dim, page, page_shift;
    int n_pages, max_seqs, max_pages;
    __host__ __device__ long page_elems() const { return 2l * kv_heads * page * head_dim; }
};

// A page operation that cannot be carried out (one thread calls it, before anything has changed). The calls queued
// behind it, recorded ones too, were made for what it should have done, so they do nothing: the mark goes, in the
// stream's order, with the call that reports this very error (the status word may hold another that came before it).
__device__ __forceinline__ void refuse(const PagesView &v, int code) {
    set_status(v.status, code | ST_REFUSED);
    *v.refused = code | ST_REFUSED;
}

// the rows of a call (msd_batch)
struct BatchView {
    int n, rows;
    const int *seqs, *row_start;
};

__device__ __forceinline__ int pages_of(int tokens, int shift, int page) { return (tokens + page - 1) >> shift; }

// The sequence of a row: the last i with row_start[i] <= row, found by the whole warp, 32
// boundaries a step (one step up to 32 sequences, two up to 1024).
__device__ __forceinline__ int row_owner(const int *row_start, int n, int row) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n;                       // row_start[lo] <= row; row_start[hi] > row or hi == n
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) >> 5;
        const int at = lo + lane * step;
        const bool below = at < hi && row_start[at] <= row;
        const int c = __popc(__ballot_sync(0xffffffffu, below));
        const int nlo = lo + (c > 0 ? c - 1 : 0) * step;
        hi = min(hi, nlo + step);
        lo = nlo;
    }
    return lo;
}

// An item whose partial results are to be joined: first row, K/V head, first packed row, packed rows, first CTA.
struct PartItem {
    int start, h, m0, rows, cta;
};

// Attention over the pages (pages_attn_*.cu).
struct PagesAttn {
    PagesView pv;
    BatchView b;
    int layer;
    const void *q;            // [rows][ldq]: head j of a row at j * head_dim
    void *out;
    float *lse;               // [rows][heads] or null
    long ldq, ldo;
    const uint64_t *mask;     // [n][nodes][words], null: each row sees the rows before it and itself
    const int *depth;         // [n][nodes]
    const int *n_nodes;       // [n] or null
    int nodes, words;
    int window, sinks;        // window 0: none
    float scale_log2;         // log2(e) / sqrt(head_dim)
    int group;                // query heads of a K/V head
    int packed;               // packed rows of a sequence, the mean of the whole call (which may take several launches)
    unsigned long long group_magic;        // ceil(2^32 / group): see group_div
    // partial results of row tiles that several CTAs share
    float *part_o, *part_ml;
    PartItem *part_item;
    bool wide;                // out and its rows are 32-byte aligned
};

// x / group for x < 2^26 (the product is off by x * group at most, below 2^32)
__device__ __forceinline__ int group_div(const PagesAttn &a, int x) {
    return (int)((unsigned)x * a.group_magic >> 32);
}

constexpr int ATTN_MAX_SEQS = 512;         // sequences of one launch
size_t pages_attn_part_rows(int sms);      // rows of partial results that a launch may leave

bool pages_attn_simt_setup();
bool pages_attn_tc_setup();
bool pages_attn_map(const PagesView &v, CUtensorMap *map);
cudaError_t launch_pages_attn_tc(const CUtensorMap &map, const PagesAttn &a, int sms, cudaStream_t s);
cudaError_t launch_pages_attn_join(const PagesAttn &a, int dtype, int ctas, int tile_rows, cudaStream_t s);
cudaError_t launch_pages_attn_simt(const PagesAttn &a, int sms, cudaStream_t s);

}  // namespace msd

struct msd_pages {
    msd::PagesView v;
    msd_pages_config cfg;
    CUtensorMap map;                   // bf16 pools
    msd::RopeTable rope;
    int dev, sms;
    volatile int *status_host;         // page-locked, written by the kernels
    char *ws;                          // one allocation: what follows
    int *mark, *flags, *off, *fresh, *plan, *old_table, *rank;
    float *part_o, *part_ml;
    msd::PartItem *part_item;
    char err[200];
};
