// Device helpers of the token tree: places to cache rows, and the division of attention work among blocks.
#pragma once
#include "dba_device.cuh"
#include "tree_internal.h"

namespace dba {

// place / page_size without a division: for places below 2^31, (place * mul) >> (32 + shift) with the numbers the host works out
__device__ __forceinline__ uint32_t tree_page(const TreePages& pg, uint32_t place) {
    return pg.page_size == 1 ? place : __umulhi(place, pg.page_mul) >> pg.page_shift;
}
// Element offset of a place of sequence b in one layer's cache; -1 where there is no such row (the place is outside the
// table, or the table names a page outside the cache: recorded in the status word).  64 bits: a cache may be longer
// than 2^31 elements.  `wanted()` is asked of a page outside the cache alone: false where nobody needs the place, and nothing is recorded.
template <typename F>
__device__ __forceinline__ int64_t tree_row(const TreePages& pg, int b, int place, F wanted) {
    const unsigned page = tree_page(pg, (unsigned)place);
    if (place < 0 || page >= (unsigned)pg.max_pages) return -1;
    const int32_t id = __ldg(pg.table + (int64_t)b * pg.table_stride + page);
    if ((unsigned)id >= (unsigned)pg.num_pages) {
        if (wanted()) atomicOr(pg.status, (uint32_t)DBA_TREE_BAD_PAGE);
        return -1;
    }
    return (int64_t)id * pg.page_stride + (int64_t)((unsigned)place - page * (unsigned)pg.page_size) * pg.token_stride;
}
__device__ __forceinline__ int64_t tree_row(const TreePages& pg, int b, int place) { return tree_row(pg, b, place, [] { return true; }); }

// Keys of a sequence are walked in tiles of `kt` places: first the arena up to the highest slot in use, then the
// context (each starts a tile of its own).  A sequence with nothing to see has one (empty) tile, so that somebody
// writes its zeros.
__device__ __forceinline__ int tree_top(const TreeAttend& a, int b) {
    if (!a.masks) return 0;
    return a.top ? min(max(__ldg(a.top + b), 0), a.A) : a.A;
}
__device__ __forceinline__ int tree_ctx(const TreeAttend& a, int b) { return min(max(__ldg(a.ctx_len + b), 0), a.ctx_cap); }
__device__ __forceinline__ int tree_tiles(const TreeAttend& a, int b, int kt) {
    return max(1, (tree_top(a, b) + kt - 1) / kt + (tree_ctx(a, b) + kt - 1) / kt);
}

// The work of a call: items (sequence, key head or group of them, block of rows), sequence by sequence, each `extra` units
// for what an item costs beside its tiles and then a unit for each of its tree_tiles() tiles, laid end to end and cut into
// `used` equal runs, one per block.  A run may begin and end inside an item; an item cut by a run's end is finished by
// tree_combine_kernel.
struct TreeRun {
    long long t, t_end, total;         // this block's units
    long long seq_t;                   // first unit of sequence b
    int b, used;
    int item, in_item;                 // where the run stands: item of sequence b (-1: to be worked out), unit of the item
    int top, ctx, len;                 // of sequence b
};
__device__ __forceinline__ long long tree_run_start(int c, long long total, int used) { return (long long)c * total / used; }
__device__ __forceinline__ int tree_run_owner(long long t, long long total, int used) { return (int)(((t + 1) * used - 1) / total); }

struct TreeRunShared { long long sums[33]; long long seq_t; int b; };

// Called by all NT threads of a block; the lengths are scanned by the block itself (B numbers out of the L2), so no
// kernel has to plan ahead and no length comes to the host.  `least`: units a run should have before the work is cut further.
template <int NT>
__device__ TreeRun tree_run(const TreeAttend& a, int kt, int items_per_seq, int extra, int least, TreeRunShared* sh) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (a.B + NT - 1) / NT, b_lo = min(tid * per, a.B), b_hi = min(b_lo + per, a.B);
    long long sum = 0;
    for (int b = b_lo; b < b_hi; ++b) sum += (long long)(tree_tiles(a, b, kt) + extra) * items_per_seq;
    long long pre = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(kFullMask, pre, o);
        if (lane >= o) pre += v;
    }
    if (lane == 31) sh->sums[warp] = pre;
    __syncthreads();
    long long before = 0, total = 0;
    for (int w = 0; w < NT / 32; ++w) {
        if (w < warp) before += sh->sums[w];
        total += sh->sums[w];
    }
    pre += before - sum;                                   // units before this thread's sequences
    TreeRun r;
    r.total = total;
    r.used = (int)min((long long)gridDim.x, max(1LL, total / least));
    r.t = r.t_end = 0;
    if ((int)blockIdx.x < r.used) {
        r.t = tree_run_start(blockIdx.x, total, r.used);
        r.t_end = tree_run_start(blockIdx.x + 1, total, r.used);
        if (r.t >= pre && r.t < pre + sum) {
            int b = b_lo;
            for (;;) {
                const long long len = (long long)(tree_tiles(a, b, kt) + extra) * items_per_seq;
                if (r.t < pre + len) break;
                pre += len; ++b;
            }
            sh->b = b; sh->seq_t = pre;
        }
    }
    __syncthreads();
    r.b = sh->b; r.seq_t = sh->seq_t; r.item = -1;
    return r;
}

// One piece of a run: a stretch of one item's tiles.
struct TreePiece {
    int b, h, rb;                      // sequence, key head (or group of heads), block of rows
    int tile, tiles, item_tiles;       // first tile, how many, of how many
    int arena_tiles, top, ctx;
    int slot;                          // where a partial result goes: 0 the run's first piece, 1 a later (its last) one
    bool whole;                        // the item begins and ends in this piece
};
// (a run's end within an item's extra units leaves the item to the next run; where items stay whole, a run has the items that
// begin in it)
__device__ __forceinline__ bool tree_next_piece(const TreeAttend& a, TreeRun& r, int kt, int groups, int row_blocks, int extra, bool first, TreePiece* p) {
    while (r.t < r.t_end) {
        if (r.item < 0) {              // a new sequence (the first one may be entered anywhere)
            r.top = tree_top(a, r.b); r.ctx = tree_ctx(a, r.b);
            r.len = max(1, (r.top + kt - 1) / kt + (r.ctx + kt - 1) / kt) + extra;
            const long long off = r.t - r.seq_t;
            r.item = off ? (int)(off / r.len) : 0;
            r.in_item = (int)(off - (long long)r.item * r.len);
            if (a.whole_items && r.in_item > 0) {      // (only the run's first item can be one that began before)
                r.t += r.len - r.in_item;
                r.in_item = 0;
                if (++r.item == groups * row_blocks) { r.item = -1; r.seq_t = r.t; ++r.b; }
                continue;
            }
        }
        const int end = a.whole_items ? r.len : (int)min((long long)r.len, (long long)r.in_item + (r.t_end - r.t)), T = r.len - extra;
        p->b = r.b; p->top = r.top; p->ctx = r.ctx;
        p->h = row_blocks == 1 ? r.item : r.item / row_blocks; p->rb = r.item - p->h * row_blocks;
        p->tile = max(0, r.in_item - extra);
        p->tiles = end - extra - p->tile;
        p->item_tiles = T;
        p->arena_tiles = (r.top + kt - 1) / kt;
        p->whole = p->tile == 0 && p->tiles == T;
        p->slot = first ? 0 : 1;
        r.t += end - r.in_item;
        r.in_item = 0;
        if (++r.item == groups * row_blocks) { r.item = -1; r.seq_t = r.t; ++r.b; }
        if (p->tiles > 0) return true;
    }
    return false;
}
// The first key place of a tile and how many places of it exist.
__device__ __forceinline__ void tree_tile_span(const TreeAttend& a, const TreePiece& p, int tile, int kt, int* place, int* count) {
    if (tile < p.arena_tiles) { *place = tile * kt; *count = min(kt, p.top - *place); return; }
    const int c = (tile - p.arena_tiles) * kt;
    *place = a.A + c; *count = max(0, min(kt, p.ctx - c));
}
// What the combining kernel is told: block c (whose run begins inside an item whose first tile is block c - 1's) names the
// item, the last block working on it, and which of block c - 1's two places holds its piece.
__device__ __forceinline__ void tree_write_meta(const TreeAttend& a, const TreeRun& r, const TreePiece* first_piece, int row_blocks, int extra) {
    int4 m = make_int4(-1, 0, 0, 0);
    if (first_piece && first_piece->tile > 0) {
        const TreePiece& p = *first_piece;
        const long long begin = tree_run_start(blockIdx.x, r.total, r.used) - p.tile;      // the unit of its first tile
        if (tree_run_owner(begin, r.total, r.used) == (int)blockIdx.x - 1) {
            const int last = tree_run_owner(begin + p.item_tiles - 1, r.total, r.used);
            const long long prev = tree_run_start((int)blockIdx.x - 1, r.total, r.used);
            m = make_int4(p.b, p.h * row_blocks + p.rb, last, prev >= begin - extra ? 0 : 1);
        }
    }
    a.meta[blockIdx.x] = m;
}

}  // namespace dba
