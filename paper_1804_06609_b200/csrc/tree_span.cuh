// Division of work whose amount only the device knows: groups (prefixes, sequences) of so many units each, laid end to end and cut into
// equal contiguous runs, one per block; and the pieces of a prefix' attention that fall into a run.
#pragma once
#include "tree_device.cuh"

namespace dba {

struct SpanRun {
    long long t, t_end, at;            // this block's units; the first unit of group g
    long long t2, t2_end;              // and units behind those, when they are done
    int g, used;                       // group the run stands in; blocks that have a run
};
struct SpanShared { long long sums[33]; long long at; int g; };

// Called by all NT threads of a block: units(g) >= 0 of `groups` groups are scanned by the block itself (numbers out of the L2).
// `least`: units a run should have before the work is cut further.
template <int NT, typename F>
__device__ SpanRun span_run(int groups, int least, SpanShared* sh, F units) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (groups + NT - 1) / NT, lo = min(tid * per, groups), hi = min(lo + per, groups);
    long long sum = 0;
    for (int g = lo; g < hi; ++g) sum += units(g);
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
    pre += before - sum;
    SpanRun r;
    r.used = (int)min((long long)gridDim.x, max(1LL, total / least));
    r.t = r.t_end = r.t2 = r.t2_end = 0;
    if ((int)blockIdx.x < r.used && total > 0) {
        r.t = (long long)blockIdx.x * total / r.used;
        r.t_end = (long long)(blockIdx.x + 1) * total / r.used;
        if (r.t >= pre && r.t < pre + sum) {
            int g = lo;
            for (;;) {
                const long long n = units(g);
                if (r.t < pre + n) break;
                pre += n; ++g;
            }
            sh->g = g; sh->at = pre;
        }
    }
    __syncthreads();
    r.g = sh->g; r.at = sh->at;
    return r;
}

// One prefix as a kernel sees it: what is out of range is brought into it, and reported by tree_prefix_check.
struct PrefixGroup { int lo, hi, len; };
__device__ __forceinline__ PrefixGroup prefix_group(const TreePrefix& a, int g) {
    PrefixGroup p;
    p.lo = min(max(__ldg(a.first + g), 0), a.B);
    p.hi = min(max(__ldg(a.first + g + 1), p.lo), a.B);
    p.len = min(max(__ldg(a.len + g), 0), a.cap);
    return p;
}
__device__ __forceinline__ void prefix_check(const TreePrefix& a) {
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
        const int lo = __ldg(a.first + g), hi = __ldg(a.first + g + 1), len = __ldg(a.len + g);
        if (lo < 0 || hi < lo || hi > a.B || len < 0 || len > a.cap) atomicOr(a.pages.status, (uint32_t)DBA_TREE_BAD_INDEX);
    }
}

// The rows of a prefix' sequences and one key head, in blocks of ROWS; an item is one of these blocks, of `tiles` tiles of KT
// keys.  A tile costs 2 units, 1 in a block of at most HALF rows (HALF = 0: 1 always), an item kExtra beside them.
template <int KT, int ROWS, int HALF> struct PrefixCut {
    static constexpr int kExtra = 2;
    struct Sizes { int rows, blocks, tiles; long long full, rest, head; };      // units of a full block, of the last one, of a key head
    static __device__ __forceinline__ int cost(int rows) { return HALF > 0 && rows > HALF ? 2 : 1; }
    static __device__ __forceinline__ Sizes sizes(const TreePrefix& a, const PrefixGroup& p) {
        Sizes s;
        s.rows = (p.hi - p.lo) * a.n * a.G;
        s.tiles = (int)((p.len + KT - 1u) / KT);           // (a length may be as large as an int is)
        s.blocks = (s.rows + ROWS - 1) / ROWS;
        if (s.tiles == 0 || s.blocks == 0) { s.full = s.rest = s.head = 0; return s; }
        s.full = (long long)cost(ROWS) * s.tiles + kExtra;
        s.rest = (long long)cost(s.rows - (s.blocks - 1) * ROWS) * s.tiles + kExtra;
        s.head = (s.blocks - 1) * s.full + s.rest;
        return s;
    }
    static __device__ __forceinline__ long long units(const TreePrefix& a, int g) { return a.K * sizes(a, prefix_group(a, g)).head; }

    // The run of this block (called by all NT threads).  One prefix whose items are alike, the usual case, needs no scan; as many whole items as come out
    // even go to each block, and only what is left of them is cut: an item cut costs its outputs' way through memory and the joining kernel (a beam of 20
    // on 64 sentences, 32 heads over 8 of 128, 6007 tokens: 157 us, all items in one line 172).
    template <int NT>
    static __device__ __forceinline__ SpanRun run(const TreePrefix& a, int least, SpanShared* sh) {
        if (a.groups > 1) return span_run<NT>(a.groups, least, sh, [&](int g) { return units(a, g); });
        const Sizes s = sizes(a, prefix_group(a, 0));
        const long long total = a.K * s.head, items = s.full > 0 && s.rest == s.full ? total / s.full : 0, each = items / gridDim.x, left = total - each * gridDim.x * s.full;
        SpanRun r;
        r.g = 0; r.at = 0;
        r.t = blockIdx.x * each * s.full;
        r.t_end = r.t + each * s.full;
        r.used = (int)min((long long)gridDim.x, max(1LL, left / least));
        r.t2 = r.t2_end = total;
        if ((int)blockIdx.x < r.used) {
            r.t2 = total - left + blockIdx.x * left / r.used;
            r.t2_end = total - left + (blockIdx.x + 1) * left / r.used;
        }
        return r;
    }

    struct Piece {
        int g, h, rb;                  // prefix, key head, block of rows
        int lo, len;                   // the prefix' first sequence, its tokens
        int row0, rows;                // the item's rows
        int tile, tile_end, tiles;     // of the item's tiles
        __device__ __forceinline__ bool whole() const { return tile == 0 && tile_end == tiles; }
    };
    static __device__ __forceinline__ bool next(const TreePrefix& a, SpanRun& r, Piece* p) {
        for (;;) {
            if (r.t >= r.t_end) {
                if (r.t2 >= r.t2_end) return false;
                r.t = r.t2; r.t_end = r.t2_end; r.t2 = r.t2_end;
                continue;
            }
            const PrefixGroup pg = prefix_group(a, r.g);
            const Sizes s = sizes(a, pg);
            if (r.t - r.at >= a.K * s.head) { r.at += a.K * s.head; ++r.g; continue; }
            long long off = r.t - r.at;
            const int h = (int)(off / s.head);
            off -= h * s.head;
            const int rb = (int)min((long long)(s.blocks - 1), off / s.full);
            const long long in_item = off - rb * s.full, all = rb == s.blocks - 1 ? s.rest : s.full;
            const long long end = min(all, in_item + (r.t_end - r.t));
            p->g = r.g; p->h = h; p->rb = rb; p->lo = pg.lo; p->len = pg.len;
            p->row0 = rb * ROWS; p->rows = min(ROWS, s.rows - p->row0);
            const int c = cost(p->rows);
            // (a run's end inside a tile's units leaves the tile to the run that has its first one)
            p->tile = in_item <= kExtra ? 0 : (int)((in_item - kExtra + c - 1) / c);
            p->tile_end = end <= kExtra ? 0 : (int)((end - kExtra + c - 1) / c);
            p->tiles = s.tiles;
            r.t += end - in_item;
            if (p->tile_end > p->tile) return true;
        }
    }
};

// Sequence, row and head of an item's row.
struct PrefixRow { int b, i, head; };
__device__ __forceinline__ PrefixRow prefix_row(const TreePrefix& a, int lo, int h, int row) {
    const int seq = row / (a.n * a.G), in = row - seq * (a.n * a.G), i = in / a.G;
    return {lo + seq, i, h * a.G + in - i * a.G};
}

// What a row's own part says of it: its log-sum-exp in powers of two (-inf: nothing seen of its own); whether the row is open.
__device__ __forceinline__ float prefix_own_lse(const TreePrefix& a, const PrefixRow& r) {
    return a.own_lse[((int64_t)r.b * a.n + r.i) * a.H + r.head] * 1.4426950408889634f;
}
__device__ __forceinline__ bool prefix_open(const TreePrefix& a, const PrefixRow& r, float own) {
    if (own != neg_inf() || !a.masks) return true;
    uint32_t any = 0;
    const uint32_t* m = a.masks + ((int64_t)r.b * a.n + r.i) * a.W;
    for (int w = 0; w < a.W; ++w) any |= __ldg(m + w);
    return any != 0;
}
__device__ __forceinline__ bool prefix_own(const TreePrefix& a, const PrefixRow& r, float* own) {
    *own = prefix_own_lse(a, r);
    return prefix_open(a, r, *own);
}

// A row's whole from its own part (log-sum-exp in powers of two `own`, output o) and the prefix' (reference m, sum l, products O):
// w_own o + w_pre O.  False: nothing is seen of the prefix, the own part stands.
__device__ __forceinline__ bool prefix_join(float own, float m, float l, float* w_own, float* w_pre, float* lse) {
    if (l == 0.f) return false;
    const float top = fmaxf(own, m), e0 = exp2f(own - top), e1 = exp2f(m - top), den = fmaf(l, e1, e0), inv = 1.f / den;
    *w_own = e0 * inv; *w_pre = e1 * inv;
    *lse = (top + log2f(den)) * 0.6931471805599453f;
    return true;
}

}  // namespace dba
