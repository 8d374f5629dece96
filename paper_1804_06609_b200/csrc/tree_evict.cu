// Eviction of context tokens by the weight they have received: which ones stay, and their keys and values to the front.
//
// For every (layer, sequence, key head) with L > keep tokens: the last `recent` of them and, of the others, the m = keep - recent of the
// largest weight.  Weights become whole numbers in the same order (ord32; NaN: 0); the m-th largest is found by its digits, the
// highest first, from histograms in shared memory, until at most 128 are in question, which are ranked among one another; a last pass counts,
// and then keeps, what is above it and the first ones at it, in order, a stretch of the row to a warp.  Everything is decided by counts, so equal inputs give equal results.
//
// Copies: row i of what is kept comes from place kept[i] >= i.  Other pages: any order.  The same pages: rows in ascending order, each
// batch read whole before it is written, by one block, since a row is written only where every later row's source lies behind it.  Arena slots whose
// page is another one in the new table go there too: nobody else writes or reads there.
//
// Measured: a quarter of four documents of up to 32768 tokens, four layers, 8 heads of 128: 220 us, the choice 33 (128 rows, a block each, of up to 130 KB
// of weights: the passes one after the other; 45 with the last one all over the row between barriers and the first digits counted after the load),
// the copies 183 to 188, 1.07 GB, 5.8 TB/s: HBM.  In place 286: 256 blocks of copies, a barrier for every 32 KB.  256 of some 300 tokens, one layer of four
// sequences: 8.8 us, in place 8.4: launches and dependent loads.
#include "tree_device.cuh"

namespace dba {

namespace {

constexpr int kEBins = 2048, kEShared = 48 * 1024, kEFew = 128;      // kEShared: weights of a row that shared memory takes
constexpr int kMThreads = 256, kMRowsAt = 256, kMCopies = 8;

// larger weight, larger number; NaN is less than any
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0u : ord32(w); }

// A block per (layer, sequence, key head), the last counting fastest.  A row of up to `room` weights is read once, into shared memory; a longer one by every pass.
template <int NT>
__global__ void __launch_bounds__(NT) tree_keep_kernel(const TreeEvict a, int room) {
    constexpr int warps = NT / 32;
    extern __shared__ float held[];
    __shared__ uint32_t bins[kEBins];
    __shared__ int sums[2][warps], digit, above_digit, n_few;
    __shared__ uint32_t few[kEFew], few_bar;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int h = (int)(blockIdx.x % a.K), b = (int)(blockIdx.x / a.K % a.B), l = (int)(blockIdx.x / a.K / a.B);
    grid_dependency_wait();
    allow_dependents();
    const int L = min(max(__ldg(a.ctx_len + b), 0), a.ctx_cap), keep = a.e.keep, n = min(L, keep);
    const int64_t row = (int64_t)l * a.e.layer_stride + (int64_t)b * a.e.seq_stride + (int64_t)h * a.e.head_stride;
    const float* w = a.e.weight + row;
    float* out = a.e.weight_out + row;
    int32_t* kept = a.e.kept + (((int64_t)l * a.B + b) * a.K + h) * keep;
    // (unsigned: lengths may be as large as an int is, and a step goes beyond)
    for (unsigned i = (unsigned)n + tid; i < (unsigned)keep; i += NT) kept[i] = -1;
    if (L <= keep) {
        for (unsigned i = tid; i < (unsigned)L; i += NT) {
            kept[i] = (int)i;
            out[i] = w[i];
        }
        return;
    }
    const int old = L - min(a.e.recent, keep);               // places that have to earn it
    int m = keep - (L - old);                              // how many of them stay: less than there are
    uint32_t bar = 0xffffffffu;
    // Counts a digit (of all lanes that are `in`).  A warp counts those with its first one's digit together: rows whose weights are alike, or nothing, would
    // wait for one another's additions.
    const auto count = [&](bool in, uint32_t mine) {
        const uint32_t who = __ballot_sync(kFullMask, in);
        if (who == 0) return;
        const int leader = __ffs(who) - 1;
        const uint32_t leaders = __shfl_sync(kFullMask, mine, leader);       // (by all lanes)
        const bool same = in && mine == leaders;
        const uint32_t together = __ballot_sync(kFullMask, same);
        if (lane == leader) atomicAdd(&bins[mine], (uint32_t)__popc(together));
        else if (in && !same) atomicAdd(&bins[mine], 1u);
    };
    const bool fits = L <= room;
    if (fits) {                                            // with the first digits counted on the way
        for (int i = tid; i < kEBins; i += NT) bins[i] = 0;
        __syncthreads();
#pragma unroll 1
        for (int i0 = 0; i0 < L; i0 += 8 * NT) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = i0 + j * NT + tid < L ? w[i0 + j * NT + tid] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = i0 + j * NT + tid;
                if (i0 + j * NT >= L) break;
                if (i < L) held[i] = x[j];
                count(i < old, weight_key(x[j]) >> 21);
            }
        }
        w = held;
    }
    if (m > 0) {
        uint32_t prefix = 0;                               // the digits found, and how many of those with them stay
        int shift = 32;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = pass == 2 ? 10 : 11;
            const uint32_t known = shift == 32 ? 0u : ~0u << shift;
            shift -= bits;
            if (pass > 0 || !fits) {
                for (int i = tid; i < kEBins; i += NT) bins[i] = 0;
                __syncthreads();
#pragma unroll 4
                for (unsigned i0 = 0; i0 < (unsigned)old; i0 += NT) {
                    const unsigned i = i0 + tid;
                    const uint32_t key = i < (unsigned)old ? weight_key(w[i]) : 0u;
                    count(i < (unsigned)old && (key & known) == prefix, (key >> shift) & ((1u << bits) - 1u));
                }
            }
            __syncthreads();
            // from the largest digit down: thread tid has bins per tid .. per tid + per - 1, counted from the top
            constexpr int per = kEBins / NT;
            const int top = kEBins - 1 - per * tid;
            int c[per], sum = 0;
#pragma unroll
            for (int i = 0; i < per; ++i) { c[i] = (int)bins[top - i]; sum += c[i]; }
            int pre = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(kFullMask, pre, o);
                if (lane >= o) pre += v;
            }
            if (lane == 31) sums[0][warp] = pre;
            __syncthreads();
            int before = pre - sum + __reduce_add_sync(kFullMask, lane < warp ? sums[0][lane] : 0);
#pragma unroll
            for (int i = 0; i < per; ++i) {
                if (before < m && before + c[i] >= m) { digit = top - i; above_digit = before; }
                before += c[i];
            }
            if (tid == 0) n_few = 0;
            __syncthreads();
            prefix |= (uint32_t)digit << shift;
            m -= above_digit;                              // of those with this digit, m stay
            const int left = (int)bins[digit];
            if (pass < 2 && left <= kEFew) {               // few have it: ranked among one another
                const uint32_t same = ~0u << shift;
                for (unsigned i = tid; i < (unsigned)old; i += NT) {
                    const uint32_t key = weight_key(w[i]);
                    if ((key & same) == prefix) few[atomicAdd(&n_few, 1)] = key;         // (in any order: only their number and size count)
                }
                __syncthreads();
                if (tid < left) {
                    const uint32_t key = few[tid];
                    int greater = 0, equal = 0;
                    for (int i = 0; i < left; ++i) { greater += few[i] > key; equal += few[i] == key; }
                    if (greater < m && greater + equal >= m) { few_bar = key; above_digit = greater; }
                }
                __syncthreads();
                prefix = few_bar;
                m -= above_digit;
                break;
            }
            __syncthreads();
        }
        bar = prefix;
    }
    // Those above the bar stay, and m of those at it, the first ones; then the last tokens.  As many places at a time as shared memory holds, a stretch of
    // them to a warp, which first counts what stays of it.  (Where weights go over themselves, what is written lies in front of what has not been read.)
    const bool none = bar == 0xffffffffu, nan_at = bar == 0u;           // (NaN is less than any)
    const float at_least = none ? __int_as_float(0x7fc00000) : nan_at ? neg_inf() : unord32(bar), more = none ? at_least : nan_at ? neg_inf() : unord32(bar + 1u);
    int n_above = 0, n_at = 0;
#pragma unroll 1
    for (unsigned at = 0; at < (unsigned)L; at += room) {
        const int at0 = (int)at, here = min(room, L - at0), choose = min(max(old - at0, 0), here);
        const int stretch = (choose + 32 * warps - 1) / (32 * warps) * 32, lo = warp * stretch, hi = min(lo + stretch, choose);
        __syncthreads();                                   // (the last ones have been written, the counts read)
        if (!fits) {
#pragma unroll 8
            for (int i = tid; i < here; i += NT) held[i] = w[at0 + i];
            __syncthreads();
        }
        int cu = 0, ce = 0;
#pragma unroll 4
        for (int i = lo + lane; i < hi; i += 32) {
            const float x = held[i];
            const bool above = x >= more;
            cu += above;
            ce += !above && (x >= at_least || nan_at);
        }
        cu = __reduce_add_sync(kFullMask, cu); ce = __reduce_add_sync(kFullMask, ce);
        if (lane == 0) { sums[0][warp] = cu; sums[1][warp] = ce; }
        __syncthreads();
        // the warps' counts: lane j has warp j's
        const int all_u = lane < warps ? sums[0][lane] : 0, all_e = lane < warps ? sums[1][lane] : 0;
        int before_u = n_above + __reduce_add_sync(kFullMask, lane < warp ? all_u : 0), before_e = n_at + __reduce_add_sync(kFullMask, lane < warp ? all_e : 0);
        n_above += __reduce_add_sync(kFullMask, all_u); n_at += __reduce_add_sync(kFullMask, all_e);
        const uint32_t below = (1u << lane) - 1u;
#pragma unroll 2
        for (int i0 = lo; i0 < hi; i0 += 32) {
            const int i = i0 + lane;
            const float x = i < hi ? held[i] : 0.f;
            const bool above = i < hi && x >= more, at_bar = i < hi && !above && (x >= at_least || nan_at);
            const uint32_t u = __ballot_sync(kFullMask, above), e = __ballot_sync(kFullMask, at_bar);
            const int mine_e = before_e + __popc(e & below);
            if (above || (at_bar && mine_e < m)) {
                const int to = before_u + __popc(u & below) + min(mine_e, m);
                kept[to] = at0 + i;
                out[to] = x;
            }
            before_u += __popc(u); before_e += __popc(e);
        }
        for (int i = choose + tid; i < here; i += NT) {    // (what is before them: all that stays of the others)
            const int to = keep - L + at0 + i;
            const float x = held[i];
            kept[to] = at0 + i;
            out[to] = x;
        }
    }
    for (unsigned i = (unsigned)n + tid; i < (unsigned)L; i += NT) out[i] = 0.f;
}

// Blocks: keys or values, layer, sequence, key head, split, the last counting fastest.
__global__ void __launch_bounds__(kMThreads) tree_move_kernel(const TreeEvict a, int splits) {
    __shared__ int64_t from_at[kMRowsAt], to_at[kMRowsAt];
    const int tid = threadIdx.x, split = (int)(blockIdx.x % splits);
    unsigned at = blockIdx.x / splits;
    const int h = (int)(at % a.K);
    at /= a.K;
    const int b = (int)(at % a.B);
    at /= a.B;
    const int l = (int)(at % a.layers);
    const bool values = at >= (unsigned)a.layers;
    grid_dependency_wait();
    allow_dependents();
    const int keep = a.e.keep;
    if (split == 0 && h == 0 && l == 0 && !values) {
        const int L = min(max(a.ctx_len[b], 0), a.ctx_cap), dropped = L - min(L, keep);
        if (a.e.slot_pos && dropped > 0)
            for (int i = tid; i < a.A; i += kMThreads) a.e.slot_pos[(int64_t)b * a.e.slot_pos_stride + i] -= dropped;
        __syncthreads();                                   // (ctx_len_out may be ctx_len)
        if (tid == 0) {
            if (a.e.dropped) a.e.dropped[b] = dropped;
            if (a.e.ctx_len_out) a.e.ctx_len_out[b] = min(L, keep);
        }
    }
    // context pages that stay the same: one block, in order; arena pages that do not
    const unsigned first_page = tree_page(a.from, (unsigned)a.A), pages = tree_page(a.from, (unsigned)(a.A + min(keep, a.ctx_cap) - 1)) + 1;
    const unsigned arena_pages = a.A ? tree_page(a.from, (unsigned)(a.A - 1)) + 1 : 0;
    bool same = false, moved = false;
    for (unsigned i = (a.A ? 0 : first_page) + tid; i < pages; i += kMThreads) {
        const bool alike = __ldg(a.to.table + (int64_t)b * a.to.table_stride + i) == __ldg(a.from.table + (int64_t)b * a.from.table_stride + i);
        same = same || (alike && i >= first_page);
        moved = moved || (!alike && i < arena_pages);
    }
    same = __syncthreads_or(same);
    if (a.A) moved = __syncthreads_or(moved);
    if (same && split > 0) return;
    const int chunks = a.D * a.es / 16;
    const int32_t* kept = a.e.kept + (((int64_t)l * a.B + b) * a.K + h) * keep;
    char* base = (values ? a.v : a.k) + l * a.layer_bytes + (int64_t)h * a.from.head_stride * a.es;
    const int step = same ? kMRowsAt : kMRowsAt * splits;
    // `rows` of them from from_at (-1: none) to to_at
    const auto copy = [&](int rows) {
        const int units = rows * chunks;
        for (int u0 = 0; u0 < units; u0 += kMCopies * kMThreads) {
            uint4 x[kMCopies];
            char* to[kMCopies];
#pragma unroll
            for (int c = 0; c < kMCopies; ++c) {
                const int u = u0 + tid + c * kMThreads;
                to[c] = nullptr;
                if (u < units) {
                    const int i = u / chunks, ch = u - i * chunks;
                    if (from_at[i] >= 0) {
                        x[c] = *reinterpret_cast<const uint4*>(base + from_at[i] + ch * 16);
                        to[c] = base + to_at[i] + ch * 16;
                    }
                }
            }
            if (same) __syncthreads();                     // the batch has been read
#pragma unroll
            for (int c = 0; c < kMCopies; ++c)
                if (to[c]) *reinterpret_cast<uint4*>(to[c]) = x[c];
        }
    };
    for (unsigned at0 = split * kMRowsAt; at0 < (unsigned)keep; at0 += step) {
        const int i0 = (int)at0, rows = min(kMRowsAt, keep - i0);
        __syncthreads();
        bool any = false;
        if (tid < rows) {
            const int src = __ldg(kept + i0 + tid);
            int64_t r0 = -1, r1 = -1;
            if (src >= 0) {
                r0 = tree_row(a.from, b, a.A + src);
                r1 = tree_row(a.to, b, a.A + i0 + tid);
                any = true;
            }
            const bool skip = r0 < 0 || r1 < 0 || r0 == r1;
            from_at[tid] = skip ? -1 : r0 * a.es; to_at[tid] = r1 * a.es;
        }
        if (!__syncthreads_or(any)) break;                 // (what is kept is at the front)
        copy(rows);
    }
    if (!moved) return;
    for (int i0 = split * kMRowsAt; i0 < a.A; i0 += step) {
        const int rows = min(kMRowsAt, a.A - i0);
        __syncthreads();
        if (tid < rows) {
            const auto quiet = [] { return false; };       // (whether a slot is in use is not known here)
            const int64_t r0 = tree_row(a.from, b, i0 + tid, quiet), r1 = tree_row(a.to, b, i0 + tid, quiet);
            const bool skip = r0 < 0 || r1 < 0 || r0 == r1;
            from_at[tid] = skip ? -1 : r0 * a.es; to_at[tid] = r1 * a.es;
        }
        __syncthreads();
        copy(rows);
    }
}

}  // namespace

cudaError_t configure_tree_evict() {
    return cudaFuncSetAttribute(tree_keep_kernel<1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, kEShared * (int)sizeof(float));
}

cudaError_t launch_tree_evict(const TreeEvict& a, cudaStream_t st, int* launches) {
    // (by the most tokens that a table holds: the lengths are on the device)
    const unsigned rows_keep = (unsigned)(a.K * a.B * a.layers);
    const int room = a.ctx_cap < kEShared ? a.ctx_cap : kEShared;
    const size_t bytes = (size_t)room * sizeof(float);
    // Both kernels, 512 rows of 1000 places: 26 us with 512 threads, 30 with 256, 31 with 1024; 256 rows of 4000 22 with 1024, 25 with 512
    cudaError_t e = a.ctx_cap <= 2048 ? launch_after(tree_keep_kernel<512>, dim3(rows_keep), dim3(512), bytes, st, a, room)
                                      : launch_after(tree_keep_kernel<1024>, dim3(rows_keep), dim3(1024), bytes, st, a, room);
    *launches += 1;
    if (e != cudaSuccess) return e;
    // some eight blocks an SM, none without a batch of rows
    const int64_t rows = (int64_t)a.K * a.B * a.layers * 2;
    const int most = (int)((a.e.keep + kMRowsAt - 1u) / kMRowsAt), want = (int)((8LL * a.sm_count + rows - 1) / rows), splits = want < most ? want : most;
    e = launch_after(tree_move_kernel, dim3((unsigned)(rows * splits)), dim3(kMThreads), 0, st, a, splits);
    *launches += 1;
    return e;
}

}  // namespace dba
