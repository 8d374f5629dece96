// The tree after a step: masks of the new rows, slots and positions of their tokens, and the list of settled slots.
//
// One block per sequence, everything in shared memory: a row's past is the mask of the old row at the root of its chain
// of parents; OR over the rows gives the slots in use, AND over the open rows the settled ones.  Bound by latency: the
// masks are a few hundred kilobytes at most, read and written once.
// Measured on the device: 256 sequences of 20 rows and 512 slots 6.2 us, one of 5 rows and 64 slots 4.3, of some eight steps
// that wait for one another (blocks of 256 threads; 6.8 with 128).
#include "tree_device.cuh"

namespace dba {

namespace {

constexpr int kVThreads = 256;

struct VSmem {
    int32_t up[kTreeMaxRows];          // earlier row of this call that the row extends, or -1
    int32_t root[kTreeMaxRows];        // old row its chain starts from
    int32_t given[kTreeMaxRows];       // given as open (its chain may still close it)
    int32_t slot[kTreeMaxRows], past[kTreeMaxRows];                // past: tokens of the row's past that hold a slot
    uint64_t chain[kTreeMaxRows];      // earlier rows of this call on the row's path
    uint32_t settled[kTreeMaxWords], used[kTreeMaxWords];
    int32_t free_before[kTreeMaxWords + 1], settled_before[kTreeMaxWords + 1];
    uint64_t open;
    int32_t top;
    // then base[rows][W], and (only where there are settled slots) their slots and positions [32 W] each
};

__global__ void __launch_bounds__(kVThreads) tree_advance_kernel(const TreeAdvance a) {
    extern __shared__ __align__(16) unsigned char raw[];
    VSmem& sm = *reinterpret_cast<VSmem*>(raw);
    uint32_t* base = reinterpret_cast<uint32_t*>(raw + sizeof(VSmem));
    const int W = a.W, n = a.rows_out, A = 32 * W;
    int32_t* list_slot = reinterpret_cast<int32_t*>(base + n * W);
    int32_t* list_pos = list_slot + A;
    const int tid = threadIdx.x, b = blockIdx.x;
    grid_dependency_wait();
    allow_dependents();
    if (tid == 0) { sm.open = 0; sm.top = 0; }
    for (int w = tid; w < W; w += kVThreads) { sm.used[w] = 0u; sm.settled[w] = 0xffffffffu; }
    const int ctx = __ldg(a.ctx_len + b);
    if (tid < n) {
        const int64_t at = (int64_t)b * n + tid;
        const int bp = __ldg(a.backptr + at);
        bool open = bp >= 0 && bp < a.rows_in + tid;               // an old row, or an earlier one of this call
        if (open && a.score) open = __ldg(a.score + at) > neg_inf();
        if (open && a.token) open = __ldg(a.token + at) != a.eos_id;
        sm.given[tid] = open;
        sm.up[tid] = bp >= a.rows_in ? bp - a.rows_in : -1;
        sm.root[tid] = bp;
    }
    __syncthreads();
    if (tid < n) {
        uint64_t chain = 0;
        bool open = sm.given[tid];
        int r = tid;
        while (open && sm.up[r] >= 0) { r = sm.up[r]; chain |= 1ull << r; open = sm.given[r]; }
        const int root = sm.root[r];
        sm.chain[tid] = chain;
        if (open) atomicOr((unsigned long long*)&sm.open, 1ull << tid);
        sm.slot[tid] = root;                                       // (for the moment)
        sm.past[tid] = 0;
    }
    __syncthreads();
    const uint64_t open = sm.open;
    for (int i = tid; i < n * W; i += kVThreads) {
        const int r = i / W, w = i - r * W;
        uint32_t x = 0u;
        if ((open >> r) & 1ull) {
            x = __ldg(a.masks_in + ((int64_t)b * a.rows_in + sm.slot[r]) * W + w);
            if (x) { atomicOr(&sm.used[w], x); atomicAdd(&sm.past[r], __popc(x)); }
            if (~x) atomicAnd(&sm.settled[w], x);
        }
        base[i] = x;
    }
    __syncthreads();
    for (int w = tid; w < W; w += kVThreads) {
        if (!open) sm.settled[w] = 0u;
        sm.free_before[w + 1] = 32 - __popc(sm.used[w]); sm.settled_before[w + 1] = __popc(sm.settled[w]);
    }
    __syncthreads();
    if (tid < 32) {        // prefix sums over at most 128 words: four to a lane
        int f[4], s[4], fs = 0, ss = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int w = 4 * tid + j;
            f[j] = w < W ? sm.free_before[w + 1] : 0; s[j] = w < W ? sm.settled_before[w + 1] : 0;
            fs += f[j]; ss += s[j];
        }
        int fp = fs, sp = ss;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(kFullMask, fp, o), y = __shfl_up_sync(kFullMask, sp, o);
            if (tid >= o) { fp += x; sp += y; }
        }
        fp -= fs; sp -= ss;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int w = 4 * tid + j;
            if (w < W) { sm.free_before[w] = fp; sm.settled_before[w] = sp; }
            fp += f[j]; sp += s[j];
            if (w == W - 1) { sm.free_before[W] = fp; sm.settled_before[W] = sp; }
        }
    }
    __syncthreads();
    int count = sm.settled_before[W];
    const bool fits = ctx >= 0 && count <= a.ctx_cap - ctx;
    if (!fits && count > 0) {
        if (tid == 0) atomicOr(a.status, (uint32_t)DBA_TREE_NO_ROOM);
        count = 0;
    }
    // new slots: the j-th open row takes the j-th lowest free one
    if (tid < n) {
        int slot = -1, pos = -1;
        if ((open >> tid) & 1ull) {
            const int j = __popcll(open & ((1ull << tid) - 1ull));
            if (j < sm.free_before[W]) {
                int w = 0;
                for (int step = 64; step; step >>= 1)              // the last word with at most j free slots before it
                    if (w + step < W && sm.free_before[w + step] <= j) w += step;
                uint32_t z = ~sm.used[w];
                for (int left = j - sm.free_before[w]; left > 0; --left) z &= z - 1u;
                slot = 32 * w + __ffs(z) - 1;
            } else atomicOr(a.status, (uint32_t)DBA_TREE_ARENA_FULL);
            pos = ctx + sm.past[tid] + __popcll(sm.chain[tid]);
            if (slot >= 0) a.slot_pos[(int64_t)b * a.slot_pos_stride + slot] = pos;
        }
        sm.slot[tid] = slot;
        const int64_t at = (int64_t)b * n + tid;
        if (a.next.slot) a.next.slot[at] = slot;
        if (a.next.position) a.next.position[at] = pos;
    }
    if (count > 0)         // (a thread per slot: the loads of the positions do not wait for one another)
#pragma unroll 4
        for (int i = tid; i < A; i += kVThreads) {
            const uint32_t x = sm.settled[i >> 5], bit = 1u << (i & 31);
            if (x & bit) {
                const int at = sm.settled_before[i >> 5] + __popc(x & (bit - 1u));
                list_slot[at] = i; list_pos[at] = a.slot_pos[(int64_t)b * a.slot_pos_stride + i];
            }
        }
    __syncthreads();
    // masks: the past without what has settled, the row's chain in this call, its own token
    int top = 0;
    for (int i = tid; i < n * W; i += kVThreads) {
        const int r = i / W, w = i - r * W;
        uint32_t x = base[i];
        if (count > 0) x &= ~sm.settled[w];
        if ((open >> r) & 1ull)
            for (uint64_t ch = sm.chain[r] | 1ull << r; ch; ch &= ch - 1ull) {
                const int s = sm.slot[__ffsll((long long)ch) - 1];
                if (s >= 0 && (s >> 5) == w) x |= 1u << (s & 31);
            }
        a.next.masks[(int64_t)b * n * W + i] = (int32_t)x;
        if (x) top = max(top, 32 * w + 32 - __clz(x));
    }
    if (top) atomicMax(&sm.top, top);
    // settled slots by position (then slot): each counts the ones before it
    if (a.next.commit_src) {
        int32_t* out = a.next.commit_src + (int64_t)b * A;
        for (int i = tid; i < A; i += kVThreads) {
            if (i >= count) { out[i] = -1; continue; }
            int before = 0;
            const int p = list_pos[i];
            for (int j = 0; j < count; ++j) before += list_pos[j] < p || (list_pos[j] == p && j < i);
            out[before] = list_slot[i];
        }
    }
    __syncthreads();
    if (tid == 0) {
        if (a.next.ctx_len) a.next.ctx_len[b] = ctx + count;
        if (a.next.commit_n) a.next.commit_n[b] = count;
        if (a.next.top) a.next.top[b] = sm.top;
    }
}

size_t advance_smem(int n, int W) { return sizeof(VSmem) + (size_t)n * W * 4 + (size_t)32 * W * 8; }

}  // namespace

cudaError_t configure_tree_advance() {
    return cudaFuncSetAttribute(tree_advance_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)advance_smem(kTreeMaxRows, kTreeMaxWords));
}

cudaError_t launch_tree_advance(const TreeAdvance& a, cudaStream_t st, int* launches) {
    *launches += 1;
    return launch_after(tree_advance_kernel, dim3(a.B), dim3(kVThreads), advance_smem(a.rows_out, a.W), st, a);
}

}  // namespace dba
