// The weight that context tokens receive from attention on the tensor cores: bf16, head sizes up to 128.
//
//     w'[p] = decay w[p] + sum over rows and heads of 2^(scale log2(e) <k_p, q> - lse log2(e))
//
// Keys are the matrix instruction's rows: S = K Q^T, 128 keys by up to 128 queries, so that a key is a lane of tensor memory, a thread has a key,
// and its sum over the queries stays in a register: no sum crosses threads, and none depends on the order of anything.
//   keys' threads  two warpgroups, every other tile each, with up to two blocks of 128 queries at a time
//   products       one lane of a warp issues
//   loaders        tiles of 128 keys by tensor-map boxes where pages are made of eights, else by 16-byte cp.async; queries by cp.async, those of closed
//                  rows as zeros.  More than 256 queries: the keys go by again for each 256, and their sums are added to what has been written.
// The tiles of all (sequence, key head)s are cut into equal runs, one to a block.  Every wait on an mbarrier is bounded: one that runs out winds
// the block down, leaves NaN in the places of its run and is reported.
//
// Measured: four documents of up to 131071 tokens, one row each (530 MB): 88 us, 6.0 TB/s, 92 % of the rate of a copy: HBM.  Beams of 20 on 16
// prompts of up to 4100 tokens, 32 heads over 8 of 128 (110 MB): 29 us, of which some 8 are the start (a context of one token takes 7) and the rest HBM's rate.
#include <cuda_bf16.h>

#include "tree_boxes.cuh"
#include "tree_span.cuh"

namespace dba {

namespace {

constexpr int kYKeys = 128, kYQueries = 128, kYSeen = 16;
constexpr uint32_t kYNoRow = 0xffffffffu;

template <int DP, bool TMA> struct YConf {
    static constexpr int load_warps = TMA ? 2 : 4, threads = 32 * (9 + load_warps);
    static constexpr int q_warps = TMA ? 1 : load_warps;       // of them, those that load queries
    static constexpr int tile_bytes = kYKeys * DP * 2, q_bytes = kYQueries * DP * 2;
    static constexpr int stages = DP == 128 ? 4 : 8;
};
template <int DP, bool TMA> struct YSmem {
    using C = YConf<DP, TMA>;
    alignas(1024) unsigned char q[2][C::q_bytes];
    unsigned char k[C::stages][C::tile_bytes];
    float lse[2][kYQueries];                    // in powers of two, taken off; -inf: the query counts nothing
    uint64_t full[C::stages], empty[C::stages];
    uint64_t s_full[2][2], s_free[2][2];        // by warpgroup and block of queries
    uint64_t q_full[2], q_empty[2], last;
    uint32_t seen[kYSeen][4];
    uint32_t tmem_base;
    int abort_flag;
    union {
        SpanShared span;
        alignas(16) uint32_t rows[kYKeys];      // a tile's rows in the cache, in 16 bytes; kYNoRow: none
    };
};

// A stretch of the tiles of a (sequence, key head), and 256 of its queries.
struct YPiece { int b, h, len, tile, tile_end, group, blocks; };
struct YRun {
    SpanRun r;
    YPiece p;
    __device__ __forceinline__ int tiles_of(const TreeWeigh& a, int b) { return (int)((min(max(__ldg(a.ctx_len + b), 0), a.ctx_cap) + kYKeys - 1u) / kYKeys); }
    __device__ __forceinline__ void start(const SpanRun& run) { r = run; p.group = -1; p.tile_end = 0; }
    __device__ __forceinline__ bool next(const TreeWeigh& a) {
        const int M = a.n * a.G, groups = (M + 2 * kYQueries - 1) / (2 * kYQueries);
        if (p.group < 0 || p.group + 1 == groups) {
            if (r.t >= r.t_end) return false;
            int tiles = tiles_of(a, r.g);
            while (r.t - r.at >= (long long)a.K * tiles) { r.at += (long long)a.K * tiles; tiles = tiles_of(a, ++r.g); }
            p.b = r.g;
            p.h = (int)((r.t - r.at) / tiles);
            p.tile = (int)((r.t - r.at) - (long long)p.h * tiles);
            p.tile_end = (int)min((long long)tiles, p.tile + (r.t_end - r.t));
            p.len = min(max(__ldg(a.ctx_len + r.g), 0), a.ctx_cap);
            r.t += p.tile_end - p.tile;
            p.group = 0;
        } else ++p.group;
        p.blocks = min(2, (M - p.group * 2 * kYQueries + kYQueries - 1) / kYQueries);
        return true;
    }
};

template <int DP, bool TMA>
__global__ void __launch_bounds__(YConf<DP, TMA>::threads, 1) tree_weigh_mma_kernel(const __grid_constant__ TreeWeigh a, const __grid_constant__ TreeBoxes maps) {
    using C = YConf<DP, TMA>;
    extern __shared__ __align__(1024) unsigned char yraw[];
    YSmem<DP, TMA>& sm = *reinterpret_cast<YSmem<DP, TMA>*>(yraw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, M = a.n * a.G;
    volatile int* abort_flag = &sm.abort_flag;
    const long long limit = a.wait_clocks > 0 ? a.wait_clocks : kMWaitClocks;
    if (tid == 0) {
        for (int s = 0; s < C::stages; ++s) { mbar_init(msmem_u32(&sm.full[s]), TMA ? 1 : 33 * C::load_warps); mbar_init(msmem_u32(&sm.empty[s]), 1); }
        for (int i = 0; i < 2; ++i) {
            // (s_full: the products, and an arrival of the issuing thread, which passes on what the loaders wrote before it)
            for (int c = 0; c < 2; ++c) { mbar_init(msmem_u32(&sm.s_full[i][c]), 2); mbar_init(msmem_u32(&sm.s_free[i][c]), 4); }
            mbar_init(msmem_u32(&sm.q_full[i]), 64 * C::q_warps); mbar_init(msmem_u32(&sm.q_empty[i]), 9);
        }
        mbar_init(msmem_u32(&sm.last), 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(msmem_u32(&sm.tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    grid_dependency_wait();
    allow_dependents();
    YRun run;
    run.start(span_run<C::threads>(a.B, 1, &sm.span, [&](int b) { return (long long)a.K * run.tiles_of(a, b); }));      // (has the block's barriers)
    const SpanRun mine = run.r;
    __syncthreads();           // its numbers have been read: their place is used again
    tc_after();
    const uint32_t tmem = sm.tmem_base;
    const YPiece& pc = run.p;
    uint32_t tiles0 = 0, q_use = 0;                        // tiles and blocks of queries before this piece
    if (warp > 8) {
        // ------------------------------------------------------------------ loaders (as those of the prefix kernel)
        constexpr int CH = DP / 8, RW = 32 / CH, NJ = 32 / RW;         // 16-byte chunks of a row, rows a warp copies at a time, and how often
        const int lw = warp - 9, ch = lane % CH, sub = lane / CH, q_warp = TMA ? lw - 1 : lw;
        const bool ch_in = ch * 8 < a.D;
        const uint32_t q_at = msmem_u32(sm.q), k_at = msmem_u32(sm.k);
        const uint32_t swz = (uint32_t)((ch & 7) ^ sub) << 4;          // the swizzle moves a chunk by its row's last three bits
        const uint32_t page16 = (uint32_t)(a.pages.page_stride / 8), token16 = (uint32_t)(a.pages.token_stride / 8);
        const int box_lane = TMA ? min(lane, kYKeys / maps.rows - 1) * maps.rows : lw * 32 + lane;       // the lane's (first) place in a tile
        uint32_t* const rows = sm.rows + lw * 32;
        uint32_t copy = 0;
        bool ok = true;
        if (TMA && lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k) : "memory");
        while (ok && run.next(a)) {
            const int32_t* const table = a.pages.table + (int64_t)pc.b * a.pages.table_stride;
            int32_t id = 0;
            const auto fetch = [&](int t) {                // page numbers are fetched a tile ahead and not looked at before their turn
                const int p = t * kYKeys + box_lane;
                id = p < pc.len ? __ldg(table + tree_page(a.pages, (uint32_t)(a.A + p))) : -1;       // (below the table's entries: the length is)
            };
            if (!TMA || lw == 0) fetch(pc.tile);
            for (int c = 0; q_warp >= 0 && c < pc.blocks; ++c) {
                const uint32_t use = q_use + c, qb = use & 1u;
                if (use >= 2 && !mbar_wait(msmem_u32(&sm.q_empty[qb]), (use / 2 - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                const char* q = (const char*)a.q + (ch_in ? ch * 16 : 0);
                const int row0 = pc.group * 2 * kYQueries + c * kYQueries;
#pragma unroll 1
                for (int r0 = q_warp * 32; r0 < kYQueries; r0 += 32 * C::q_warps) {
                    int64_t q_row = -1;
                    float lse = neg_inf();
                    if (row0 + r0 + lane < M) {
                        const int rr = row0 + r0 + lane, tok = rr / a.G, head = pc.h * a.G + rr - tok * a.G;
                        lse = a.lse[((int64_t)pc.b * a.n + tok) * a.H + head];
                        if (lse != neg_inf()) {            // (else the query may hold anything)
                            q_row = 2 * ((int64_t)pc.b * a.q_seq + (int64_t)tok * a.q_row + (int64_t)head * a.q_head);
                            lse = -lse * 1.4426950408889634f;
                        }
                    }
                    sm.lse[qb][r0 + lane] = lse;
                    const uint32_t to = q_at + qb * C::q_bytes + (uint32_t)(ch >> 3) * (kYQueries * 128) + (uint32_t)(r0 + sub) * 128;
#pragma unroll 1
                    for (int j0 = 0; j0 < 32; j0 += 8 * RW) {
                        int64_t from[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) from[j] = __shfl_sync(kFullMask, q_row, j0 + j * RW + sub);
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            cp_async16(to + (j0 + j * RW) * 128 + (swz ^ (uint32_t)((j * RW & 7) << 4)), from[j] >= 0 ? q + from[j] : q, from[j] >= 0 && ch_in ? 16u : 0u);
                    }
                }
                mbar_arrive(msmem_u32(&sm.q_full[qb]));    // (for the log-sum-exps)
                cp_arrive(msmem_u32(&sm.q_full[qb]));
            }
            if (!ok) break;
            const char* const from = (const char*)a.k + 2 * (int64_t)pc.h * a.pages.head_stride + (ch_in ? ch * 16 : 0);
#pragma unroll 1
            for (int t = pc.tile; t < (TMA && lw > 0 ? 0 : pc.tile_end); ++t, ++copy) {
                const int p = t * kYKeys + box_lane;
                const uint32_t place = (uint32_t)(a.A + p), in_page = place - tree_page(a.pages, place) * (uint32_t)a.pages.page_size;
                const bool there = (uint32_t)id < (uint32_t)a.pages.num_pages;
                if (!there && p < pc.len) atomicOr(a.pages.status, (uint32_t)DBA_TREE_BAD_PAGE);
                const uint32_t stage = copy % C::stages, use = copy / C::stages, full = msmem_u32(&sm.full[stage]);
                uint32_t* const seen_at = sm.seen[(tiles0 + t - pc.tile) % kYSeen];
                if (TMA) {
                    const int page = there ? id : a.pages.num_pages;   // (a page that there is not: zeros)
                    boxes_seen(seen_at, maps.rows, box_lane, there, pc.len - t * kYKeys);
                    __syncwarp();
                    if (t + 1 < pc.tile_end) fetch(t + 1);
                    if (use > 0 && !mbar_wait(msmem_u32(&sm.empty[stage]), (use - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                    if (lane == 0) mbar_expect(full, C::tile_bytes);
                    __syncwarp();
                    if ((int)copy != a.drop_item && lane * maps.rows < kYKeys) {
#pragma unroll
                        for (int c = 0; c < DP / 64; ++c)
                            copy_box(k_at + stage * C::tile_bytes + c * (kYKeys * 128) + box_lane * 128, &maps.k, 64 * c, (int)in_page, page, pc.h, full);
                    }
                } else {
                    const uint32_t at = there ? (uint32_t)id * page16 + in_page * token16 : kYNoRow, seen = __ballot_sync(kFullMask, there);     // (the host has seen to it that 32 bits are enough)
                    __syncwarp();                          // the last tile's rows have been read
                    rows[(lane % RW) * NJ + lane / RW] = at;           // a lane will copy rows sub, sub + RW, ..: its numbers lie side by side
                    if (lane == 0) seen_at[lw] = seen;
                    __syncwarp();
                    if (t + 1 < pc.tile_end) fetch(t + 1);
                    uint32_t row[NJ];                      // (read before the copies: they are not reordered)
#pragma unroll
                    for (int j = 0; j < NJ; j += 4) {
                        const uint4 r4 = *reinterpret_cast<const uint4*>(rows + sub * NJ + j);
                        row[j] = r4.x; row[j + 1] = r4.y; row[j + 2] = r4.z; row[j + 3] = r4.w;
                    }
                    if (use > 0 && !mbar_wait(msmem_u32(&sm.empty[stage]), (use - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                    const uint32_t to = k_at + stage * C::tile_bytes + (uint32_t)(ch >> 3) * (kYKeys * 128) + (uint32_t)(lw * 32 + sub) * 128;
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const bool in = row[j] != kYNoRow && ch_in;
                        cp_async16(to + j * RW * 128 + (swz ^ (uint32_t)((j * RW & 7) << 4)), from + (uint64_t)(in ? row[j] : 0u) * 16, in ? 16u : 0u);
                    }
                    if (lane == 0) mbar_arrive(full);
                    if ((int)copy != a.drop_item) cp_arrive(full);
                }
            }
            tiles0 += pc.tile_end - pc.tile;
            q_use += pc.blocks;
        }
        // nothing of this block is in flight when it leaves (where nobody gave up, all boxes have been waited for)
        cp_wait_all();
        if (TMA && lw == 0 && *abort_flag)
            for (uint32_t c = copy > C::stages ? copy - C::stages : 0; c < copy; ++c)
                for (int i = 0; i < 100000 && (int)c != a.drop_item && !__all_sync(kFullMask, mbar_try(msmem_u32(&sm.full[c % C::stages]), (c / C::stages) & 1u)); ++i) {}
    } else if (warp == 8) {
        // ------------------------------------------------------------------ products: the warp walks in step, one lane issues
        const int steps16 = (a.D + 15) / 16;
        const uint64_t k_desc = sw128_desc(msmem_u32(sm.k), 16), q_desc = sw128_desc(msmem_u32(sm.q), 16);
        uint32_t used[2][2] = {{0, 0}, {0, 0}};            // how often each S has been written
        bool ok = true;
        while (ok && run.next(a)) {
#pragma unroll 1
            for (int t = pc.tile; t < pc.tile_end && ok; ++t) {
                const uint32_t copy = tiles0 + t - pc.tile, stage = copy % C::stages, wg = (uint32_t)(t - pc.tile + pc.h) & 1u;
                if (!(ok = mbar_wait(msmem_u32(&sm.full[stage]), (copy / C::stages) & 1u, abort_flag, limit))) break;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (c >= pc.blocks) break;
                    const uint32_t use = q_use + c, qb = use & 1u, times = wg ? used[1][c] : used[0][c];
                    if (t == pc.tile && !(ok = mbar_wait(msmem_u32(&sm.q_full[qb]), (use / 2) & 1u, abort_flag, limit))) break;
                    if (times > 0 && !(ok = mbar_wait(msmem_u32(&sm.s_free[wg][c]), (times - 1) & 1u, abort_flag, limit))) break;
                    const int queries = min(kYQueries, M - (pc.group * 2 + c) * kYQueries);
                    const uint32_t idesc = mma_idesc((queries + 15) / 16 * 16, false), d = tmem + (wg * 2 + c) * kYQueries;
                    const uint64_t dk = k_desc + (uint64_t)(stage * (C::tile_bytes / 16)), dq = q_desc + (uint64_t)(qb * (C::q_bytes / 16));
                    if (elect_one()) {
                        if (!TMA || t == pc.tile) fence_async_proxy();         // the copies' writes (generic) before the products' reads
                        tc_after();
#pragma unroll
                        for (int ks = 0; ks < DP / 16; ++ks)       // 16 dimensions = 32 bytes along a swizzled row; 64 to a block of columns
                            if (ks < steps16)
                                mma_ss(d, dk + (uint64_t)((ks >> 2) * (kYKeys * 128 / 16) + (ks & 3) * 2), dq + (uint64_t)((ks >> 2) * (kYQueries * 128 / 16) + (ks & 3) * 2), idesc, ks != 0, -1);
                        mma_commit(msmem_u32(&sm.s_full[wg][c]));
                        mbar_arrive(msmem_u32(&sm.s_full[wg][c]));
                        if (c + 1 == pc.blocks) mma_commit(msmem_u32(&sm.empty[stage]));
                        if (t + 1 == pc.tile_end) mma_commit(msmem_u32(&sm.q_empty[qb]));
                    }
                    __syncwarp();
                    if (wg) ++used[1][c]; else ++used[0][c];
                }
            }
            tiles0 += pc.tile_end - pc.tile;
            q_use += pc.blocks;
        }
        // nothing of this block is in flight when it leaves, whatever happened
        if (elect_one()) mma_commit(msmem_u32(&sm.last));
        for (int i = 0; i < 1000000 && !__all_sync(kFullMask, mbar_try(msmem_u32(&sm.last), 0)); ++i) {}
    } else {
        // ------------------------------------------------------------------ a key to a thread
        const uint32_t wg = warp >> 2, key = tid & 127, lanes = (uint32_t)((warp & 3) * 32) << 16;
        uint32_t used[2] = {0, 0};
        bool ok = true;
        while (ok && run.next(a)) {
            for (int t = pc.tile + (int)((wg ^ (uint32_t)pc.h) & 1u); t < pc.tile_end && ok; t += 2) {          // (the same for all of a key's queries)
                const int p = t * kYKeys + (int)key;
                const int64_t at = (int64_t)pc.b * a.w_seq + (int64_t)pc.h * a.w_head + p;
                const bool in = p < pc.len;
                // (what this thread has written for the queries before these)
                const float before = !in ? 0.f : pc.group > 0 ? a.out[at] : a.in ? a.decay * a.in[at] : 0.f;
                float s = 0.f;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (c >= pc.blocks) break;
                    if (!mbar_wait(msmem_u32(&sm.s_full[wg][c]), used[c] & 1u, abort_flag, limit)) { ok = false; break; }
                    ++used[c];
                    tc_after();
                    const float4* z = reinterpret_cast<const float4*>(sm.lse[(q_use + c) & 1u]);
                    const int queries = min(kYQueries, M - (pc.group * 2 + c) * kYQueries);
                    float t0 = 0.f, t1 = 0.f, t2 = 0.f, t3 = 0.f;
#pragma unroll 1
                    for (int j0 = 0; j0 < queries; j0 += 16) {
                        uint32_t x[16];
                        tm_ld16(tmem + lanes + (wg * 2 + c) * kYQueries + j0, x);
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const float4 zz = z[(j0 + j) / 4];
                            t0 += ex2(fmaf(__uint_as_float(x[j]), a.scale_log2e, zz.x));
                            t1 += ex2(fmaf(__uint_as_float(x[j + 1]), a.scale_log2e, zz.y));
                            t2 += ex2(fmaf(__uint_as_float(x[j + 2]), a.scale_log2e, zz.z));
                            t3 += ex2(fmaf(__uint_as_float(x[j + 3]), a.scale_log2e, zz.w));
                        }
                    }
                    float sum = (t0 + t1) + (t2 + t3);
                    // Queries that count nothing are zeros, and zero times a key that is not finite is not: once more, without them.  (Looking each of them
                    // over costs a beam of 20 on 16 sentences 3 of 32 us.)
                    if (__any_sync(kFullMask, sum != sum)) {
                        sum = 0.f;
#pragma unroll 1
                        for (int j0 = 0; j0 < queries; j0 += 16) {
                            uint32_t x[16];
                            tm_ld16(tmem + lanes + (wg * 2 + c) * kYQueries + j0, x);
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                const float zz = sm.lse[(q_use + c) & 1u][j0 + j];
                                if (zz != neg_inf()) sum += ex2(fmaf(__uint_as_float(x[j]), a.scale_log2e, zz));
                            }
                        }
                    }
                    s += sum;
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(msmem_u32(&sm.s_free[wg][c]));
                }
                if (!ok) break;
                const uint32_t seen = sm.seen[(tiles0 + t - pc.tile) % kYSeen][key >> 5];
                if (in) a.out[at] = before + ((seen >> (key & 31)) & 1u ? s : 0.f);
            }
            if (!ok) break;
            __syncwarp();
            for (int c = 0; c < pc.blocks; ++c) {          // (a warpgroup without a tile here must not be ahead by a phase)
                const uint32_t use = q_use + c;
                if (use >= 2 && !mbar_wait(msmem_u32(&sm.q_empty[use & 1u]), (use / 2 - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                if (lane == 0) mbar_arrive(msmem_u32(&sm.q_empty[use & 1u]));
            }
            if (!ok) break;
            tiles0 += pc.tile_end - pc.tile;
            q_use += pc.blocks;
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    if (sm.abort_flag) {                                   // nothing that this block wrote can be trusted
        if (tid == 0) atomicOr(a.pages.status, (uint32_t)DBA_TREE_TIMEOUT);
        run.start(mine);
        while (run.next(a))
            for (uint32_t p = pc.tile * kYKeys + tid; p < min((uint32_t)pc.tile_end * kYKeys, (uint32_t)pc.len); p += C::threads)
                a.out[(int64_t)pc.b * a.w_seq + (int64_t)pc.h * a.w_head + p] = __int_as_float(0x7fc00000);
    }
}

template <int DP, bool TMA>
cudaError_t configure_weigh_mma() {
    static_assert(sizeof(YSmem<DP, TMA>) <= 227 * 1024, "a block's shared memory");
    return cudaFuncSetAttribute(tree_weigh_mma_kernel<DP, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(YSmem<DP, TMA>));
}
template <int DP, bool TMA>
cudaError_t launch_weigh_mma(const TreeWeigh& a, const TreeBoxes& m, int grid, cudaStream_t st) {
    return launch_after(tree_weigh_mma_kernel<DP, TMA>, dim3(grid), dim3(YConf<DP, TMA>::threads), sizeof(YSmem<DP, TMA>), st, a, m);
}

}  // namespace

cudaError_t configure_tree_weigh_mma() {
    cudaError_t e = configure_weigh_mma<64, true>();
    if (e == cudaSuccess) e = configure_weigh_mma<128, true>();
    if (e == cudaSuccess) e = configure_weigh_mma<64, false>();
    return e == cudaSuccess ? configure_weigh_mma<128, false>() : e;
}
cudaError_t launch_tree_weigh_mma(const TreeWeigh& a, int grid, cudaStream_t st) {
    TreeBoxes m{};
    if (tree_boxes(&m, a.k, nullptr, a.pages, a.K, a.D, a.A))
        return a.D <= 64 ? launch_weigh_mma<64, true>(a, m, grid, st) : launch_weigh_mma<128, true>(a, m, grid, st);
    return a.D <= 64 ? launch_weigh_mma<64, false>(a, m, grid, st) : launch_weigh_mma<128, false>(a, m, grid, st);
}

}  // namespace dba
