// Attention over prefixes that sequences share on the tensor cores: bf16, head sizes up to 128.
//
// The rows of all sequences of a prefix and all query heads of a key head are one matrix Q [rows, D], the prefix the other:
//     S = Q K^T,   P = 2^(scale log2(e) S - m),   O += P V,   l += sum P,
// in items of 256 rows (see tree_span.cuh).  One block an SM, two streams of 128 rows that take turns: while one stream's scores go
// through the softmax the tensor cores have the other's products.  An item of at most 128 rows gives both streams the same rows and
// every other tile of keys, and their two results are added in the end.
//   softmax    two warpgroups, one to a stream, a thread to a row.  Scores come out of tensor memory, P goes back over them (bf16, as the
//              matrix instruction needs it: half a unit in the 8th bit of each; the sum is taken before the rounding).  The reference m
//              is raised only when a tile's maximum lies more than 2^8 above it, and O rescaled in tensor memory then.
//   products   one lane of a warp issues, in this order: S0 S1 | O0 S2 | O1 S3 | ..; a stream's next scores come behind its outputs, so
//              their completion shows that of the outputs before, and P may lie over S.
//   loaders    three warps: 16-byte cp.async with zero fill, every place looked up in the page table by itself, so pages of any size
//              may end inside a tile; keys K-major, values MN-major, both [key][d] in the 128-byte swizzle.
// The epilogue joins a whole item with the rows' own part and writes the result; pieces of an item go to scratch, and to the joining
// kernel (tree_prefix.cu).  Every wait on an mbarrier is bounded: one that runs out winds the block down and marks the call as failed.
#include <cuda_bf16.h>

#include "tree_mma.cuh"
#include "tree_span.cuh"

namespace dba {

namespace {

constexpr int kXKeys = 128, kXRows = 256, kXThreads = 384, kXLoadWarps = 3, kXLoadThreads = 32 * kXLoadWarps;
constexpr int kXSeen = 8;              // more than the tiles the loaders may be ahead by
constexpr int kXWarpRows = 44;         // rows of a tile that a loader copies: 44, 44, 40

template <int DP> struct XConf {
    static constexpr int tile_bytes = kXKeys * DP * 2, q_half = 128 * DP * 2, q_bytes = 2 * q_half;
    static constexpr int stages = DP == 128 ? 4 : 8, q_bufs = DP == 128 ? 1 : 2;
    static constexpr int s_col = 0, o_col = 256, tmem_cols = 512;
};
template <int DP> struct XSmem {
    using C = XConf<DP>;
    alignas(1024) unsigned char q[C::q_bufs][C::q_bytes];
    unsigned char kv[C::stages][C::tile_bytes];
    float4 turn[8][32][8];                      // by softmax warp: 32 columns of its rows, on their way to memory
    uint64_t full[C::stages], empty[C::stages];
    uint64_t s_full[2], p_ready[2][2], half_done[2], o_done[2];
    uint64_t q_full[C::q_bufs], q_empty[C::q_bufs];
    uint64_t o_free, ml_ready, last;
    float ml[2][128][2];
    uint32_t seen[kXSeen][kXLoadWarps][2];      // (by tile, in turn) which rows of a loader's there are
    uint32_t tmem_base;
    int abort_flag;
    union {
        SpanShared span;                        // (until the roles begin)
        uint32_t rows[kXLoadWarps * kXWarpRows];       // a tile's rows in the cache, in 16 bytes; kXNoRow: none
    };
};
constexpr uint32_t kXNoRow = 0xffffffffu;
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
using XCut = PrefixCut<kXKeys, kXRows, 128>;

template <int DP>
__global__ void __launch_bounds__(kXThreads, 1) tree_prefix_mma_kernel(const __grid_constant__ TreePrefix a, const uint32_t negate) {
    using C = XConf<DP>;
    extern __shared__ __align__(1024) unsigned char xraw[];
    XSmem<DP>& sm = *reinterpret_cast<XSmem<DP>*>(xraw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile int* abort_flag = &sm.abort_flag;
    const long long limit = a.wait_clocks > 0 ? a.wait_clocks : kMWaitClocks;
    if (tid == 0) {
        for (int s = 0; s < C::stages; ++s) { mbar_init(msmem_u32(&sm.full[s]), kXLoadThreads + kXLoadWarps); mbar_init(msmem_u32(&sm.empty[s]), 1); }
        // (s_full: the products, and an arrival of the issuing thread, which passes on what the loaders wrote before it)
        for (int s = 0; s < 2; ++s) { mbar_init(msmem_u32(&sm.s_full[s]), 2); mbar_init(msmem_u32(&sm.p_ready[s][0]), 4); mbar_init(msmem_u32(&sm.p_ready[s][1]), 4);
                                      mbar_init(msmem_u32(&sm.half_done[s]), 1); mbar_init(msmem_u32(&sm.o_done[s]), 1); }
        for (int i = 0; i < C::q_bufs; ++i) { mbar_init(msmem_u32(&sm.q_full[i]), kXLoadThreads); mbar_init(msmem_u32(&sm.q_empty[i]), 1); }
        mbar_init(msmem_u32(&sm.o_free), 8);
        mbar_init(msmem_u32(&sm.ml_ready), 8); mbar_init(msmem_u32(&sm.last), 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(msmem_u32(&sm.tmem_base)), "r"(C::tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    // Nothing but the rows' own part comes from the kernel before this one, and that kernel has waited for what came before it: the wait
    // is the epilogue's.
    allow_dependents();
    if (blockIdx.x == 0) prefix_check(a);
    SpanRun run = span_run<kXThreads>(a.groups, 3, &sm.span, [&](int g) { return XCut::units(a, g); });      // (has the block's barriers)
    __syncthreads();           // its numbers have been read: their place is used again
    tc_after();
    const uint32_t tmem = sm.tmem_base;
    XCut::Piece pc;
    int piece = 0;
    uint32_t tiles0 = 0;                                   // tiles before this piece
    if (warp > 8) {
        // ------------------------------------------------------------------ loaders
        constexpr int CH = DP / 8, RW = 32 / CH;           // 16-byte chunks of a row, rows a warp copies at a time
        const int lw = warp - 9, ch = lane % CH, sub = lane / CH, base = lw * kXWarpRows, mine = lw < 2 ? kXWarpRows : kXKeys - 2 * kXWarpRows;
        const bool ch_in = ch * 8 < a.D;
        const int64_t page16 = a.pages.page_stride / 8, token16 = a.pages.token_stride / 8;
        const uint32_t q_at = msmem_u32(sm.q), kv_at = msmem_u32(sm.kv) + (uint32_t)(ch >> 3) * (kXKeys * 128) + (uint32_t)(base + sub) * 128;
        // the swizzle moves a chunk by its row's last three bits (of the queries' rows, and of a tile's: base is 0 or 4 of 8)
        const uint32_t swz = (uint32_t)((ch & 7) ^ sub) << 4, kv_swz = swz ^ (uint32_t)((base & 7) << 4);
        uint32_t* const rows = sm.rows + base;
        uint32_t copy = 0;
        int cut = 0;
        int4 meta[2] = {make_int4(-1, 0, 0, 0), make_int4(-1, 0, 0, 0)};
        bool ok = true;
        while (ok && XCut::next(a, run, &pc)) {
            if (!pc.whole()) { if (cut == 0) meta[0] = make_int4(pc.g, pc.h, pc.rb, 0); else meta[1] = make_int4(pc.g, pc.h, pc.rb, 0); ++cut; }
            const uint32_t qb = (uint32_t)piece % C::q_bufs;
            if (piece >= C::q_bufs && !mbar_wait(msmem_u32(&sm.q_empty[qb]), ((uint32_t)piece / C::q_bufs - 1) & 1u, abort_flag, limit)) { ok = false; break; }
            // where a tile's rows are, looked up one tile ahead
            const int64_t head_at = 2 * (int64_t)pc.h * a.pages.head_stride + (ch_in ? ch * 16 : 0);
            uint32_t at[2];
            auto look_up = [&](int t) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = lane + 32 * i, place = t * kXKeys + base + r;
                    at[i] = kXNoRow;
                    if (r < mine && place < pc.len && t < pc.tile_end) {
                        const uint32_t page = tree_page(a.pages, (uint32_t)place);       // (below the table's entries: len is)
                        const int32_t id = __ldg(a.pages.table + (int64_t)pc.g * a.pages.table_stride + page);
                        if ((uint32_t)id < (uint32_t)a.pages.num_pages)
                            at[i] = (uint32_t)((int64_t)id * page16 + (int64_t)((uint32_t)place - page * (uint32_t)a.pages.page_size) * token16);
                        else atomicOr(a.pages.status, (uint32_t)DBA_TREE_BAD_PAGE);
                    }
                }
            };
            look_up(pc.tile);
            // queries, zeros beyond the rows and the head size
            const char* q = (const char*)a.q + (ch_in ? ch * 16 : 0);
#pragma unroll 1
            for (int r0 = lw * 32; r0 < (pc.rows > 128 ? kXRows : 128); r0 += 32 * kXLoadWarps) {        // a lane finds one row, and every lane copies chunks of all
                int64_t q_row = -1;
                if (r0 + lane < pc.rows) {
                    const PrefixRow w = prefix_row(a, pc.lo, pc.h, pc.row0 + r0 + lane);
                    q_row = 2 * ((int64_t)w.b * a.q_seq + (int64_t)w.i * a.q_row + (int64_t)w.head * a.q_head);
                }
                const uint32_t to = q_at + qb * C::q_bytes + (r0 >= 128 ? C::q_half : 0) + (uint32_t)(ch >> 3) * (128 * 128) + (uint32_t)((r0 & 127) + sub) * 128;
#pragma unroll 1
                for (int j0 = 0; j0 < 32; j0 += 8 * RW) {
                    int64_t from[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) from[j] = j0 + j * RW < 32 ? __shfl_sync(kFullMask, q_row, j0 + j * RW + sub) : -1;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j0 + j * RW < 32)
                            cp_async16(to + (j0 + j * RW) * 128 + (swz ^ (uint32_t)((j * RW & 7) << 4)), from[j] >= 0 ? q + from[j] : q, from[j] >= 0 && ch_in ? 16u : 0u);
                }
            }
            cp_arrive(msmem_u32(&sm.q_full[qb]));
#pragma unroll 1
            for (int t = pc.tile; t < pc.tile_end; ++t) {
                const uint32_t seen0 = __ballot_sync(kFullMask, at[0] != kXNoRow), seen1 = __ballot_sync(kFullMask, at[1] != kXNoRow);
                __syncwarp();                              // the last tile's rows have been read
                rows[lane] = at[0];
                if (lane + 32 < mine) rows[lane + 32] = at[1];
                if (lane < 2) sm.seen[(tiles0 + t - pc.tile) % kXSeen][lw][lane] = lane ? seen1 : seen0;
                __syncwarp();
                look_up(t + 1);
                constexpr int NJ = kXWarpRows / RW;
                uint32_t row[NJ];                          // (read before the copies: they are not reordered)
#pragma unroll
                for (int j = 0; j < NJ; ++j) row[j] = rows[j * RW + sub];
#pragma unroll 1
                for (int k = 0; k < 2; ++k, ++copy) {
                    const uint32_t stage = copy % C::stages, use = copy / C::stages;
                    if (use > 0 && !mbar_wait(msmem_u32(&sm.empty[stage]), (use - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                    const char* from = (const char*)(k ? a.v : a.k) + head_at;
                    const uint32_t to = kv_at + stage * C::tile_bytes;
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        if (j * RW >= mine) break;
                        const bool in = row[j] != kXNoRow && ch_in;
                        cp_async16(to + j * RW * 128 + (kv_swz ^ (uint32_t)((j * RW & 7) << 4)), from + (uint64_t)(in ? row[j] : 0u) * 16, in ? 16u : 0u);
                    }
                    if (lane == 0) mbar_arrive(msmem_u32(&sm.full[stage]));
                    if ((int)copy != a.drop_item) cp_arrive(msmem_u32(&sm.full[stage]));
                }
                if (!ok) break;
            }
            tiles0 += pc.tile_end - pc.tile;
            ++piece;
        }
        cp_wait_all();
        if (lw == 0 && lane < 2) a.meta[2 * blockIdx.x + lane] = lane ? meta[1] : meta[0];
    } else if (warp == 8) {
        // ------------------------------------------------------------------ matrix products: the warp walks in step, one lane issues
        const int steps16 = (a.D + 15) / 16;
        const uint32_t idesc_s = mma_idesc(kXKeys, false) | negate, idesc_o = mma_idesc(steps16 * 16, true);
        const uint32_t q_at = msmem_u32(sm.q), kv_at = msmem_u32(sm.kv);
        uint32_t done[2] = {0, 0};                         // outputs issued for each stream
        bool ok = true;
        while (ok && XCut::next(a, run, &pc)) {
            const bool two = pc.rows > 128;
            const int n = (pc.tile_end - pc.tile) * (two ? 2 : 1);
            const uint32_t qb = (uint32_t)piece % C::q_bufs;
            if (!(ok = mbar_wait(msmem_u32(&sm.q_full[qb]), ((uint32_t)piece / C::q_bufs) & 1u, abort_flag, limit))) break;
#pragma unroll 1
            for (int i = 0; i < n + 2; ++i) {
                const uint32_t s = i & 1;
                if (i >= 2) {                              // outputs of step i - 2
                    const int j = i - 2;
                    const uint32_t copy = 2 * (tiles0 + (two ? j >> 1 : j)) + 1, stage = copy % C::stages;
                    if (!(ok = mbar_wait(msmem_u32(&sm.full[stage]), (copy / C::stages) & 1u, abort_flag, limit))) break;
                    if (j == 0 && piece > 0 && !(ok = mbar_wait(msmem_u32(&sm.o_free), (piece - 1) & 1, abort_flag, limit))) break;
                    const uint64_t dv = sw128_desc(kv_at + stage * C::tile_bytes, kXKeys * 128);
                    const uint32_t p = tmem + C::s_col + s * kXKeys, d = tmem + C::o_col + s * DP, parity = (s ? done[1] : done[0]) & 1u;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (!(ok = mbar_wait(msmem_u32(&sm.p_ready[s][h]), parity, abort_flag, limit))) break;
                        if (elect_one()) {
                            fence_async_proxy();           // the copies' writes (generic) before the products' reads
                            tc_after();
#pragma unroll
                            for (int ks = 4 * h; ks < 4 * h + 4; ++ks) mma_ts(d, p + ks * 8, dv + (uint64_t)(ks * 2048 / 16), idesc_o, j >= 2 || ks != 0, -1);
                            if (h == 0) mma_commit(msmem_u32(&sm.half_done[s]));
                            else {
                                if (!two || s == 1) mma_commit(msmem_u32(&sm.empty[stage]));
                                if (j + 2 >= n) mma_commit(msmem_u32(&sm.o_done[s]));
                                if (n == 1) mma_commit(msmem_u32(&sm.o_done[1]));
                            }
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (s) ++done[1]; else ++done[0];
                }
                if (i < n) {
                    const uint32_t copy = 2 * (tiles0 + (two ? i >> 1 : i)), stage = copy % C::stages;
                    if (!(ok = mbar_wait(msmem_u32(&sm.full[stage]), (copy / C::stages) & 1u, abort_flag, limit))) break;
                    const uint64_t dq = sw128_desc(q_at + qb * C::q_bytes + (two ? s * C::q_half : 0), 16), dk = sw128_desc(kv_at + stage * C::tile_bytes, 16);
                    const uint32_t d = tmem + C::s_col + s * kXKeys;
                    if (elect_one()) {
                        fence_async_proxy();
                        tc_after();
#pragma unroll
                        for (int ks = 0; ks < DP / 16; ++ks)       // 16 dimensions = 32 bytes along a swizzled row; 64 to a block of columns
                            if (ks < steps16)
                                mma_ss(d, dq + (uint64_t)((ks >> 2) * (128 * 128 / 16) + (ks & 3) * 2), dk + (uint64_t)((ks >> 2) * (kXKeys * 128 / 16) + (ks & 3) * 2),
                                       idesc_s, ks != 0, -1);
                        if (!two || s == 1) mma_commit(msmem_u32(&sm.empty[stage]));
                        mma_commit(msmem_u32(&sm.s_full[s]));
                        mbar_arrive(msmem_u32(&sm.s_full[s]));
                        if (i + 1 == n) mma_commit(msmem_u32(&sm.q_empty[qb]));
                    }
                    __syncwarp();
                }
            }
            if (!ok) break;
            tiles0 += pc.tile_end - pc.tile;
            ++piece;
        }
        // nothing of this block is in flight when it leaves, whatever happened
        if (elect_one()) mma_commit(msmem_u32(&sm.last));
        for (int i = 0; i < 1000000 && !__all_sync(kFullMask, mbar_try(msmem_u32(&sm.last), 0)); ++i) {}
    } else {
        // ------------------------------------------------------------------ softmax: stream s, a row per thread
        const int s = warp >> 2, in_stream = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lanes + C::s_col + s * kXKeys, o_at = tmem + lanes + C::o_col;
        const float scale = fabsf(a.scale_log2e);
        uint32_t steps = 0, shared_pieces = 0;             // steps of this stream so far, pieces whose rows both streams had
        int cut = 0;
        bool ok = true;
        while (ok && XCut::next(a, run, &pc)) {
            const bool two = pc.rows > 128;
            float ref = neg_inf(), sum = 0.f;
            const int first = pc.tile + (two ? 0 : s), by = two ? 1 : 2;
#pragma unroll 1
            for (int t = first; t < pc.tile_end; t += by, ++steps) {
                if (!mbar_wait(msmem_u32(&sm.s_full[s]), steps & 1u, abort_flag, limit)) { ok = false; break; }
                tc_after();
                const uint32_t (*seen)[2] = sm.seen[(tiles0 + t - pc.tile) % kXSeen];
                const bool all = (seen[0][0] & seen[1][0] & seen[2][0]) == 0xffffffffu && seen[0][1] == 0xfffu && seen[1][1] == 0xfffu && seen[2][1] == 0xffu;
                // Half a tile at a time: the first half's outputs are under way while the second goes through here, and 64 scores fit
                // the registers.
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[64];
                    tm_ld64(s_at + 64 * h, x);
                    if (!all) {                            // the end of the prefix, or a page that there is not
                        const uint64_t m0 = (uint64_t)seen[0][1] << 32 | seen[0][0], m1 = (uint64_t)seen[1][1] << 32 | seen[1][0], m2 = (uint64_t)seen[2][1] << 32 | seen[2][0];
                        const uint64_t see = h ? m1 >> 20 | m2 << 24 : m0 | m1 << 44;
                        const uint32_t see0 = (uint32_t)see, see1 = (uint32_t)(see >> 32);
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            if (!((see0 >> j) & 1u)) x[j] = 0xff800000u;
                            if (!((see1 >> j) & 1u)) x[32 + j] = 0xff800000u;
                        }
                    }
                    float m0 = neg_inf(), m1 = m0;
#pragma unroll
                    for (int j = 0; j < 64; j += 4) {
                        m0 = max3(m0, __uint_as_float(x[j]), __uint_as_float(x[j + 1]));
                        m1 = max3(m1, __uint_as_float(x[j + 2]), __uint_as_float(x[j + 3]));
                    }
                    const float top = fmaxf(m0, m1) * scale;
                    const bool raise = top > (ref == neg_inf() ? ref : ref + kRaise);
                    if (__any_sync(kFullMask, raise)) {
                        const float factor = raise ? ex2(ref - top) : 1.f;         // 0 where nothing has been seen before
                        if (raise) { ref = top; sum *= factor; }
                        if (h && !mbar_wait(msmem_u32(&sm.half_done[s]), steps & 1u, abort_flag, limit)) { ok = false; break; }
                        if (t > first || h) {              // (these scores came behind the outputs of all steps before)
                            tc_after();
#pragma unroll 1
                            for (int c = 0; c < DP; c += 16) {
                                uint32_t o[16];
                                tm_ld16(o_at + s * DP + c, o);
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * factor);
                                tm_st16(o_at + s * DP + c, o);
                            }
                        }
                    }
                    const float shift = ref == neg_inf() ? 0.f : -ref;
                    float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t p[16];
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            float e0, e1, e2, e3;
                            fma2(e0, e1, __uint_as_float(x[32 * q + j]), __uint_as_float(x[32 * q + j + 1]), scale, shift);
                            fma2(e2, e3, __uint_as_float(x[32 * q + j + 2]), __uint_as_float(x[32 * q + j + 3]), scale, shift);
                            e0 = ex2(e0); e1 = ex2(e1); e2 = ex2(e2); e3 = ex2(e3);
                            add2(s0, s1, e0, e1); add2(s2, s3, e2, e3);
                            p[j / 2] = pack_bf16(e0, e1); p[j / 2 + 1] = pack_bf16(e2, e3);
                        }
                        tm_st16(s_at + 32 * h + 16 * q, p);
                    }
                    sum += (s0 + s1) + (s2 + s3);
                    tm_wait_st();
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(msmem_u32(&sm.p_ready[s][h]));
                }
                if (!ok) break;
            }
            if (!ok) break;
            // --- the item's outputs.  A thread has a row's, and memory wants rows' neighbours: 32 columns at a time go through shared memory, and
            // four lanes (a piece of an item: eight) have a row.
            const int64_t part = pc.whole() ? -1 : (int64_t)(2 * blockIdx.x + cut) * kXRows;
            if (part >= 0) ++cut;
            const int row0 = (two ? s * 128 : 0) + (warp & 3) * 32, row = row0 + lane;
            const bool in = row < pc.rows;
            const PrefixRow w = prefix_row(a, pc.lo, pc.h, pc.row0 + (in ? row : 0));
            const int64_t out_at = (int64_t)w.b * a.o_seq + (int64_t)w.i * a.o_row + (int64_t)w.head * a.o_head;
            grid_dependency_wait();                        // the rows' own part
            float own = neg_inf();
            bool write = in;
            if (part < 0) write = prefix_own(a, w, &own) && in;
            const int c0 = two ? 0 : s * (DP / 2), c1 = two ? DP : c0 + DP / 2;
            uint4 old[4];                                  // what the rows that this lane will write have of their own, one block of columns ahead
            const auto fetch = [&](int c) {
                const int col = c + (lane & 3) * 8;
                const uint32_t rows_in = __ballot_sync(kFullMask, write);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = i * 8 + (lane >> 2);
                    const int64_t at = __shfl_sync(kFullMask, out_at, r);
                    if (((rows_in >> r) & 1u) && col < a.D) old[i] = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.out + at + col);
                    else old[i] = make_uint4(0, 0, 0, 0);
                }
            };
            if (part < 0) fetch(c0);
            if (!mbar_wait(msmem_u32(&sm.o_done[s]), piece & 1, abort_flag, limit)) { ok = false; break; }
            float f = 1.f, g = 0.f;                        // factors of this stream's output, and of the other's
            if (!two) {
                if (!mbar_wait(msmem_u32(&sm.o_done[s ^ 1]), piece & 1, abort_flag, limit)) { ok = false; break; }
                sm.ml[s][in_stream][0] = ref; sm.ml[s][in_stream][1] = sum;
                __syncwarp();
                if (lane == 0) mbar_arrive(msmem_u32(&sm.ml_ready));
                if (!mbar_wait(msmem_u32(&sm.ml_ready), shared_pieces & 1u, abort_flag, limit)) { ok = false; break; }
                ++shared_pieces;
                const float ref2 = sm.ml[s ^ 1][in_stream][0], sum2 = sm.ml[s ^ 1][in_stream][1], m = fmaxf(ref, ref2);
                f = sum == 0.f ? 0.f : ex2(ref - m); g = sum2 == 0.f ? 0.f : ex2(ref2 - m);
                // (in the same order on either side)
                const float l0 = s ? sum2 * g : sum * f, l1 = s ? sum * f : sum2 * g;
                sum = l0 + l1; ref = m;
            } else if (sum == 0.f) f = 0.f;
            float w_own = 0.f, w_pre = 1.f, lse = 0.f;
            if (part < 0) write = prefix_join(own, ref, sum, &w_own, &w_pre, &lse) && write;
            const uint32_t rows_in = __ballot_sync(kFullMask, write);
            tc_after();
            float4 (*turn)[8] = sm.turn[warp];
#pragma unroll 1
            for (int c = c0; c < c1; c += 32) {
                if (c >= a.D) break;
                uint32_t u[32];
                float y[32];
                tm_ld32(o_at + s * DP + c, u);
#pragma unroll
                for (int j = 0; j < 32; ++j) y[j] = f == 0.f ? 0.f : __uint_as_float(u[j]) * f;      // (where nothing was seen O may hold anything)
                if (!two) {
                    tm_ld32(o_at + (s ^ 1) * DP + c, u);
#pragma unroll
                    for (int j = 0; j < 32; ++j) y[j] += g == 0.f ? 0.f : __uint_as_float(u[j]) * g;
                }
                __syncwarp();                              // the last block of columns has been read
#pragma unroll
                for (int j = 0; j < 8; ++j) turn[lane][j ^ (lane & 7)] = make_float4(y[4 * j] * w_pre, y[4 * j + 1] * w_pre, y[4 * j + 2] * w_pre, y[4 * j + 3] * w_pre);
                __syncwarp();
                if (part >= 0) {
                    const int col = c + (lane & 7) * 4;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = i * 4 + (lane >> 3);
                        const float4 v = turn[r][(lane & 7) ^ (r & 7)];
                        if (((rows_in >> r) & 1u) && col < a.D) *reinterpret_cast<float4*>(a.part_o + (part + row0 + r) * a.D + col) = v;
                    }
                } else {
                    const int col = c + (lane & 3) * 8;
                    uint4 now[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) now[i] = old[i];
                    if (c + 32 < c1 && c + 32 < a.D) fetch(c + 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 8 + (lane >> 2);
                        const int64_t at = __shfl_sync(kFullMask, out_at, r);
                        const float wo = __shfl_sync(kFullMask, w_own, r);
                        const float4 v0 = turn[r][((lane & 3) * 2) ^ (r & 7)], v1 = turn[r][((lane & 3) * 2 + 1) ^ (r & 7)];
                        const uint32_t o[4] = {now[i].x, now[i].y, now[i].z, now[i].w};
                        const float v[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
                        uint32_t z[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            z[k] = pack_bf16(fmaf(wo, __uint_as_float(o[k] << 16), v[2 * k]), fmaf(wo, __uint_as_float(o[k] & 0xffff0000u), v[2 * k + 1]));
                        if (((rows_in >> r) & 1u) && col < a.D) *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + at + col) = make_uint4(z[0], z[1], z[2], z[3]);
                    }
                }
            }
            if (write && (two || s == 0)) {
                if (part >= 0) { a.part_ml[2 * (part + row)] = ref; a.part_ml[2 * (part + row) + 1] = sum; }
                else a.own_lse[((int64_t)w.b * a.n + w.i) * a.H + w.head] = lse;
            }
            tc_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(msmem_u32(&sm.o_free));
            tiles0 += pc.tile_end - pc.tile;
            ++piece;
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    grid_dependency_wait();                                // (a block without work too: what follows this kernel follows the one before it)
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::tmem_cols) : "memory");
    if (sm.abort_flag && tid == 0) {
        atomicOr(a.pages.status, (uint32_t)DBA_TREE_TIMEOUT);
        a.meta[2 * blockIdx.x] = make_int4(-2, 0, 0, 0);   // (over what the loader wrote)
    }
}

template <int DP>
cudaError_t configure_prefix_mma() {
    static_assert(sizeof(XSmem<DP>) <= 227 * 1024, "a block's shared memory");
    return cudaFuncSetAttribute(tree_prefix_mma_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(XSmem<DP>));
}
template <int DP>
cudaError_t launch_prefix_mma(const TreePrefix& a, int grid, cudaStream_t st) {
    const uint32_t negate = a.scale_log2e < 0.f ? 1u << 13 : 0u;       // the scores' sign by the instruction, their size by the softmax
    return launch_after(tree_prefix_mma_kernel<DP>, dim3(grid), dim3(kXThreads), sizeof(XSmem<DP>), st, a, negate);
}

}  // namespace

int tree_prefix_mma_rows() { return kXRows; }
cudaError_t configure_tree_prefix_mma() {
    const cudaError_t e = configure_prefix_mma<64>();
    return e == cudaSuccess ? configure_prefix_mma<128>() : e;
}
cudaError_t launch_tree_prefix_mma(const TreePrefix& a, int grid, cudaStream_t st) {
    return a.D <= 64 ? launch_prefix_mma<64>(a, grid, st) : launch_prefix_mma<128>(a, grid, st);
}

}  // namespace dba
