// Attention over prefixes that sequences share on the tensor cores: bf16, head sizes up to 128.
//
// The rows of all sequences of a prefix and all query heads of a key head are one matrix Q [rows, D], the prefix the other:
//     S = Q K^T,   P = 2^(scale log2(e) S - m),   O += P V,   l += sum P,
// in items of 256 rows (see tree_span.cuh).  One block an SM, two streams of 128 rows, each with a warp for its products: while one stream's
// scores go through the softmax the tensor cores have the other's products.  An item of at most 128 rows gives both streams the same rows and
// every other tile of 128 keys, and their two results are added in the end.
//   softmax    two warpgroups, one to a stream, a thread to a row, half a tile (64 keys) at a time.  Scores come out of tensor memory, P goes
//              back over them (bf16, as the matrix instruction needs it: half a unit in the 8th bit of each; the sum is taken before the
//              rounding).  The reference m is raised only when a half's maximum lies more than 2^8 above it, and O rescaled in tensor memory then.
//              Three of four exponentials by ex2, the fourth by a polynomial on the fma pipes (below).
//   products   one lane of a stream's warp issues, a half at a time: P V of half h, then the next tile's scores into the half that P has left.
//              A stream's next scores come behind its outputs, so their completion shows that of the outputs before.
//   loaders    keys and values K-major and MN-major, both [key][d] in the 128-byte swizzle.  Pages made of eights of places: one warp sends
//              tensor-map boxes, a lane to a stretch of a page, another one fetches queries (16-byte cp.async; a block's first ones the
//              softmax warps, which have nothing to do yet); places of a box that lie
//              behind the prefix are hidden from the scores, and their values made zeros.  Other pages, and strides that no tensor map has: four
//              warps of cp.async with zero fill, every place looked up by itself, so pages of any size may end inside a tile.
// The epilogue joins a whole item with the rows' own part and writes the result; pieces of an item go to scratch, and to the joining
// kernel (tree_prefix.cu).  Only the epilogue needs the kernel before this one, so the rest runs beside its last blocks.  Every wait on an
// mbarrier is bounded: one that runs out winds the block down and marks the call as failed.
//
// Measured: beams of 20 on 64 sentences, 32 heads over 8 of 128, 6007 tokens (126 GFLOP, 40960 rows, and 5 of the rows' own part): the call 160 us with
// idle time around it, 170 call after call at the clocks that this brings (0.82 and 0.77 PFLOP/s, 51 and 48 % of the rate of a large matrix product), 30 of them the
// own part.  No pipe is full (tensor cores 51 %, exponentials 38 %, issue 46 %): what bounds it is the chain of a softmax warp, with two of them a scheduler.  A
// tile of 128 keys takes a stream's warps some 3500 cycles, of which exponentials, sums and packing 2000, and the same warps write the outputs.  Eight rows on
// 100003 tokens (205 MB): 54 us, of which the main loop 29, at HBM's rate.  Both sides of what was chosen, the document's call in us, all with idle time around
// it and in one session: half tiles 157, whole ones 170; a quarter of the exponentials as polynomials 157, none 162, half of them 164; the first queries by one
// warp 156, by eight 154.
#include <cuda_bf16.h>

#include "tree_boxes.cuh"
#include "tree_span.cuh"

namespace dba {

namespace {

constexpr int kXKeys = 128, kXRows = 256;
constexpr int kXSeen = 8;              // more than the tiles the loader may be ahead by

template <int DP, bool TMA> struct XConf {
    static constexpr int load_warps = TMA ? 2 : 4, threads = 32 * (10 + load_warps);
    static constexpr int q_warps = TMA ? 1 : load_warps;               // of them, those that load queries
    static constexpr int tile_bytes = kXKeys * DP * 2, q_half = 128 * DP * 2, q_bytes = 2 * q_half;
    static constexpr int stages = DP == 128 ? 4 : 8, q_bufs = DP == 128 ? 1 : 2;
    static constexpr int s_col = 0, o_col = 256, tmem_cols = 512;
};
template <int DP, bool TMA> struct XSmem {
    using C = XConf<DP, TMA>;
    alignas(1024) unsigned char q[C::q_bufs][C::q_bytes];
    unsigned char kv[C::stages][C::tile_bytes];
    float4 turn[8][32][8];                      // by softmax warp: 32 columns of its rows, on their way to memory
    uint64_t full[C::stages], empty[C::stages];
    uint64_t s_full[2][2], p_ready[2][2], pv_done[2], o_done[2];
    uint64_t q_full[C::q_bufs], q_empty[C::q_bufs];
    uint64_t q_first, o_free, ml_ready, last[2];
    float ml[2][128][2];
    uint32_t seen[kXSeen][4];                   // (by tile, in turn) which of its rows there are
    uint32_t tmem_base;
    int abort_flag;
    union {
        SpanShared span;                        // (until the roles begin)
        alignas(16) uint32_t rows[kXKeys];      // a tile's rows in the cache, in 16 bytes; kXNoRow: none
    };
};
constexpr uint32_t kXNoRow = 0xffffffffu;
// NaN where one of them is
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
// (x, y) = (a0, a1) * b + (c0, c1), and (x, y) = (x, y) * (a0, a1) + c
__device__ __forceinline__ void fma2v(float& x, float& y, float a0, float a1, float b, float c0, float c1) {
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%5, %6};\n\tfma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(x), "=f"(y) : "f"(a0), "f"(a1), "f"(b), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void fma2v2(float& x, float& y, float a0, float a1, float c) {
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\tmov.b64 c, {%4, %4};\n\tfma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "+f"(x), "+f"(y) : "f"(a0), "f"(a1), "f"(c));
}
// 2^x of two numbers on the fused multiply-add pipes, x up to some 2^7: the whole number next to x by adding and taking away 1.5 2^23, a polynomial of
// degree 4 for the rest f in -1/2 .. 1/2 (least largest relative error, fitted by reweighted least squares with 1 at 0: 2.9e-6), the whole
// number into the exponent.  Below -126 it goes to 0 through subnormals, and is 0 from -127 on.  NaN gives 0 too: the softmax sees to it that a row with such
// a score has a reference of NaN, and with it the exponentials beside these.
__device__ __forceinline__ void ex2_pair(float& x, float& y) {
    float tx = fmaxf(x, -127.f), ty = fmaxf(y, -127.f), fx = tx, fy = ty, nx, ny, px, py;
    add2(tx, ty, 12582912.f, 12582912.f);
    nx = tx; ny = ty;
    add2(nx, ny, -12582912.f, -12582912.f);
    fma2v(fx, fy, nx, ny, -1.f, fx, fy);
    px = py = 0.009582852944731712f;
    fma2v2(px, py, fx, fy, 0.055906426161527634f);
    fma2v2(px, py, fx, fy, 0.24024099111557007f);
    fma2v2(px, py, fx, fy, 0.6931241750717163f);
    fma2v2(px, py, fx, fy, 1.f);
    x = __uint_as_float(__float_as_uint(px) + (__float_as_uint(tx) << 23));
    y = __uint_as_float(__float_as_uint(py) + (__float_as_uint(ty) << 23));
}
using XCut = PrefixCut<kXKeys, kXRows, 128>;

// 32 queries of an item from its row r0 on into their place in shared memory (both halves begin at q_at), zeros beyond the rows and the head size: a lane finds
// one row, and every lane copies chunks of all.
template <int DP>
__device__ __forceinline__ void copy_queries(const TreePrefix& a, const XCut::Piece& pc, uint32_t q_at, int r0, int lane) {
    constexpr int CH = DP / 8, RW = 32 / CH, NJ = 32 / RW;             // 16-byte chunks of a row, rows a warp copies at a time, and how often
    const int ch = lane % CH, sub = lane / CH;
    const bool ch_in = ch * 8 < a.D;
    const uint32_t swz = (uint32_t)((ch & 7) ^ sub) << 4;              // the swizzle moves a chunk by its row's last three bits
    const char* const q = (const char*)a.q + (ch_in ? ch * 16 : 0);
    int64_t q_row = -1;
    if (r0 + lane < pc.rows) {
        const PrefixRow w = prefix_row(a, pc.lo, pc.h, pc.row0 + r0 + lane);
        q_row = 2 * ((int64_t)w.b * a.q_seq + (int64_t)w.i * a.q_row + (int64_t)w.head * a.q_head);
    }
    const uint32_t to = q_at + (r0 >= 128 ? 128 * DP * 2 : 0) + (uint32_t)(ch >> 3) * (128 * 128) + (uint32_t)((r0 & 127) + sub) * 128;
#pragma unroll
    for (int j0 = 0; j0 < NJ; j0 += 8) {
        int64_t from[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) from[j] = __shfl_sync(kFullMask, q_row, (j0 + j) * RW + sub);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            cp_async16(to + (j0 + j) * RW * 128 + (swz ^ (uint32_t)(((j0 + j) * RW & 7) << 4)), from[j] >= 0 ? q + from[j] : q, from[j] >= 0 && ch_in ? 16u : 0u);
    }
}

template <int DP, bool TMA>
__global__ void __launch_bounds__(XConf<DP, TMA>::threads, 1) tree_prefix_mma_kernel(const __grid_constant__ TreePrefix a, const __grid_constant__ TreeBoxes maps,
                                                                        const uint32_t negate) {
    using C = XConf<DP, TMA>;
    extern __shared__ __align__(1024) unsigned char xraw[];
    XSmem<DP, TMA>& sm = *reinterpret_cast<XSmem<DP, TMA>*>(xraw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile int* abort_flag = &sm.abort_flag;
    const long long limit = a.wait_clocks > 0 ? a.wait_clocks : kMWaitClocks;
    if (tid == 0) {
        for (int s = 0; s < C::stages; ++s) { mbar_init(msmem_u32(&sm.full[s]), TMA ? 1 : 33 * C::load_warps); mbar_init(msmem_u32(&sm.empty[s]), 2); }
        // (s_full: the products, and an arrival of the issuing thread, which passes on what the loader wrote before it)
        for (int s = 0; s < 2; ++s) {
            for (int h = 0; h < 2; ++h) { mbar_init(msmem_u32(&sm.s_full[s][h]), 2); mbar_init(msmem_u32(&sm.p_ready[s][h]), 4); }
            mbar_init(msmem_u32(&sm.pv_done[s]), 1); mbar_init(msmem_u32(&sm.o_done[s]), 1); mbar_init(msmem_u32(&sm.last[s]), 1);
        }
        for (int i = 0; i < C::q_bufs; ++i) { mbar_init(msmem_u32(&sm.q_full[i]), 32 * C::q_warps); mbar_init(msmem_u32(&sm.q_empty[i]), 2); }
        mbar_init(msmem_u32(&sm.q_first), 256);
        mbar_init(msmem_u32(&sm.o_free), 8);
        mbar_init(msmem_u32(&sm.ml_ready), 8);
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
    SpanRun run = XCut::run<C::threads>(a, 3, &sm.span);
    __syncthreads();           // its numbers have been read: their place is used again
    tc_after();
    const uint32_t tmem = sm.tmem_base;
    XCut::Piece pc;
    int piece = 0;
    uint32_t tiles0 = 0;                                   // tiles before this piece
    if (warp > 9) {
        // ------------------------------------------------------------------ loaders.  TMA: one warp for keys and values, a lane to a box, one for queries.
        // Else all of them for everything, warp lw rows 32 lw .. 32 lw + 31 of a tile.
        constexpr int CH = DP / 8, RW = 32 / CH, NJ = 32 / RW;         // 16-byte chunks of a row, rows a warp copies at a time, and how often
        const int lw = warp - 10, ch = lane % CH, sub = lane / CH, q_warp = TMA ? lw - 1 : lw;
        const bool ch_in = ch * 8 < a.D;
        const uint32_t q_at = msmem_u32(sm.q), kv_at = msmem_u32(sm.kv);
        const uint32_t swz = (uint32_t)((ch & 7) ^ sub) << 4;          // the swizzle moves a chunk by its row's last three bits
        const uint32_t page16 = (uint32_t)(a.pages.page_stride / 8), token16 = (uint32_t)(a.pages.token_stride / 8);
        const int box_lane = TMA ? min(lane, kXKeys / maps.rows - 1) * maps.rows : lw * 32 + lane;       // the lane's (first) place in a tile
        uint32_t* const rows = sm.rows + lw * 32;
        uint32_t copy = 0;
        int cut = 0;
        int4 meta[2] = {make_int4(-1, 0, 0, 0), make_int4(-1, 0, 0, 0)};
        bool ok = true;
        if (TMA && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane ? &maps.v : &maps.k) : "memory");
        while (ok && XCut::next(a, run, &pc)) {
            if (!pc.whole()) { if (cut == 0) meta[0] = make_int4(pc.g, pc.h, pc.rb, 0); else meta[1] = make_int4(pc.g, pc.h, pc.rb, 0); ++cut; }
            // where a tile's rows are: page numbers are fetched a tile ahead and not looked at before their turn
            const int32_t* const table = a.pages.table + (int64_t)pc.g * a.pages.table_stride;
            int32_t id = 0;
            const auto fetch = [&](int t) {
                const int place = t * kXKeys + box_lane;
                id = place < pc.len ? __ldg(table + tree_page(a.pages, (uint32_t)place)) : -1;       // (below the table's entries: len is)
            };
            if (!TMA || lw == 0) fetch(pc.tile);
            if (q_warp >= 0) {                             // queries
                const uint32_t qb = (uint32_t)piece % C::q_bufs;
                if (piece >= C::q_bufs && !mbar_wait(msmem_u32(&sm.q_empty[qb]), ((uint32_t)piece / C::q_bufs - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                if (piece > 0)                             // (the first ones are the softmax warps' to copy, which have nothing to do yet)
#pragma unroll 1
                    for (int r0 = q_warp * 32; r0 < (pc.rows > 128 ? kXRows : 128); r0 += 32 * C::q_warps) copy_queries<DP>(a, pc, q_at + qb * C::q_bytes, r0, lane);
                cp_arrive(msmem_u32(&sm.q_full[qb]));
            }
            const int64_t head_at = 2 * (int64_t)pc.h * a.pages.head_stride + (ch_in ? ch * 16 : 0);
#pragma unroll 1
            for (int t = pc.tile; t < (TMA && lw > 0 ? 0 : pc.tile_end); ++t) {
                const int place = t * kXKeys + box_lane;
                const uint32_t in_page = (uint32_t)place - tree_page(a.pages, (uint32_t)place) * (uint32_t)a.pages.page_size;
                const bool there = (uint32_t)id < (uint32_t)a.pages.num_pages;
                if (!there && place < pc.len) atomicOr(a.pages.status, (uint32_t)DBA_TREE_BAD_PAGE);
                const int page = there ? id : a.pages.num_pages;       // (a page that there is not: zeros)
                if (TMA) {
                    boxes_seen(sm.seen[(tiles0 + t - pc.tile) % kXSeen], maps.rows, box_lane, there, pc.len - t * kXKeys);
                    __syncwarp();
                    if (t + 1 < pc.tile_end) fetch(t + 1);
#pragma unroll
                    for (int k = 0; k < 2; ++k, ++copy) {
                        const uint32_t stage = copy % C::stages, use = copy / C::stages, full = msmem_u32(&sm.full[stage]);
                        if (use > 0 && !mbar_wait(msmem_u32(&sm.empty[stage]), (use - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                        if (lane == 0) mbar_expect(full, C::tile_bytes);
                        __syncwarp();
                        if ((int)copy != a.drop_item && lane * maps.rows < kXKeys) {
#pragma unroll
                            for (int c = 0; c < DP / 64; ++c)
                                copy_box(kv_at + stage * C::tile_bytes + c * (kXKeys * 128) + box_lane * 128, k ? &maps.v : &maps.k, 64 * c, (int)in_page, page, pc.h, full);
                        }
                    }
                } else {
                    const uint32_t at = there ? (uint32_t)id * page16 + in_page * token16 : kXNoRow, seen = __ballot_sync(kFullMask, there);     // (the host has seen to it that 32 bits are enough)
                    __syncwarp();                          // the last tile's rows have been read
                    rows[(lane % RW) * NJ + lane / RW] = at;           // a lane will copy rows sub, sub + RW, ..: its numbers lie side by side
                    if (lane == 0) sm.seen[(tiles0 + t - pc.tile) % kXSeen][lw] = seen;
                    __syncwarp();
                    if (t + 1 < pc.tile_end) fetch(t + 1);
                    uint32_t row[NJ];                      // (read before the copies: they are not reordered)
#pragma unroll
                    for (int j = 0; j < NJ; j += 4) {
                        const uint4 r4 = *reinterpret_cast<const uint4*>(rows + sub * NJ + j);
                        row[j] = r4.x; row[j + 1] = r4.y; row[j + 2] = r4.z; row[j + 3] = r4.w;
                    }
#pragma unroll 1
                    for (int k = 0; k < 2; ++k, ++copy) {
                        const uint32_t stage = copy % C::stages, use = copy / C::stages;
                        if (use > 0 && !mbar_wait(msmem_u32(&sm.empty[stage]), (use - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                        const char* from = (const char*)(k ? a.v : a.k) + head_at;
                        const uint32_t to = kv_at + stage * C::tile_bytes + (uint32_t)(ch >> 3) * (kXKeys * 128) + (uint32_t)(lw * 32 + sub) * 128;
#pragma unroll
                        for (int j = 0; j < NJ; ++j) {
                            const bool in = row[j] != kXNoRow && ch_in;
                            cp_async16(to + j * RW * 128 + (swz ^ (uint32_t)((j * RW & 7) << 4)), from + (uint64_t)(in ? row[j] : 0u) * 16, in ? 16u : 0u);
                        }
                        if (lane == 0) mbar_arrive(msmem_u32(&sm.full[stage]));
                        if ((int)copy != a.drop_item) cp_arrive(msmem_u32(&sm.full[stage]));
                    }
                }
                if (!ok) break;
            }
            tiles0 += pc.tile_end - pc.tile;
            ++piece;
        }
        if (lw == 0 && lane < 2) a.meta[2 * blockIdx.x + lane] = lane ? meta[1] : meta[0];
        // nothing of this block is in flight when it leaves (where nobody gave up, all boxes have been waited for)
        cp_wait_all();
        if (TMA && lw == 0 && *abort_flag)
            for (uint32_t c = copy > C::stages ? copy - C::stages : 0; c < copy; ++c)
                for (int i = 0; i < 100000 && (int)c != a.drop_item && !__all_sync(kFullMask, mbar_try(msmem_u32(&sm.full[c % C::stages]), (c / C::stages) & 1u)); ++i) {}
    } else if (warp > 7) {
        // ------------------------------------------------------------------ matrix products of stream s: the warp walks in step, one lane issues
        const int s = warp - 8, steps16 = (a.D + 15) / 16;
        const uint32_t idesc_s = mma_idesc(kXKeys / 2, false) | negate, idesc_o = mma_idesc(steps16 * 16, true);
        const uint32_t p_at = tmem + C::s_col + s * kXKeys, o_at = tmem + C::o_col + s * DP;
        const uint32_t s_full = msmem_u32(&sm.s_full[s][0]), p_ready = msmem_u32(&sm.p_ready[s][0]), pv_done = msmem_u32(&sm.pv_done[s]);
        const uint64_t k_desc = sw128_desc(msmem_u32(sm.kv), 16), v_desc = sw128_desc(msmem_u32(sm.kv), kXKeys * 128);
        uint32_t done = 0;                                 // outputs issued
        bool ok = true, shared_before = false;             // the last piece's tiles went to the two streams in turn
        while (ok && XCut::next(a, run, &pc)) {
            const bool two = pc.rows > 128;
            const int tiles = pc.tile_end - pc.tile, by = two ? 1 : 2, n = two ? tiles : (tiles + 1 - s) / 2;
            const uint32_t qb = (uint32_t)piece % C::q_bufs;
            if (!(ok = mbar_wait(msmem_u32(&sm.q_full[qb]), ((uint32_t)piece / C::q_bufs) & 1u, abort_flag, limit))) break;
            if (piece == 0 && !(ok = mbar_wait(msmem_u32(&sm.q_first), 0, abort_flag, limit))) break;
            // A stage's wait tells a phase from the one before it alone, so what was there before has to have come.  This stream has waited for its own tiles; the
            // other one's keys of the last piece have come when its scores are done (one buffer of queries: their wait has shown it), and all the rest
            // before this piece by the wait for the outputs' place below.
            if (C::q_bufs > 1 && shared_before &&
                !(ok = mbar_wait(msmem_u32(&sm.q_empty[(uint32_t)(piece - 1) % C::q_bufs]), ((uint32_t)(piece - 1) / C::q_bufs) & 1u, abort_flag, limit))) break;
            shared_before = !two;
            const uint64_t dq = sw128_desc(msmem_u32(sm.q[qb]) + (two ? s * C::q_half : 0), 16);
            // rows of this stream's last tile behind the prefix' end
            const int n_tail = pc.tile_end == pc.tiles && (pc.tiles - 1 - pc.tile) % by == (two ? 0 : s) ? (int)((uint32_t)pc.tiles * kXKeys - (uint32_t)pc.len) : 0;
            uint32_t k_copy = 2 * (tiles0 + (two ? 0 : s)), v_copy = k_copy + 1;
#pragma unroll 1
            for (int g = n ? -1 : 0; g < n; ++g) {
                const uint32_t v_stage = v_copy % C::stages, k_stage = k_copy % C::stages;
                const uint64_t dv = v_desc + (uint64_t)(v_stage * (C::tile_bytes / 16)), dk = k_desc + (uint64_t)(k_stage * (C::tile_bytes / 16));
                if (g == 0 && piece > 0 && !(ok = mbar_wait(msmem_u32(&sm.o_free), (piece - 1) & 1, abort_flag, limit))) break;      // (the outputs' place)
                if (g >= 0 && !(ok = mbar_wait(msmem_u32(&sm.full[v_stage]), (v_copy / C::stages) & 1u, abort_flag, limit))) break;
                // the scores of half a tile, over the probabilities of the same half of the one before
                const auto scores = [&](int h) {
                    if (elect_one()) {
                        if (!TMA || g < 0) fence_async_proxy();        // the copies' writes (generic) before the products' reads
                        tc_after();
#pragma unroll
                        for (int ks = 0; ks < DP / 16; ++ks)       // 16 dimensions = 32 bytes along a swizzled row; 64 to a block of columns
                            if (ks < steps16)
                                mma_ss(p_at + 64 * h, dq + (uint64_t)((ks >> 2) * (128 * 128 / 16) + (ks & 3) * 2),
                                       dk + (uint64_t)(h * (64 * 128 / 16) + (ks >> 2) * (kXKeys * 128 / 16) + (ks & 3) * 2), idesc_s, ks != 0, -1);
                        mma_commit(s_full + 8 * h);
                        mbar_arrive(s_full + 8 * h);
                        if (h) {
                            mma_commit(msmem_u32(&sm.empty[k_stage]));
                            if (!two) mma_commit(msmem_u32(&sm.empty[k_stage]));       // (for the other stream too)
                            if (g + 2 == n) mma_commit(msmem_u32(&sm.q_empty[qb]));    // the queries have been used
                        }
                    }
                    __syncwarp();
                };
                const uint32_t k_full = msmem_u32(&sm.full[k_stage]), k_parity = (k_copy / C::stages) & 1u;
                bool early = false;                        // the next keys are there before these values are done with
                if (g >= 0) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {          // outputs of half a tile
                        if (!(ok = mbar_wait(p_ready + 8 * h, done & 1u, abort_flag, limit))) break;
                        if (TMA && h == 0 && n_tail && g + 1 == n) {       // (places behind the prefix hold anything, and 0 times it may be anything)
                            for (int i = lane; i < n_tail * (DP / 8); i += 32) {
                                const int r = kXKeys - 1 - i / (DP / 8), c = i % (DP / 8);
                                *reinterpret_cast<uint4*>(&sm.kv[v_stage][(c >> 3) * (kXKeys * 128) + r * 128 + (c & 7) * 16]) = make_uint4(0, 0, 0, 0);
                            }
                            fence_async_proxy();
                            __syncwarp();
                        }
                        if (elect_one()) {
                            if (!TMA) fence_async_proxy();
                            tc_after();
#pragma unroll
                            for (int ks = 0; ks < 4; ++ks)
                                mma_ts(o_at, p_at + 64 * h + ks * 8, dv + (uint64_t)((4 * h + ks) * 2048 / 16), idesc_o, g > 0 || h > 0 || ks > 0, -1);
                            mma_commit(pv_done);
                            if (h) {
                                mma_commit(msmem_u32(&sm.empty[v_stage]));
                                if (!two) mma_commit(msmem_u32(&sm.empty[v_stage]));
                            }
                        }
                        __syncwarp();
                        if (h == 0 && g + 1 < n && __all_sync(kFullMask, mbar_test(k_full, k_parity))) {
                            early = true;
                            scores(0);
                        }
                    }
                    if (!ok) break;
                }
                if (g + 1 < n) {
                    if (!early) {
                        if (!(ok = mbar_wait(k_full, k_parity, abort_flag, limit))) break;
                        scores(0);
                    }
                    scores(1);
                }
                if (!ok) break;
                if (g >= 0) { ++done; v_copy += 2 * by; }
                k_copy += 2 * by;
            }
            if (!ok) break;
            if (n == 0) {                                  // (one tile for both streams)
                if (elect_one()) mma_commit(msmem_u32(&sm.q_empty[qb]));
                __syncwarp();
                if (piece > 0 && !(ok = mbar_wait(msmem_u32(&sm.o_free), (piece - 1) & 1, abort_flag, limit))) break;
            }
            if (elect_one()) mma_commit(msmem_u32(&sm.o_done[s]));
            __syncwarp();
            tiles0 += tiles;
            ++piece;
        }
        // nothing of this block is in flight when it leaves, whatever happened
        if (elect_one()) mma_commit(msmem_u32(&sm.last[s]));
        for (int i = 0; i < 1000000 && !__all_sync(kFullMask, mbar_try(msmem_u32(&sm.last[s]), 0)); ++i) {}
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
            if (piece == 0) {
                if (two || warp < 4) copy_queries<DP>(a, pc, msmem_u32(sm.q), 32 * warp, lane);
                cp_arrive(msmem_u32(&sm.q_first));
            }
            float ref = neg_inf(), sum = 0.f;
            const int first = pc.tile + (two ? 0 : s), by = two ? 1 : 2;
#pragma unroll 1
            for (int t = first; t < pc.tile_end; t += by, ++steps) {
                const uint32_t* seen = sm.seen[(tiles0 + t - pc.tile) % kXSeen];
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {              // half a tile at a time
                    if (!mbar_wait(msmem_u32(&sm.s_full[s][h]), steps & 1u, abort_flag, limit)) { ok = false; break; }
                    tc_after();
                    uint32_t x[64];
                    tm_ld64(s_at + 64 * h, x);
                    const uint32_t see0 = seen[2 * h], see1 = seen[2 * h + 1];
                    if ((see0 & see1) != 0xffffffffu) {    // the end of the prefix, or a page that there is not
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
                    const float top = max3(m0, m1, m1) * scale;
                    const bool raise = !(top <= (ref == neg_inf() ? ref : ref + kRaise));
                    if (__any_sync(kFullMask, raise)) {
                        const float factor = raise ? ex2(ref - top) : 1.f;         // 0 where nothing has been seen before
                        if (raise) {           // (a score of NaN or +inf makes NaN of the sum, which it stays, and so of the row)
                            ref = top < -neg_inf() ? top : __int_as_float(0x7fc00000);
                            sum *= factor;
                        }
                        if (t > first || h) {
                            // the outputs before this half (those before them came before these scores, so the parity cannot be an older phase's)
                            if (!mbar_wait(msmem_u32(&sm.pv_done[s]), (2 * steps + h - 1) & 1u, abort_flag, limit)) { ok = false; break; }
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
                            e0 = ex2(e0); e1 = ex2(e1);
                            if (j % 8 == 8 - 4) ex2_pair(e2, e3);
                            else { e2 = ex2(e2); e3 = ex2(e3); }
                            add2(s0, s1, e0, e1); add2(s2, s3, e2, e3);
                            p[j / 2] = pack_bf16(e0, e1); p[j / 2 + 1] = pack_bf16(e2, e3);
                        }
                        tm_st16(s_at + 64 * h + 16 * q, p);
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
            const int c0 = two ? 0 : s * (DP / 2), c1 = two ? DP : c0 + DP / 2;
            uint4 old[4], next[4];                               // what the rows that this lane will write have of their own, two blocks of columns ahead
            const uint32_t rows_here = __ballot_sync(kFullMask, in);
            const auto fetch = [&](int c, uint4* to) {
                const int col = c + (lane & 3) * 8;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = i * 8 + (lane >> 2);
                    const int64_t at = __shfl_sync(kFullMask, out_at, r);
                    if (((rows_here >> r) & 1u) && col < a.D && c < c1) to[i] = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.out + at + col);
                    else to[i] = make_uint4(0, 0, 0, 0);
                }
            };
            float own = neg_inf();
            bool write = in;
            if (part < 0) {
                fetch(c0, old);
                fetch(c0 + 32, next);
                write = prefix_own(a, w, &own) && in;
            }
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
            f *= w_pre; g *= w_pre;
            // (of an item of one tile the second stream has no outputs: their place may hold anything, and 0 times it may be anything)
            const bool lone = !two && pc.tile_end - pc.tile == 1;
            const uint32_t o_mine = o_at + (lone ? 0 : s * DP), o_other = o_at + (lone ? 0 : (s ^ 1) * DP);
            const uint32_t rows_in = __ballot_sync(kFullMask, write);
            tc_after();
            float4 (*turn)[8] = sm.turn[warp];
#pragma unroll 1
            for (int c = c0; c < c1 && c < a.D; c += 32) {
                uint32_t u[32];
                float y[32];
                tm_ld32(o_mine + c, u);
#pragma unroll
                for (int j = 0; j < 32; ++j) y[j] = __uint_as_float(u[j]) * f;
                if (!two) {
                    tm_ld32(o_other + c, u);
#pragma unroll
                    for (int j = 0; j < 32; ++j) y[j] = fmaf(__uint_as_float(u[j]), g, y[j]);
                }
                __syncwarp();                              // the last block of columns has been read
#pragma unroll
                for (int j = 0; j < 8; ++j) turn[lane][j ^ (lane & 7)] = make_float4(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
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
                    for (int i = 0; i < 4; ++i) { now[i] = old[i]; old[i] = next[i]; }
                    fetch(c + 64, next);
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
        cp_wait_all();
    }
    tc_before();
    __syncthreads();
    tc_after();
    grid_dependency_wait();                                // (a block without work too: what follows this kernel follows the one before it)
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::tmem_cols) : "memory");
    if (sm.abort_flag) {
        if (tid == 0) {
            atomicOr(a.pages.status, (uint32_t)DBA_TREE_TIMEOUT);
            a.meta[2 * blockIdx.x] = make_int4(-2, 0, 0, 0);           // (over what the loader wrote)
        }
        if (!a.joined) {               // (else the joining kernel sees to it)
            run = XCut::run<C::threads>(a, 3, &sm.span);
            while (XCut::next(a, run, &pc))
                for (int i = tid; i < pc.rows * a.D; i += C::threads) {
                    const int r = i / a.D, d = i - r * a.D;
                    const PrefixRow w = prefix_row(a, pc.lo, pc.h, pc.row0 + r);
                    ((__nv_bfloat16*)a.out)[(int64_t)w.b * a.o_seq + (int64_t)w.i * a.o_row + (int64_t)w.head * a.o_head + d] = __float2bfloat16_rn(__int_as_float(0x7fc00000));
                    if (d == 0) a.own_lse[((int64_t)w.b * a.n + w.i) * a.H + w.head] = __int_as_float(0x7fc00000);
                }
        }
    }
}

template <int DP, bool TMA>
cudaError_t configure_prefix_mma() {
    static_assert(sizeof(XSmem<DP, TMA>) <= 227 * 1024, "a block's shared memory");
    return cudaFuncSetAttribute(tree_prefix_mma_kernel<DP, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(XSmem<DP, TMA>));
}
template <int DP, bool TMA>
cudaError_t launch_prefix_mma(const TreePrefix& a, const TreeBoxes& m, int grid, cudaStream_t st) {
    const uint32_t negate = a.scale_log2e < 0.f ? 1u << 13 : 0u;       // the scores' sign by the instruction, their size by the softmax
    return launch_after(tree_prefix_mma_kernel<DP, TMA>, dim3(grid), dim3(XConf<DP, TMA>::threads), sizeof(XSmem<DP, TMA>), st, a, m, negate);
}

}  // namespace

int tree_prefix_mma_rows() { return kXRows; }
int tree_prefix_mma_keys() { return kXKeys; }
cudaError_t configure_tree_prefix_mma() {
    cudaError_t e = configure_prefix_mma<64, true>();
    if (e == cudaSuccess) e = configure_prefix_mma<128, true>();
    if (e == cudaSuccess) e = configure_prefix_mma<64, false>();
    return e == cudaSuccess ? configure_prefix_mma<128, false>() : e;
}
cudaError_t launch_tree_prefix_mma(const TreePrefix& a, int grid, cudaStream_t st) {
    TreeBoxes m{};
    if (tree_boxes(&m, a.k, a.v, a.pages, a.K, a.D, 0))
        return a.D <= 64 ? launch_prefix_mma<64, true>(a, m, grid, st) : launch_prefix_mma<128, true>(a, m, grid, st);
    return a.D <= 64 ? launch_prefix_mma<64, false>(a, m, grid, st) : launch_prefix_mma<128, false>(a, m, grid, st);
}

}  // namespace dba
