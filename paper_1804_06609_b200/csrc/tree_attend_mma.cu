// Attention of the rows of a token tree over a paged cache on the tensor cores: bf16, head sizes up to 128.
//
// For one (sequence, key head) the rows of all its query heads are one matrix Q [rows, D], and
//     S = Q K^T (tcgen05.mma, both operands in shared memory),  P = 2^(scale log2(e) S - m),  O += P V (P from tensor memory),
// tile by tile of 64 keys, so a key and a value leave HBM once per 128 rows however many hypotheses read them.
//
// A block is one stream of tiles (its run of the work, see tree_device.cuh).  Two blocks share an SM (four where one softmax warp
// serves heads of up to 64): so many hold their 256 or 128 columns of tensor memory and their shared memory, and the steps of
// one, load -> S -> P -> O, fall into the gaps of the others.  Every role walks its warp in step; SW softmax warps:
//   softmax    thread = row = lane of tensor memory.  Reads the row's 64 scores, keeps a reference m and the sum of the
//              exponentials in fp32, writes P over the scores (bf16, as the matrix instruction needs it: half a unit in the 8th
//              bit of every probability; the sum is taken before the rounding).  m is only raised when the tile's maximum
//              is more than 2^8 above it; then the row's O is rescaled in tensor memory.  Quotients are unaffected.
//   products   one lane issues the matrix instructions; with two S in tensor memory, a tile's scores before the outputs of the
//              tile before it.
//   inspector  values that are not finite would reach all rows of the tile through 0 * inf: in arena tiles (the only ones
//              that rows see differently) it looks the values over, puts zeros in their place and says so; the rows that do
//              see such a slot add it at the end.  (With one softmax warp the products' warp does it.)
//   loaders    two warps: walk the run and tell the others its pieces; 16-byte cp.async with zero fill, every place looked up
//              in the page table by itself, so pages of any size may end inside a tile (a tensor map's box could not); written
//              in the 128-byte swizzle both operand forms want: keys K-major, values MN-major ([key][d] either way).  Rows
//              that do not exist, or that no row of the sequence sees, are zeros.
// Every wait on an mbarrier is bounded: one that runs out winds the block down and marks the call as failed.
//
// What bounds it, measured (6551 GB/s is what a copy reaches; times of calls among others, then of six calls at a time, whose clocks
// are higher): with few rows and long contexts HBM: one row, 32 heads over 4 key heads of 128, 4 x up to 131071 tokens, 1.03 GB:
// 176 to 186 us (5.5 to 5.9 TB/s), 168.  With many rows the two longest chains of a tile, which take about as long: the loader's
// instructions (2000 to 2600 cycles; dropping the exponentials, or most of the products, or reading everything from L2,
// each changes under 3 %) and the softmax warps' (2600): 61 rows, 32 heads over 8 of 128, 8 x up to 8189 tokens: 122 us, 110, of
// which 10 join the pieces; 37 would do.  Two softmax threads to a row were 158 us when they were tried: a thread that holds
// 64 scores takes 128 registers, and the SM has 65536.  Many short items (256 x 16 heads of 64, 20 rows, 30 to 160 keys):
// what an item costs from its look-up to its output, 41 us; 15 would do.
#include <cuda_bf16.h>

#include "tree_device.cuh"
#include "tree_mma.cuh"

namespace dba {

namespace {

constexpr int kMKeys = 64;                  // keys of a tile
constexpr int kLoadWarps = 2, kLoadThreads = 32 * kLoadWarps;
constexpr int kSeen = 8;               // more than the tiles the loader may be ahead by
constexpr int kItemUnits = 2;               // what an item costs beside its tiles, in tiles (see tree_device.cuh)
constexpr uint32_t kNoRow = 0xffffffffu;
constexpr int kPieces = 4;                  // pieces the loader may be ahead by

// SW softmax warps; an item is a block of rows of HP key heads.
//   <DP, 4, 1>  up to 128 rows of one key head
//   <64, 4, 4>  up to 32 rows of each of four neighbouring key heads, a softmax warp to each.  Four products per tile, each of
//               which writes the quarter of the lanes that is its head's.  The four share what a tile costs beside its
//               bytes: its look-ups, masks and the way through the roles.
//   <DP, 1, 1>  up to 32 rows of one key head, where there are not four to take.  The other 96 rows of the products are what
//               lies around the queries in shared memory, and nobody reads their results.
template <int DP, int SW, int HP> struct MConf {
    static constexpr int rows = 32 * SW / HP;                        // of a key head
    static constexpr int inspectors = SW == 4 ? 1 : 0;               // with one softmax warp the products' warp looks values over itself
    static constexpr int threads = 32 * (SW + 1 + inspectors + kLoadWarps);
    static constexpr int stages = HP == 4 ? 3 : DP == 128 ? (SW == 1 ? 6 : 5) : SW == 1 ? 5 : 9;      // tiles of keys or values in shared memory
    static constexpr int head_bytes = kMKeys * DP * 2, stage_bytes = HP * head_bytes;
    static constexpr int q_half = 32 * SW * 128;                     // 64 columns of the queries
    static constexpr int q_bytes = 32 * SW * DP * 2;
    static constexpr int q_bufs = SW == 1 || (DP == 64 && HP == 1) ? 2 : 1;
    static constexpr int s_bufs = DP == 64 && SW == 1 ? 1 : 2;
    static constexpr int blocks_per_sm = DP == 64 && SW == 1 ? 4 : 2;
    static constexpr int tmem_cols = s_bufs == 1 ? 128 : 256;
    static constexpr int o_col = 0, s_col = DP;
    // stages that lie before the queries: with one softmax warp the products' other rows are read up to 96 rows before and
    // after the queries
    static constexpr int pre = SW == 1 ? (DP == 64 ? 2 : 1) : 0;
    static constexpr int q_at = pre * stage_bytes;
    static constexpr int tile_bytes = stages * stage_bytes + q_bufs * q_bytes;
    static_assert(SW > 1 || (q_at >= 96 * 128 && q_at + q_bufs * q_bytes - q_half + kMRows * 128 <= tile_bytes), "rows beside the queries");
    // where a stage of keys or values lies
    static __device__ __forceinline__ uint32_t stage_at(uint32_t s) { return s * stage_bytes + (pre == 0 || (int)s >= pre ? q_bufs * q_bytes : 0); }
};

template <int DP, int SW, int HP> struct MSmem {
    using C = MConf<DP, SW, HP>;
    alignas(1024) unsigned char tiles[C::tile_bytes];       // keys, values and queries
    uint64_t full[C::stages], empty[C::stages], landed[C::inspectors ? C::stages : 1];
    uint64_t s_full[C::s_bufs], p_ready[C::s_bufs];
    uint64_t q_empty[C::q_bufs];
    uint64_t pv_done, o_free, told, last;
    uint64_t published[kPieces], released[kPieces];
    int4 piece[kPieces][2];                 // (in turn) what the loader tells the others of a piece
    uint32_t seen[kSeen][kLoadWarps];   // places of the tile that exist (by tile, in turn)
    uint32_t bad[kPieces];                // (by piece, in turn) 1 + the last piece that had a value that is not finite in an arena tile
    uint32_t tmem_base;
    int abort_flag, turn, scheduler[4];
    union {
        TreeRunShared run;                  // (until the roles begin)
        uint32_t rows[2][kMKeys];           // the last two tiles' rows in the cache, in 16 bytes; kNoRow: none
    };
};

// a word whose bf16 halves that are not finite are zeroed
__device__ __forceinline__ uint32_t only_finite(uint32_t x) {
    if ((x & 0x00007f80u) == 0x00007f80u) x &= 0xffff0000u;
    if ((x & 0x7f800000u) == 0x7f800000u) x &= 0x0000ffffu;
    return x;
}
// bits that show whether a bf16 half of a word is not finite (its exponent is all ones)
__device__ __forceinline__ uint32_t not_finite(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
// Looks a stage of an arena tile's values over (a warp in step): halves that are not finite become zeros.  They are rare:
// loads go eight at a time, and are gone through again only where something was found.
template <int BYTES>
__device__ __forceinline__ bool look_over(unsigned char* stage, int lane) {
    uint4* const mine = reinterpret_cast<uint4*>(stage) + lane;
    uint32_t seen = 0;
#pragma unroll 1
    for (int i = 0; i < BYTES / 16; i += 8 * 32) {
        uint4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = mine[i + 32 * k];
#pragma unroll
        for (int k = 0; k < 8; ++k) seen |= not_finite(x[k].x) | not_finite(x[k].y) | not_finite(x[k].z) | not_finite(x[k].w);
    }
    if (!__any_sync(kFullMask, seen != 0)) return false;
#pragma unroll 1
    for (int i = 0; i < BYTES / 16; i += 32) {
        uint4 x = mine[i];
        x.x = only_finite(x.x); x.y = only_finite(x.y); x.z = only_finite(x.z); x.w = only_finite(x.w);
        mine[i] = x;
    }
    return true;
}

// The outputs of an item whose block gave up.
template <int HP>
__device__ __noinline__ void undo_item(const TreeAttend& a, TreePiece pc, int item_rows) {
    const int M = a.n * a.G, rows = min(item_rows, M - pc.rb * item_rows);
    for (int i = threadIdx.x; i < HP * rows * a.D; i += blockDim.x) {
        const int r = i / a.D, d = i - r * a.D, w = r / rows, rr = pc.rb * item_rows + r - w * rows, tok = rr / a.G;
        const int head = (pc.h * HP + w) * a.G + rr - tok * a.G;
        ((__nv_bfloat16*)a.out)[(int64_t)pc.b * a.o_seq + (int64_t)tok * a.o_row + (int64_t)head * a.o_head + d] = __float2bfloat16_rn(__int_as_float(0x7fc00000));
        if (a.lse && d == 0) a.lse[((int64_t)pc.b * a.n + tok) * a.H + head] = __int_as_float(0x7fc00000);
    }
}

template <int DP, int SW, int HP>
__global__ void __launch_bounds__(MConf<DP, SW, HP>::threads, MConf<DP, SW, HP>::blocks_per_sm) tree_attend_mma_kernel(const __grid_constant__ TreeAttend a, const uint32_t negate) {
    using C = MConf<DP, SW, HP>;
    extern __shared__ __align__(1024) unsigned char mraw[];
    MSmem<DP, SW, HP>& sm = *reinterpret_cast<MSmem<DP, SW, HP>*>(mraw);
    const int tid = threadIdx.x, lane = tid & 31;
    volatile int* abort_flag = &sm.abort_flag;
    const long long limit = a.wait_clocks > 0 ? a.wait_clocks : kMWaitClocks;
    const int M = a.n * a.G, row_blocks = (M + C::rows - 1) / C::rows, groups = a.K / HP;

    if (tid == 0) {
        for (int s = 0; s < C::stages; ++s) { mbar_init(msmem_u32(&sm.full[s]), kLoadThreads + kLoadWarps); mbar_init(msmem_u32(&sm.empty[s]), 1); if (C::inspectors) mbar_init(msmem_u32(&sm.landed[s]), kLoadThreads); }
        // (s_full counts the product and, beside it, an arrival of the issuing thread, which passes on what the loader wrote
        // before it; `told` does that once a piece for its values, and its product is the piece's last, so all its outputs are
        // there.  pv_done, a phase to a tile, does not show that: the last two outputs may be issued together, and a wait for
        // a phase's parity passes while the phase before it is still open.  It serves rows that raise their reference, whose
        // tile's scores came after the outputs of two tiles before)
        for (int s = 0; s < C::s_bufs; ++s) { mbar_init(msmem_u32(&sm.s_full[s]), 2); mbar_init(msmem_u32(&sm.p_ready[s]), SW); }
        for (int s = 0; s < C::q_bufs; ++s) mbar_init(msmem_u32(&sm.q_empty[s]), 1);
        mbar_init(msmem_u32(&sm.pv_done), 1); mbar_init(msmem_u32(&sm.told), 2); mbar_init(msmem_u32(&sm.o_free), SW);
        mbar_init(msmem_u32(&sm.last), 1);
        for (int i = 0; i < kPieces; ++i) { mbar_init(msmem_u32(&sm.published[i]), 1); mbar_init(msmem_u32(&sm.released[i]), SW + 1 + C::inspectors); }
        for (int i = 0; i < kPieces; ++i) sm.bad[i] = 0;
        sm.abort_flag = 0;
        if (SW == 1) {
            uint32_t sm_id;
            asm volatile("mov.u32 %0, %smid;" : "=r"(sm_id));
            sm.turn = (int)(atomicAdd(a.turns + sm_id % kTreeTurns, 1u) & 3u);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (SW == 1 && lane == 0) {
        uint32_t slot;
        asm volatile("mov.u32 %0, %warpid;" : "=r"(slot));
        sm.scheduler[tid >> 5] = (int)(slot & 3u);
    }
    __syncthreads();
    // The warp's role: 0 .. SW-1 softmax, SW products, then the loaders.  A warp reaches the quarter of the tensor memory's lanes
    // that its number modulo 4 names, and issues from the scheduler of that number.  With one softmax warp to a block of
    // four warps, the blocks of an SM take turns, so that their softmax warps do not share a scheduler.
    int quarter = 0;
    if (SW == 1) {
#pragma unroll
        for (int w = 0; w < 4; ++w) if (sm.scheduler[w] == sm.turn) quarter = w;
    }
    const int warp = SW == 1 ? ((tid >> 5) + 4 - quarter) & 3 : tid >> 5;
    if (warp == SW) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(msmem_u32(&sm.tmem_base)), "r"(C::tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    grid_dependency_wait();
    allow_dependents();
    TreeRun run = tree_run<C::threads>(a, kMKeys, groups * row_blocks, kItemUnits, 1, &sm.run);      // (has the block's barriers)
    __syncthreads();           // its numbers have been read: their place is used again
    tc_after();
    const uint32_t tmem = sm.tmem_base;
    if (warp > SW + C::inspectors) {
        // ------------------------------------------------------------------ loader: warp lw has rows 32 lw .. 32 lw + 31 of a tile
        constexpr int CH = DP / 8;                     // 16-byte chunks of a row
        constexpr int RW = 32 / CH, NJ = 32 / RW;      // rows the warp copies at a time, and how often
        const int lw = warp - SW - C::inspectors - 1, ch = lane % CH, sub = lane / CH;
        const bool ch_in = ch * 8 < a.D;
        const uint32_t tiles = msmem_u32(sm.tiles);
        const int64_t head2 = 2 * a.pages.head_stride;          // bytes from a key head to the next
        // this lane's place in rows sub, sub + RW, ..: the swizzle moves a chunk by the row's last three bits
        const uint32_t in_kv = (uint32_t)(ch >> 3) * (kMKeys * 128) + (uint32_t)(lw * 32 + sub) * 128;
        const uint32_t swz = ((uint32_t)(ch & 7) ^ (uint32_t)sub) << 4;
        const int64_t page16 = a.pages.page_stride / 8, token16 = a.pages.token_stride / 8;        // rows in 16 bytes
        int step = 0;
        uint32_t stage = 0, phase = 1;                 // of the next copy (a barrier's first wait does not wait)
        // The loader walks the pieces of the run and tells the others.  Tiles are looked up one ahead of the one being copied:
        // numbers, masks and page entries come out of the L2.
        TreePiece pc, nx;
        int piece = -1, tile_no = 0, t = 0, f_row = 0, f_id = 0;
        bool f_arena = false, f_in = false, ok = true;
        uint32_t f_m0 = 0, f_m1 = 0;
        pc.tile = pc.tiles = pc.top = pc.ctx = pc.b = pc.h = pc.rb = pc.arena_tiles = pc.slot = 0; pc.whole = false;
#pragma unroll 1
        for (;;) {
            // --- the tile looked up last
            const int c_row = f_row, c_id = f_id, c_t = t;
            const bool c_arena = f_arena;
            bool c_in = f_in;
            const uint32_t c_any = f_m0 | f_m1;
            const bool last = c_t + 1 == pc.tile + pc.tiles;
            bool more = true;
            // --- look the next one up: of this piece, or the first of the next
            if (piece < 0 || last) {
                more = tree_next_piece(a, run, kMKeys, groups, row_blocks, kItemUnits, piece < 0, &nx);
                if (piece < 0 && lw == 0 && lane == 0) tree_write_meta(a, run, more ? &nx : nullptr, row_blocks, kItemUnits);
                t = nx.tile;
            } else { nx = pc; t = c_t + 1; }
            if (more) {
                int place, count;
                tree_tile_span(a, nx, t, kMKeys, &place, &count);
                f_arena = t < nx.arena_tiles;
                f_in = lw * 32 + lane < count;
                f_m0 = f_m1 = 0;
                if (f_arena) {
                    const int w = (place >> 5) + lw;
                    const uint32_t* mk = a.masks + (int64_t)nx.b * a.n * a.W + w;
                    if (w < a.W) {
                        if (lane < a.n) f_m0 = __ldg(mk + lane * a.W);
                        if (lane + 32 < a.n) f_m1 = __ldg(mk + (lane + 32) * a.W);
                    }
                }
                const uint32_t at = (uint32_t)(place + lw * 32 + lane), page = tree_page(a.pages, at);
                f_row = (int)(at - page * (uint32_t)a.pages.page_size);
                f_in = f_in && page < (uint32_t)a.pages.max_pages;
                f_id = f_in ? __ldg(a.pages.table + (int64_t)nx.b * a.pages.table_stride + page) : 0;
            }
            if (piece >= 0) {
                const uint32_t qb = (uint32_t)piece % C::q_bufs;
                if (c_t == pc.tile) {                  // a new piece: the others are told, and its item's queries fetched
                    if (lw == 0 && piece >= kPieces && !mbar_wait(msmem_u32(&sm.released[piece % kPieces]), (piece / kPieces - 1) & 1, abort_flag, limit)) { ok = false; break; }
                    if (lw == 0 && lane == 0) {
                        sm.piece[piece % kPieces][0] = make_int4(pc.b, pc.h, pc.rb, pc.top);
                        sm.piece[piece % kPieces][1] = make_int4(pc.tile, pc.tiles, pc.arena_tiles, pc.slot | (pc.whole ? 2 : 0));
                        mbar_arrive(msmem_u32(&sm.published[piece % kPieces]));
                    }
                    if (piece >= C::q_bufs && !mbar_wait(msmem_u32(&sm.q_empty[qb]), ((uint32_t)piece / C::q_bufs - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                    // beyond the rows and the head size, zeros
                    const int rows_here = min(C::rows, M - pc.rb * C::rows);
                    const char* q = (const char*)a.q + 2 * ((int64_t)pc.b * a.q_seq + (int64_t)pc.h * HP * a.G * a.q_head) + (ch_in ? ch * 16 : 0);
                    const uint32_t dst = tiles + C::q_at + qb * C::q_bytes + (uint32_t)(ch >> 3) * C::q_half + (uint32_t)sub * 128;
#pragma unroll 1
                    for (int r0 = 0; r0 < rows_here; r0 += 32) {      // a lane finds one row, and every lane copies chunks of all
                        const int rr = min(pc.rb * C::rows + r0 + lane, M - 1), tok = a.G == 1 ? rr : rr / a.G;
                        const int64_t mine = 2 * ((int64_t)tok * a.q_row + (int64_t)(rr - tok * a.G) * a.q_head);
                        const int left = ch_in ? rows_here - r0 - sub : 0;
#pragma unroll 2
                        for (int j = lw; j < NJ; j += kLoadWarps) {
                            const char* from = q + __shfl_sync(kFullMask, mine, j * RW + sub);
                            const uint32_t bytes = j * RW < left ? 16u : 0u;
                            const uint32_t to = dst + (r0 + j * RW) * 128 + (swz ^ (uint32_t)((j * RW & 7) << 4));
#pragma unroll
                            for (int w = 0; w < HP; ++w) cp_async16(to + w * 32 * 128, from + 2 * (int64_t)(w * a.G) * a.q_head, bytes);
                        }
                    }                                   // (the first keys' arrival counts them too)
                }
                // --- where its rows are
                if (c_arena) {                          // slots no row of the sequence sees are not read
                    const uint32_t any = __reduce_or_sync(kFullMask, c_any);
                    c_in = c_in && ((any >> lane) & 1u);
                }
                if (c_in && (uint32_t)c_id >= (uint32_t)a.pages.num_pages) {
                    atomicOr(a.pages.status, (uint32_t)DBA_TREE_BAD_PAGE);
                    c_in = false;
                }
                const uint32_t there = __ballot_sync(kFullMask, c_in);
                if (lane == 0) sm.seen[tile_no % kSeen][lw] = there;
                const bool whole = there == 0xffffffffu && a.D == DP;       // every byte of the warp's rows is there to be copied
                // (the host has seen to it that a layer's rows are within 2^32 times 16 bytes)
                sm.rows[tile_no & 1][lw * 32 + lane] = c_in ? (uint32_t)((int64_t)c_id * page16 + (int64_t)c_row * token16) : kNoRow;
                __syncwarp();
                // --- copies: the keys and the values, into two stages.  A stage is handed on by the copies themselves; the
                // issuing thread of the matrix products has the fence between their writes and its reads (here it would wait
                // for every copy in flight: twice the time on long contexts).  Values of an arena tile go through the
                // inspector first.
                const bool look = c_arena && C::inspectors;
                const uint32_t* rows = &sm.rows[tile_no & 1][lw * 32 + sub];
                uint32_t at[NJ];
#pragma unroll
                for (int j = 0; j < NJ; ++j) at[j] = rows[j * RW];
                const int64_t head_at = pc.h * HP * head2 + (ch_in ? ch * 16 : 0);
                // With one head the two go side by side, so that a warp waits for the steps of one address at a time half as
                // often (a tree of 61 rows over 8189 tokens, heads of 128, in short runs: 107 us, one after the other 114); with four, one
                // after the other, as either may begin when its own stage is free and there are only three.
                constexpr int SIDE = HP == 1 ? 2 : 1;
#pragma unroll 1
                for (int k = 0; k < 2; k += SIDE) {
                    uint32_t st[SIDE], dst[SIDE];
                    const char* base[SIDE];
#pragma unroll
                    for (int i = 0; i < SIDE; ++i) {
                        if (ok) ok = mbar_wait(msmem_u32(&sm.empty[stage]), phase, abort_flag, limit);
                        st[i] = stage; dst[i] = tiles + C::stage_at(stage) + in_kv;
                        base[i] = (const char*)(k + i == 0 ? a.k : a.v) + head_at;
                        if (++stage == C::stages) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
                    if (HP == 1 && whole) {
#pragma unroll
                        for (int j = 0; j < NJ; ++j) {
                            const uint32_t to = j * RW * 128 + (swz ^ (uint32_t)((j * RW & 7) << 4));
#pragma unroll
                            for (int i = 0; i < SIDE; ++i) cp_async16(dst[i] + to, base[i] + (uint64_t)at[j] * 16, 16u);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < NJ; ++j) {
                            const uint32_t bytes = at[j] != kNoRow && ch_in ? 16u : 0u;
                            const uint64_t from = (uint64_t)(at[j] != kNoRow ? at[j] : 0u) * 16;
                            const uint32_t to = j * RW * 128 + (swz ^ (uint32_t)((j * RW & 7) << 4));
#pragma unroll
                            for (int i = 0; i < SIDE; ++i)
#pragma unroll
                                for (int w = 0; w < HP; ++w) cp_async16(dst[i] + to + w * C::head_bytes, base[i] + from + w * head2, bytes);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < SIDE; ++i) {
                        if (lane == 0) mbar_arrive(msmem_u32(&sm.full[st[i]]));      // (for what this warp wrote beside the copies)
                        if (step != a.drop_item) cp_arrive(msmem_u32(look && k + i == 1 ? &sm.landed[C::inspectors ? st[i] : 0] : &sm.full[st[i]]));
                        ++step;
                    }
                }
                if (!ok) break;
                ++tile_no;
            }
            if (!more) break;
            if (piece < 0 || last) ++piece;
            pc = nx;
        }
        ++piece;
        if (ok && lw == 0 &&                            // the end of the run
            (piece < kPieces || mbar_wait(msmem_u32(&sm.released[piece % kPieces]), (piece / kPieces - 1) & 1, abort_flag, limit)) && lane == 0) {
            sm.piece[piece % kPieces][1] = make_int4(0, 0, 0, 0);
            mbar_arrive(msmem_u32(&sm.published[piece % kPieces]));
        }
        cp_wait_all();
    } else if (warp == SW) {
        // ------------------------------------------------------------------ matrix products: the warp walks in step, one lane issues
        constexpr uint32_t idesc_s = mma_idesc(kMKeys, false), idesc_o = mma_idesc(DP, true);
        const uint32_t tiles = msmem_u32(sm.tiles), q0 = tiles + C::q_at - quarter * (32 * 128);      // the queries are the lanes from 32 quarter on
        uint32_t stage = 0, phase = 0, v_stage = 1, v_phase = 0;      // of the next keys and the next values, two copies on each time
        int piece = 0;
        bool ok = true;
        auto next_stage = [&](uint32_t& st, uint32_t& ph) { st += 2; if (st >= C::stages) { st -= C::stages; ph ^= 1u; } };
        constexpr int LAG = C::s_bufs - 1;             // one S in tensor memory: S0 O0 S1 O1 ..;  two: S0 S1 O0 S2 O1 ..
        uint32_t n_s = 0, n_o = 0;                     // tiles whose scores, and whose outputs, have been issued
#pragma unroll 1
        for (;; ++piece) {
            if (!mbar_wait(msmem_u32(&sm.published[piece % kPieces]), (piece / kPieces) & 1, abort_flag, limit)) break;
            const int4 i1 = sm.piece[piece % kPieces][1];
            const int n_tiles = i1.y;
            if (n_tiles == 0) break;
            const uint32_t qb = (uint32_t)piece % C::q_bufs;
#pragma unroll 1
            for (int t = 0; t < n_tiles + LAG; ++t) {
                if (t < n_tiles) {
                    if (!(ok = mbar_wait(msmem_u32(&sm.full[stage]), phase, abort_flag, limit))) break;
                    const uint32_t sb = n_s % C::s_bufs;
                    const uint64_t dq = sw128_desc(q0 + qb * C::q_bytes, 16), dk = sw128_desc(tiles + C::stage_at(stage), 16);
                    const uint32_t d = tmem + C::s_col + sb * kMKeys;
                    if (elect_one()) {
                        fence_async_proxy();           // the copies' writes (generic) before the products' reads
                        tc_after();
#pragma unroll
                        for (int w = 0; w < HP; ++w)
#pragma unroll
                            for (int ks = 0; ks < DP / 16; ++ks)      // 16 dimensions = 32 bytes along a swizzled row; 64 to a block of columns (zeros beyond the head size)
                                mma_ss(d, dq + (uint64_t)((ks >> 2) * (C::q_half / 16) + (ks & 3) * 2),
                                       dk + (uint64_t)((w * C::head_bytes + (ks >> 2) * (kMKeys * 128)) / 16 + (ks & 3) * 2), idesc_s | negate, ks != 0, HP > 1 ? w : -1);
                        mma_commit(msmem_u32(&sm.empty[stage]));
                        mma_commit(msmem_u32(&sm.s_full[sb]));
                        mbar_arrive(msmem_u32(&sm.s_full[sb]));
                        if (t + 1 == n_tiles) mma_commit(msmem_u32(&sm.q_empty[qb]));
                    }
                    __syncwarp();
                    ++n_s;
                    next_stage(stage, phase);
                }
                if (t >= LAG) {
                    const int of = t - LAG;
                    const uint32_t sb = n_o % C::s_bufs;
                    if (!(ok = mbar_wait(msmem_u32(&sm.full[v_stage]), v_phase, abort_flag, limit))) break;
                    if (!C::inspectors && i1.x + of < i1.z && look_over<C::stage_bytes>(sm.tiles + C::stage_at(v_stage), lane)) {
                        if (lane == 0) sm.bad[piece % kPieces] = (uint32_t)piece + 1;
                        __syncwarp();
                    }
                    if (!(ok = mbar_wait(msmem_u32(&sm.p_ready[sb]), (n_o / C::s_bufs) & 1u, abort_flag, limit))) break;
                    if (of == 0 && piece > 0 && !(ok = mbar_wait(msmem_u32(&sm.o_free), (piece - 1) & 1u, abort_flag, limit))) break;
                    const uint64_t dv = sw128_desc(tiles + C::stage_at(v_stage), kMKeys * 128);
                    const uint32_t p = tmem + C::s_col + sb * kMKeys;
                    if (elect_one()) {
                        fence_async_proxy();
                        tc_after();
#pragma unroll
                        for (int w = 0; w < HP; ++w)
#pragma unroll
                            for (int ks = 0; ks < kMKeys / 16; ++ks)  // 16 keys = two groups of eight rows of 128 bytes
                                mma_ts(tmem + C::o_col, p + ks * 8, dv + (uint64_t)((w * C::head_bytes + ks * 2048) / 16), idesc_o, (of | ks) != 0, HP > 1 ? w : -1);
                        mma_commit(msmem_u32(&sm.empty[v_stage]));
                        mma_commit(msmem_u32(&sm.pv_done));
                        if (of + 1 == n_tiles) { mma_commit(msmem_u32(&sm.told)); mbar_arrive(msmem_u32(&sm.told)); }
                    }
                    __syncwarp();
                    ++n_o;
                    next_stage(v_stage, v_phase);
                }
            }
            if (!ok) break;
            if (lane == 0) mbar_arrive(msmem_u32(&sm.released[piece % kPieces]));
        }
        // nothing of this block is in flight when it leaves, whatever happened
        if (elect_one()) mma_commit(msmem_u32(&sm.last));
        for (int i = 0; i < 1000000 && !__all_sync(kFullMask, mbar_try(msmem_u32(&sm.last), 0)); ++i) {}
    } else if (C::inspectors && warp == SW + 1) {
        // ------------------------------------------------------------------ inspector: values of arena tiles
        uint32_t stage = 0;
        uint32_t uses[C::stages];                      // how often each stage has held values to be looked over
#pragma unroll
        for (int i = 0; i < C::stages; ++i) uses[i] = 0;
        for (int piece = 0;; ++piece) {
            if (!mbar_wait(msmem_u32(&sm.published[piece % kPieces]), (piece / kPieces) & 1, abort_flag, limit)) break;
            const int4 i1 = sm.piece[piece % kPieces][1];
            if (i1.y == 0) break;
            const int n_arena = min(i1.y, max(0, i1.z - i1.x));      // its first so many tiles are of the arena
            const uint32_t begin = stage;
            bool ok = true;
            for (int t = 0; t < n_arena && ok; ++t) {
                const uint32_t s = (begin + 2u * (uint32_t)t + 1u) % C::stages;      // copies go K0 V0 K1 V1 ..
                uint32_t use = 0;
#pragma unroll
                for (int i = 0; i < C::stages; ++i) if (i == (int)s) use = uses[i]++;
                if (!(ok = mbar_wait(msmem_u32(&sm.landed[s]), use & 1u, abort_flag, limit))) break;
                if (look_over<C::stage_bytes>(sm.tiles + C::stage_at(s), lane) && lane == 0) sm.bad[piece % kPieces] = (uint32_t)piece + 1;
                __syncwarp();
                if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(msmem_u32(&sm.full[s])), "r"((uint32_t)kLoadThreads) : "memory");
            }
            if (!ok) break;
            if (lane == 0) mbar_arrive(msmem_u32(&sm.released[piece % kPieces]));
            stage = (begin + 2u * (uint32_t)i1.y) % C::stages;
        }
    } else {
        // ------------------------------------------------------------------ softmax: a row per thread
        const uint32_t lanes = (uint32_t)((SW == 1 ? quarter : warp) * 32) << 16;
        const float scale = fabsf(a.scale_log2e);
        const int row = warp * 32 + lane;
        bool ok = true;
        int piece = 0;
        uint32_t g = 0;
        while (ok) {
            if (!mbar_wait(msmem_u32(&sm.published[piece % kPieces]), (piece / kPieces) & 1, abort_flag, limit)) { ok = false; break; }
            const int4 i0 = sm.piece[piece % kPieces][0], i1 = sm.piece[piece % kPieces][1];
            if (i1.y == 0) break;
            const int p_b = i0.x, p_top = i0.w, p_tile = i1.x, p_end = i1.x + i1.y, p_arena = i1.z;
            const int rr = i0.z * C::rows + (HP > 1 ? lane : row);
            const bool active = HP > 1 || i0.z * C::rows + warp * 32 < M;       // the warp has rows
            const int tok = min(rr, M - 1) / a.G;
            // the row's mask words of the tile to come
            const uint32_t* mask = a.masks ? a.masks + ((int64_t)p_b * a.n + tok) * a.W : nullptr;
            uint32_t next0 = 0, next1 = 0;
            auto fetch_mask = [&](int t) {
                if (t < p_arena) {
                    next0 = __ldg(mask + 2 * t);
                    next1 = 2 * t + 1 < a.W ? __ldg(mask + 2 * t + 1) : 0u;
                }
            };
            fetch_mask(p_tile);
            uint32_t any = a.masks ? 0u : 1u;                         // an empty mask closes the row: its words, as the tiles come by
            if (a.masks)
                for (int w = 0; w < min(2 * p_tile, (p_top + 31) / 32); ++w) any |= __ldg(mask + w);      // (those before a piece that begins inside)
            float ref = neg_inf(), sum = 0.f;
#pragma unroll 1
            for (int t = p_tile; t < p_end; ++t, ++g) {
                const uint32_t sb = g % C::s_bufs;
                uint32_t see0, see1;
                if (t < p_arena) { see0 = next0; see1 = next1; any |= see0 | see1; }
                else see0 = see1 = any ? 0xffffffffu : 0u;
                if (rr >= M) see0 = see1 = 0;
                if (t + 1 < p_end) fetch_mask(t + 1);
                if (!mbar_wait(msmem_u32(&sm.s_full[sb]), (g / C::s_bufs) & 1u, abort_flag, limit)) { ok = false; break; }
                if (active) {
                    tc_after();
                    see0 &= sm.seen[g % kSeen][0]; see1 &= sm.seen[g % kSeen][1];
                    // 32 columns at a time; where no row of the warp sees any of them (the end of the arena or of the context), none
                    const bool half[2] = {__any_sync(kFullMask, see0 != 0) != 0, __any_sync(kFullMask, see1 != 0) != 0};
                    uint32_t u[kMKeys];
                    tm_ld64(tmem + lanes + C::s_col + sb * kMKeys, u);
                    float m0 = neg_inf(), m1 = m0, m2 = m0, m3 = m0;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (!half[h]) continue;
                        const uint32_t see = h ? see1 : see0;
                        uint32_t* x = u + 32 * h;
                        if (__any_sync(kFullMask, see != 0xffffffffu)) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) if (!(see & (1u << j))) x[j] = 0xff800000u;
                        }
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            m0 = fmaxf(m0, __uint_as_float(x[j])); m1 = fmaxf(m1, __uint_as_float(x[j + 1]));
                            m2 = fmaxf(m2, __uint_as_float(x[j + 2])); m3 = fmaxf(m3, __uint_as_float(x[j + 3]));
                        }
                    }
                    const float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * scale;
                    const bool raise = top > (ref == neg_inf() ? ref : ref + kRaise);
                    if (__any_sync(kFullMask, raise)) {
                        const float factor = raise ? ex2(ref - top) : 1.f;             // 0 where nothing has been seen before
                        if (raise) { ref = top; sum *= factor; }
                        if (t > p_tile) {
                            if (!mbar_wait(msmem_u32(&sm.pv_done), (g - 1) & 1u, abort_flag, limit)) { ok = false; break; }
                            tc_after();
#pragma unroll 1
                            for (int c = 0; c < DP; c += 16) {
                                uint32_t o[16];
                                tm_ld16(tmem + lanes + C::o_col + c, o);
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * factor);
                                tm_st16(tmem + lanes + C::o_col + c, o);
                            }
                        }
                    }
                    const float shift = ref == neg_inf() ? 0.f : -ref;
                    float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t p[16];
                        if (half[h]) {
                            const uint32_t* x = u + 32 * h;
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {
                                float e0, e1, e2, e3;
                                fma2(e0, e1, __uint_as_float(x[j]), __uint_as_float(x[j + 1]), scale, shift);
                                fma2(e2, e3, __uint_as_float(x[j + 2]), __uint_as_float(x[j + 3]), scale, shift);
                                e0 = ex2(e0); e1 = ex2(e1); e2 = ex2(e2); e3 = ex2(e3);
                                add2(s0, s1, e0, e1); add2(s2, s3, e2, e3);
                                p[j / 2] = pack_bf16(e0, e1); p[j / 2 + 1] = pack_bf16(e2, e3);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j) p[j] = 0;
                        }
                        tm_st16(tmem + lanes + C::s_col + sb * kMKeys + 16 * h, p);
                    }
                    sum += (s0 + s1) + (s2 + s3);
                    tm_wait_st();
                    tc_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(msmem_u32(&sm.p_ready[sb]));
            }
            if (!ok) break;
            if (!mbar_wait(msmem_u32(&sm.told), piece & 1, abort_flag, limit)) { ok = false; break; }
            if (active) {
                tc_after();
                const bool bad = sm.bad[piece % kPieces] == (uint32_t)piece + 1;
                const bool whole = i1.w & 2;
                const float inv = !(sum > 0.f) ? 0.f : whole ? __frcp_rn(sum) : 1.f;
                const int p_h = sm.piece[piece % kPieces][0].y * HP + (HP > 1 ? warp : 0), head = p_h * a.G + rr - tok * a.G;
                const int64_t part = (int64_t)(2 * blockIdx.x + (i1.w & 1)) * (32 * SW) + row;
                __nv_bfloat16* out = (__nv_bfloat16*)a.out + (int64_t)p_b * a.o_seq + (int64_t)tok * a.o_row + (int64_t)head * a.o_head;
#pragma unroll 1
                for (int c = 0; c < DP; c += 32) {
                    uint32_t u[32];
                    tm_ld32(tmem + lanes + C::o_col + c, u);
#pragma unroll
                    for (int j = 0; j < 32; ++j) u[j] = sum == 0.f ? 0u : __float_as_uint(__uint_as_float(u[j]) * inv);      // (a closed row's O may hold anything)
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        const bool in = rr < M && c + j < a.D;
                        if (whole) {
                            uint4 w;
                            w.x = pack_bf16(__uint_as_float(u[j]), __uint_as_float(u[j + 1])); w.y = pack_bf16(__uint_as_float(u[j + 2]), __uint_as_float(u[j + 3]));
                            w.z = pack_bf16(__uint_as_float(u[j + 4]), __uint_as_float(u[j + 5])); w.w = pack_bf16(__uint_as_float(u[j + 6]), __uint_as_float(u[j + 7]));
                            if (in) *reinterpret_cast<uint4*>(out + c + j) = w;
                        } else if (in) {
                            uint4* po = reinterpret_cast<uint4*>(a.part_o + part * a.D + c + j);
                            po[0] = make_uint4(u[j], u[j + 1], u[j + 2], u[j + 3]);
                            po[1] = make_uint4(u[j + 4], u[j + 5], u[j + 6], u[j + 7]);
                        }
                    }
                    __syncwarp();
                }
                if (bad && rr < M && sum > 0.f)        // values that are not finite, at the slots this row sees, onto what has been written
                    for (int j = p_tile * kMKeys; j < min(p_end * kMKeys, p_top); ++j) {
                        if (!((__ldg(mask + (j >> 5)) >> (j & 31)) & 1u)) continue;
                        const int64_t at = tree_row(a.pages, p_b, j);
                        if (at < 0) continue;
                        const __nv_bfloat16* v = (const __nv_bfloat16*)a.v + at + (int64_t)p_h * a.pages.head_stride;
                        for (int d = 0; d < a.D; ++d) {
                            const float x = __bfloat162float(v[d]);
                            if (fabsf(x) <= 3.4e38f) continue;
                            if (whole) out[d] = __float2bfloat16_rn(__bfloat162float(out[d]) + x);
                            else a.part_o[part * a.D + d] += x;
                        }
                    }
                if (rr < M) {
                    if (!whole) { a.part_ml[2 * part] = ref; a.part_ml[2 * part + 1] = sum; }
                    else if (a.lse) a.lse[((int64_t)p_b * a.n + tok) * a.H + head] = sum == 0.f ? neg_inf() : (ref + log2f(sum)) * 0.6931471805599453f;
                }
                tc_before();
            }
            __syncwarp();
            if (lane == 0) { mbar_arrive(msmem_u32(&sm.o_free)); mbar_arrive(msmem_u32(&sm.released[piece % kPieces])); }
            ++piece;
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == SW) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::tmem_cols) : "memory");
    if (sm.abort_flag) {
        if (tid == 0) { atomicOr(a.pages.status, (uint32_t)DBA_TREE_TIMEOUT); a.meta[blockIdx.x] = make_int4(-2, 0, 0, 0); }       // (over what the loader wrote)
        if (a.whole_items) {           // (else the joining kernel sees to it)
            run = tree_run<C::threads>(a, kMKeys, groups * row_blocks, kItemUnits, 1, &sm.run);
            TreePiece pc;
            while (tree_next_piece(a, run, kMKeys, groups, row_blocks, kItemUnits, false, &pc)) undo_item<HP>(a, pc, C::rows);
        }
    }
}

template <int DP, int SW, int HP>
cudaError_t configure_mma() {
    static_assert(MConf<DP, SW, HP>::blocks_per_sm * (sizeof(MSmem<DP, SW, HP>) + 1024) <= 228 * 1024, "blocks of the grid that an SM holds");
    return cudaFuncSetAttribute(tree_attend_mma_kernel<DP, SW, HP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(MSmem<DP, SW, HP>));
}
template <int DP, int SW, int HP>
cudaError_t launch_mma(const TreeAttend& a, int grid, cudaStream_t st) {
    const uint32_t negate = a.scale_log2e < 0.f ? 1u << 13 : 0u;       // the scores' sign by the instruction, their size by the softmax
    return launch_after(tree_attend_mma_kernel<DP, SW, HP>, dim3(grid), dim3(MConf<DP, SW, HP>::threads), sizeof(MSmem<DP, SW, HP>), st, a, negate);
}
}  // namespace

bool tree_mma_usable(int dtype, int D) { return dtype == DBA_BF16 && D <= 128; }
// Up to 32 rows to a key head: four heads of up to 64 at a time where their number allows (beside one softmax warp to a block:
// 172 against 262 us on 4 x 131071 keys of 8 heads of 64, one row each; heads of 128 lose by it, 185 against 172 us), else
// one softmax warp.
void tree_mma_plan(int M, int K, int D, int sm_count, TreeAttendPlan* p) {
    p->item_heads = M <= 32 && K % 4 == 0 && D <= 64 ? 4 : 1;
    p->rows = M <= 32 && p->item_heads == 1 ? 32 : kMRows;
    p->grid = sm_count * (D > 64 ? (p->rows == 32 ? MConf<128, 1, 1>::blocks_per_sm : MConf<128, 4, 1>::blocks_per_sm)
                          : p->item_heads == 4 ? MConf<64, 4, 4>::blocks_per_sm
                          : p->rows == 32 ? MConf<64, 1, 1>::blocks_per_sm : MConf<64, 4, 1>::blocks_per_sm);
}
cudaError_t configure_tree_mma() {
    cudaError_t e = configure_mma<64, 1, 1>();
    if (e == cudaSuccess) e = configure_mma<64, 4, 1>();
    if (e == cudaSuccess) e = configure_mma<64, 4, 4>();
    if (e == cudaSuccess) e = configure_mma<128, 1, 1>();
    return e == cudaSuccess ? configure_mma<128, 4, 1>() : e;
}
cudaError_t launch_tree_mma(const TreeAttend& a, int rows, int grid, cudaStream_t st) {
    if (a.D > 64) return rows == 32 ? launch_mma<128, 1, 1>(a, grid, st) : launch_mma<128, 4, 1>(a, grid, st);
    return a.item_heads == 4 ? launch_mma<64, 4, 4>(a, grid, st) : rows == 32 ? launch_mma<64, 1, 1>(a, grid, st) : launch_mma<64, 4, 1>(a, grid, st);
}

}  // namespace dba
