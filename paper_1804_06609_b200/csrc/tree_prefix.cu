// Attention over prefixes that sequences share, on the general cores: fp32 (whose products the tensor cores would round to 10 bits) and
// head sizes over 128.  And the kernel that joins the pieces of either prefix kernel.
//
// The rows of all sequences of a prefix and of all query heads of a key head are one matrix Q [rows, D]:
//     x = scale log2(e) Q K^T,   O = sum_p 2^(x_p - m) v_p,   l = sum_p 2^(x_p - m),
// m the running maximum, so that the prefix is gone through once for 64 rows and not once for each sequence.  The rows' own
// part (context and arena) comes out of dba_tree_attend's kernels before, with its log-sum-exp; out = w_own o + w_pre O.
//
// A block has 64 rows: thread (ty, tx) the scores of rows ty, ty+16, .. with keys tx, tx+TX, .. and the outputs of the same rows x columns
// 4 tx .. 4 tx + 3 (+ 4 TX, ..); a row's statistics stay in the TX threads that use them.  Sixteen bytes of queries and keys feed products of
// pairs (fma.rn.f32x2): 4 x 8 of them where eight threads have a row (head sizes to 64, three blocks of 128 threads an SM), else 4 x 4 or
// less.  The keys of the next tile and the values of this one are on their way (cp.async) while the scores are computed.  Only the epilogue needs
// the kernel before this one, so the rest runs beside its last blocks.
//
// Measured, fp32, beams of 20 on 16 sentences, three prefixes of up to 700 tokens, 16 heads (16 MB and 0.8 GFLOP with heads of 64), the whole call with the
// rows' own part of 27 us: heads of 64 73 us (81 with sixteen threads to a row, two blocks of 256), of 128 125, of 256 233; waiting for the kernel before
// at once 76, 133 and 237.  A block's chain bounds it: queries 5 us, then 6 us a tile with two others on the SM, of which the products of the scores
// are half (their operands come through shared memory), those of the outputs a third, near the rate of the fma pipes.
#include <cuda_bf16.h>

#include "tree_span.cuh"

namespace dba {

namespace {

constexpr int kPRows = 64;

__device__ __forceinline__ float p_ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }     // (within 2^-22)
// (a0, a1) += (b0, b1) * (c0, c1)
__device__ __forceinline__ void p_fma2(float2& a, float b0, float b1, float c0, float c1) {
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\tfma.rn.f32x2 x, y, z, x;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a.x), "+f"(a.y) : "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ float p_widen(float x) { return x; }
__device__ __forceinline__ float p_widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void p_store(float* p, float x) { *p = x; }
__device__ __forceinline__ void p_store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
// four neighbours, all of them there (a head's size and the strides are multiples of 16 bytes)
__device__ __forceinline__ float4 p_load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 p_load4(const __nv_bfloat16* p) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
}
__device__ __forceinline__ void p_store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
__device__ __forceinline__ void p_store4(__nv_bfloat16* p, float4 x) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
// w o + y
__device__ __forceinline__ float4 p_mix(float w, float4 o, float4 y) { return make_float4(fmaf(w, o.x, y.x), fmaf(w, o.y, y.y), fmaf(w, o.z, y.z), fmaf(w, o.w, y.w)); }

template <int DP> struct PSmem {
    static constexpr int tx = DP == 64 ? 8 : 16, threads = 16 * tx;    // threads to a row
    static constexpr int kt = DP == 64 ? 64 : DP == 128 ? 32 : 16;     // keys per tile: 16 KB of fp32
    static constexpr int blocks = DP == 64 ? 3 : DP == 128 ? 2 : 1;    // an SM's
    static constexpr int half = DP == 64 ? 32 : 0, least = DP == 64 ? 4 : 2;       // of PrefixCut and of its runs: 16 rows cost less than 64 where eight threads have a row
    static constexpr bool over = DP == 64;                             // probabilities come over the keys: a third block has room
    static constexpr int pitch = DP + 4, p_pitch = over ? kt + 8 : kt + 4;
    float q[kPRows][pitch];
    float k[2][over ? kt + 4 : kt][pitch];
    float v[kt][pitch];
    float p[over ? 1 : kPRows][p_pitch];
    int64_t row[2][kt];
    SpanShared span;
};

// One tile of keys or values; rows at -1 and what lies beyond the head size are zeros.  fp32 is copied, bf16 widened through registers.
template <int DP>
__device__ __forceinline__ void p_load(int D, const float* base, const int64_t* row, float (*dst)[DP + 4]) {
    constexpr int CH = DP / 4;
#pragma unroll
    for (int i = threadIdx.x; i < PSmem<DP>::kt * CH; i += PSmem<DP>::threads) {
        const int r = i / CH, d = (i - r * CH) * 4;
        const bool in = row[r] >= 0 && d < D;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(&dst[r][d])), "l"(in ? base + row[r] + d : base), "r"(in ? 16u : 0u) : "memory");
    }
}
template <int DP>
__device__ __forceinline__ void p_load(int D, const __nv_bfloat16* base, const int64_t* row, float (*dst)[DP + 4]) {
    constexpr int CH = DP / 8;
#pragma unroll
    for (int i = threadIdx.x; i < PSmem<DP>::kt * CH; i += PSmem<DP>::threads) {
        const int r = i / CH, d = (i - r * CH) * 8;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (row[r] >= 0 && d < D) x = *reinterpret_cast<const uint4*>(base + row[r] + d);
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { dst[r][d + 2 * j] = __uint_as_float(u[j] << 16); dst[r][d + 2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
    }
}
__device__ __forceinline__ void p_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void p_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A piece with at most 16 RI rows.
template <typename T, int DP, int RI>
__device__ __forceinline__ void prefix_piece(const TreePrefix& a, PSmem<DP>& sm, const typename PrefixCut<PSmem<DP>::kt, kPRows, PSmem<DP>::half>::Piece& pc, int64_t part) {
    constexpr int KT = PSmem<DP>::kt, TX = PSmem<DP>::tx, NK = KT / TX, NC = DP / (4 * TX);
    const int tid = threadIdx.x, ty = tid / TX, tx = tid % TX;
    const T* const kb = (const T*)a.k + (int64_t)pc.h * a.pages.head_stride;
    const T* const vb = (const T*)a.v + (int64_t)pc.h * a.pages.head_stride;
    auto find_rows = [&](int t) {
        if (t < pc.tile_end && tid < KT) sm.row[t & 1][tid] = t * KT + tid < pc.len ? tree_row(a.pages, pc.g, t * KT + tid) : -1;
    };
    __syncthreads();                                       // the last piece is done with
    find_rows(pc.tile);
    constexpr int VEC = 16 / (int)sizeof(T);
#pragma unroll 4
    for (int i = tid; i < 16 * RI * (DP / VEC); i += PSmem<DP>::threads) {       // queries, zero beyond the rows and the head size
        const int r = i / (DP / VEC), d = (i - r * (DP / VEC)) * VEC;
        alignas(16) T x[VEC];
        *reinterpret_cast<uint4*>(x) = make_uint4(0, 0, 0, 0);
        if (r < pc.rows && d < a.D) {
            const PrefixRow w = prefix_row(a, pc.lo, pc.h, pc.row0 + r);
            *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>((const T*)a.q + (int64_t)w.b * a.q_seq + (int64_t)w.i * a.q_row + (int64_t)w.head * a.q_head + d);
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) sm.q[r][d + j] = p_widen(x[j]);
    }
    __syncthreads();
    p_load<DP>(a.D, kb, sm.row[pc.tile & 1], sm.k[pc.tile & 1]);
    p_commit();
    find_rows(pc.tile + 1);
    float m[RI], l[RI];
    float2 o[RI][NC * 2];
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        m[i] = neg_inf(); l[i] = 0.f;
#pragma unroll
        for (int j = 0; j < NC * 2; ++j) o[i][j] = make_float2(0.f, 0.f);
    }
#pragma unroll 1
    for (int t = pc.tile; t < pc.tile_end; ++t) {
        const int count = min(KT, pc.len - t * KT);
        p_wait<0>();
        __syncthreads();                                   // this tile's keys and the next one's rows are there; the last values have been used
        p_load<DP>(a.D, vb, sm.row[t & 1], sm.v);
        p_commit();
        if (t + 1 < pc.tile_end) p_load<DP>(a.D, kb, sm.row[(t + 1) & 1], sm.k[(t + 1) & 1]);
        p_commit();
        const float (*const keys)[DP + 4] = sm.k[t & 1];
        float (*const p)[PSmem<DP>::p_pitch] = PSmem<DP>::over ? reinterpret_cast<float (*)[PSmem<DP>::p_pitch]>(&sm.k[t & 1][0][0]) : sm.p;
        float2 s[RI][NK];
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int j = 0; j < NK; ++j) s[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int d = 0; d < DP; d += 4) {
            float4 qv[RI];
#pragma unroll
            for (int i = 0; i < RI; ++i) qv[i] = *reinterpret_cast<const float4*>(&sm.q[ty + 16 * i][d]);
#pragma unroll
            for (int j = 0; j < NK; ++j) {
                const float4 kv = *reinterpret_cast<const float4*>(&keys[tx + TX * j][d]);
#pragma unroll
                for (int i = 0; i < RI; ++i) p_fma2(s[i][j], qv[i].x, qv[i].y, kv.x, kv.y);
#pragma unroll
                for (int i = 0; i < RI; ++i) p_fma2(s[i][j], qv[i].z, qv[i].w, kv.z, kv.w);
            }
        }
        if (PSmem<DP>::over) __syncthreads();              // the keys have been used
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            float x[NK], top = neg_inf();
#pragma unroll
            for (int j = 0; j < NK; ++j) {
                const int kk = tx + TX * j;
                x[j] = sm.row[t & 1][kk] >= 0 ? (s[i][j].x + s[i][j].y) * a.scale_log2e : neg_inf();
                top = fmaxf(top, x[j]);
            }
#pragma unroll
            for (int k = TX / 2; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, k));
            const float mn = fmaxf(m[i], top), ref = mn == neg_inf() ? 0.f : mn, corr = p_ex2(m[i] - ref);      // 0 while nothing has been seen
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NK; ++j) {
                const float e = p_ex2(x[j] - ref);
                p[ty + 16 * i][tx + TX * j] = e;
                sum += e;
            }
#pragma unroll
            for (int k = TX / 2; k; k >>= 1) sum += __shfl_xor_sync(kFullMask, sum, k);
            l[i] = fmaf(l[i], corr, sum);
            m[i] = mn;
#pragma unroll
            for (int j = 0; j < NC * 2; ++j) { o[i][j].x *= corr; o[i][j].y *= corr; }
        }
        p_wait<1>();                                       // the values (the next keys may still be on their way)
        __syncthreads();
#pragma unroll 2
        for (int k = 0; k < count; k += 4) {               // (rows that do not exist are zeros, and so are their probabilities)
            float4 e[RI];
#pragma unroll
            for (int i = 0; i < RI; ++i) e[i] = *reinterpret_cast<const float4*>(&p[ty + 16 * i][k]);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const float4 vv = *reinterpret_cast<const float4*>(&sm.v[k + kk][c * (4 * TX) + 4 * tx]);
#pragma unroll
                    for (int i = 0; i < RI; ++i) {
                        const float w = kk == 0 ? e[i].x : kk == 1 ? e[i].y : kk == 2 ? e[i].z : e[i].w;
                        p_fma2(o[i][2 * c], w, w, vv.x, vv.y); p_fma2(o[i][2 * c + 1], w, w, vv.z, vv.w);
                    }
                }
        }
        find_rows(t + 2);
    }
    if (part >= 0) {
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            const int r = ty + 16 * i;
            if (r >= pc.rows) continue;
            const int64_t at = part + r;
            if (tx == 0) { a.part_ml[2 * at] = m[i]; a.part_ml[2 * at + 1] = l[i]; }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int d = c * (4 * TX) + 4 * tx;
                if (d < a.D) *reinterpret_cast<float4*>(a.part_o + at * a.D + d) = make_float4(o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y);
            }
        }
        return;
    }
    grid_dependency_wait();
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        const int r = ty + 16 * i;
        const PrefixRow w = prefix_row(a, pc.lo, pc.h, pc.row0 + (r < pc.rows ? r : 0));
        T* const out = (T*)a.out + (int64_t)w.b * a.o_seq + (int64_t)w.i * a.o_row + (int64_t)w.head * a.o_head + 4 * tx;
        float4 old[NC];                                    // what the row has of its own: all of it on its way before anything is written
        float own, w_own, w_pre, lse;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (c * (4 * TX) + 4 * tx < a.D) old[c] = p_load4(out + c * (4 * TX));
        const bool is_open = prefix_own(a, w, &own) && r < pc.rows;
        __syncwarp();                                      // (the row's threads have read what one of them writes)
        if (!is_open || !prefix_join(own, m[i], l[i], &w_own, &w_pre, &lse)) continue;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const float2 y0 = o[i][2 * c], y1 = o[i][2 * c + 1];
            if (c * (4 * TX) + 4 * tx < a.D) p_store4(out + c * (4 * TX), p_mix(w_own, old[c], make_float4(w_pre * y0.x, w_pre * y0.y, w_pre * y1.x, w_pre * y1.y)));
        }
        if (tx == 0) a.own_lse[((int64_t)w.b * a.n + w.i) * a.H + w.head] = lse;
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(PSmem<DP>::threads, PSmem<DP>::blocks) tree_prefix_kernel(const TreePrefix a) {
    using S = PSmem<DP>;
    using Cut = PrefixCut<S::kt, kPRows, S::half>;
    extern __shared__ __align__(16) unsigned char praw[];
    S& sm = *reinterpret_cast<S*>(praw);
    // Nothing but the rows' own part comes from the kernel before this one, and that kernel has waited for what came before it: the wait
    // is the epilogue's.
    allow_dependents();
    if (blockIdx.x == 0) prefix_check(a);
    SpanRun run = Cut::template run<S::threads>(a, S::least, &sm.span);
    typename Cut::Piece pc;
    int cut = 0;
    int4 meta[2] = {make_int4(-1, 0, 0, 0), make_int4(-1, 0, 0, 0)};
    while (Cut::next(a, run, &pc)) {
        int64_t part = -1;
        if (!pc.whole()) {
            part = (int64_t)(2 * blockIdx.x + cut) * kPRows;
            meta[cut++] = make_int4(pc.g, pc.h, pc.rb, 0);
        }
        if (pc.rows <= 16) prefix_piece<T, DP, 1>(a, sm, pc, part);
        else if (pc.rows <= 32) prefix_piece<T, DP, 2>(a, sm, pc, part);
        else prefix_piece<T, DP, 4>(a, sm, pc, part);
    }
    if (threadIdx.x < 2) a.meta[2 * blockIdx.x + threadIdx.x] = meta[threadIdx.x];
    grid_dependency_wait();            // (a block without work too: what follows this kernel follows the one before it)
}

// Finishes the items that several blocks worked on.  A block's run leaves at most two pieces of such items, in the order of the
// units, so the pieces of an item are neighbours in the list of all blocks' pieces.  Every block here reads the list and takes every
// gridDim-th stretch of the items' rows: 32 rows where no item has more than kPJoinFew pieces, 8 up to twice as many, 2 beyond.  First the rows'
// weights for each piece, a thread to a piece, then the outputs, four columns to a thread, all loads of which are in the air together; of two rows
// the pieces are shared among threads, too, and their sums added (eight rows on 100003 tokens: 73 us without that, 66 with it).  Pieces are added
// in a fixed order: equal inputs give equal bits.  A block that gave up says so in its entry, which every launch writes anew.
constexpr int kPJoinThreads = 256, kPJoinWarps = kPJoinThreads / 32, kPJoinFew = 8, kPJoinRows = kPJoinThreads / kPJoinFew, kPJoinSomeRows = kPJoinWarps, kPJoinManyRows = 2;

template <typename T>
__global__ void __launch_bounds__(kPJoinThreads) tree_prefix_join_kernel(const TreePrefix a, int item_rows, int blocks) {
    extern __shared__ int4 pieces[];                       // [2 * blocks]; places of the pieces there are; of items' first ones among them; weights
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = 2 * blocks;
    int32_t* const list = reinterpret_cast<int32_t*>(pieces + n);
    int32_t* const items = list + n;
    float* const weights = reinterpret_cast<float*>(items + n);      // [rows][pieces]
    __shared__ int counts[kPJoinWarps];
    __shared__ int64_t out_at[kPJoinRows];                 // -1: the row stays as it is
    __shared__ float own_weight[kPJoinRows];
    __shared__ float4 sums[kPJoinThreads];
    grid_dependency_wait();
    allow_dependents();
    bool failed = false;
    for (int i = tid; i < n; i += kPJoinThreads) {
        pieces[i] = a.meta[i];
        failed = failed || pieces[i].x == -2;
    }
    failed = __syncthreads_or(failed);
    if (failed) {                            // a wait of this call ran out: nothing it wrote can be trusted
        const int64_t all = (int64_t)a.B * a.n * a.H;
        for (int64_t i = (int64_t)blockIdx.x * kPJoinThreads + tid; i < all * a.D; i += (int64_t)gridDim.x * kPJoinThreads) {
            const int64_t r = i / a.D, tok = r / a.H, b = tok / a.n;
            p_store((T*)a.out + b * a.o_seq + (tok - b * a.n) * a.o_row + (r - tok * a.H) * a.o_head + (i - r * a.D), __int_as_float(0x7fc00000));
            if (i == r * a.D) a.own_lse[r] = __int_as_float(0x7fc00000);
        }
        return;
    }
    // the numbers of those for which `is` holds, in order, to `to`; returns how many
    const auto compact = [&](int32_t* to, int count, auto is) {
        int total = 0;
        for (int i0 = 0; i0 < count; i0 += kPJoinThreads) {
            const bool mine = i0 + tid < count && is(i0 + tid);
            const uint32_t votes = __ballot_sync(kFullMask, mine);
            if (lane == 0) counts[warp] = __popc(votes);
            __syncthreads();
            int before = total + __popc(votes & ((1u << lane) - 1u));
#pragma unroll
            for (int w = 0; w < kPJoinWarps; ++w) {
                if (w < warp) before += counts[w];
                total += counts[w];
            }
            if (mine) to[before] = i0 + tid;
            __syncthreads();
        }
        return total;
    };
    const int n_pieces = compact(list, n, [&](int i) { return pieces[i].x >= 0; });
    if (n_pieces == 0) return;
    const int n_items = compact(items, n_pieces, [&](int i) {
        if (i == 0) return true;
        const int4 x = pieces[list[i]], y = pieces[list[i - 1]];
        return x.x != y.x || x.y != y.y || x.z != y.z;
    });
    int most = 0;
    for (int i = tid; i < n_items; i += kPJoinThreads) most = max(most, (i + 1 < n_items ? items[i + 1] : n_pieces) - items[i]);
    const bool some = __syncthreads_or(most > kPJoinFew), many = __syncthreads_or(most > 2 * kPJoinFew);
    const int rows = many ? kPJoinManyRows : some ? kPJoinSomeRows : kPJoinRows, per_item = item_rows / rows, vecs = a.D / 4;
    const int shares = many ? min(8, kPJoinThreads / (rows * vecs)) : 1;         // threads that the pieces of an output are shared among
    for (int task = blockIdx.x; task < n_items * per_item; task += gridDim.x) {
        const int item = task / per_item, r0 = (task - item * per_item) * rows, first = items[item];
        const int count = (item + 1 < n_items ? items[item + 1] : n_pieces) - first;
        const int4 id = pieces[list[first]];
        const PrefixGroup pg = prefix_group(a, id.x);
        const int left = (pg.hi - pg.lo) * a.n * a.G - (id.z * item_rows + r0);       // rows from here on
        if (left <= 0) continue;
        // --- weights: a warp to a row, or eight lanes
        const int lanes = some ? 32 : kPJoinFew, r = tid / lanes, l0 = tid - r * lanes;
        const bool in = r < left && r < rows;
        const PrefixRow w = prefix_row(a, pg.lo, id.y, id.z * item_rows + r0 + (in ? r : 0));
        float own, w_own = 0.f, w_pre, lse, m = neg_inf(), l = 0.f;
        const bool is_open = prefix_own(a, w, &own) && in;
        for (int i = l0; i < count; i += lanes) {
            const int64_t at = (int64_t)list[first + i] * item_rows + r0 + r;
            if (in) m = fmaxf(m, a.part_ml[2 * at]);
        }
        for (int o = lanes >> 1; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFullMask, m, o));
        const float ref = m == neg_inf() ? 0.f : m;
        for (int i = l0; i < count; i += lanes) {
            const int64_t at = (int64_t)list[first + i] * item_rows + r0 + r;
            float e = 0.f;
            if (in) {
                const float sum = a.part_ml[2 * at + 1];
                e = sum == 0.f ? 0.f : exp2f(a.part_ml[2 * at] - ref);
                l += sum * e;
            }
            if (r < rows) weights[r * count + i] = e;
        }
        for (int o = lanes >> 1; o; o >>= 1) l += __shfl_xor_sync(kFullMask, l, o);
        const bool write = prefix_join(own, ref, l, &w_own, &w_pre, &lse) && is_open;
        if (write)
            for (int i = l0; i < count; i += lanes) weights[r * count + i] *= w_pre;
        if (l0 == 0 && r < rows) {
            out_at[r] = write ? (int64_t)w.b * a.o_seq + (int64_t)w.i * a.o_row + (int64_t)w.head * a.o_head : -1;
            own_weight[r] = w_own;
        }
        __syncthreads();                                   // (and every lane has read what one of the row's writes)
        if (write && l0 == 0) a.own_lse[((int64_t)w.b * a.n + w.i) * a.H + w.head] = lse;
        // --- outputs
        for (int u0 = 0; u0 < rows * vecs * shares; u0 += kPJoinThreads) {
            const int u = u0 + tid, share = u / (rows * vecs), in_share = u - share * (rows * vecs), row = in_share / vecs, d = (in_share - row * vecs) * 4;
            const bool here = share < shares && row < left && out_at[row] >= 0;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f), old = o;
            if (here) {
                if (share == 0) old = p_load4((const T*)a.out + out_at[row] + d);
#pragma unroll 8
                for (int i = share; i < count; i += shares) {
                    const float4 v = *reinterpret_cast<const float4*>(a.part_o + ((int64_t)list[first + i] * item_rows + r0 + row) * a.D + d);
                    const float e = weights[row * count + i];
                    o.x = fmaf(e, v.x, o.x); o.y = fmaf(e, v.y, o.y); o.z = fmaf(e, v.z, o.z); o.w = fmaf(e, v.w, o.w);
                }
            }
            if (shares > 1) {                              // (all of them are in one round)
                sums[tid] = o;
                __syncthreads();
                if (share == 0)
                    for (int k = 1; k < shares; ++k) {
                        const float4 v = sums[tid + k * rows * vecs];
                        o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
                    }
            }
            if (!here || share > 0) continue;
            p_store4((T*)a.out + out_at[row] + d, p_mix(own_weight[row], old, o));
        }
        __syncthreads();
    }
}

template <typename T, int DP>
cudaError_t configure_prefix() {
    static_assert(PSmem<DP>::blocks * (sizeof(PSmem<DP>) + 1024) <= 228 * 1024, "blocks of the grid that an SM holds");
    return cudaFuncSetAttribute(tree_prefix_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PSmem<DP>));
}
template <typename T, int DP>
cudaError_t launch_prefix(const TreePrefix& a, int grid, cudaStream_t st) {
    return launch_after(tree_prefix_kernel<T, DP>, dim3(grid), dim3(PSmem<DP>::threads), sizeof(PSmem<DP>), st, a);
}

}  // namespace

TreePrefixPlan plan_tree_prefix(int dtype, int D, int sm_count) {
    TreePrefixPlan p{};
    p.sm_count = sm_count;
    if (tree_mma_usable(dtype, D)) {
        p.tensor = true;
        p.grid = sm_count;
        p.rows = tree_prefix_mma_rows();
        p.keys = tree_prefix_mma_keys();
        return p;
    }
    p.grid = (D <= 64 ? PSmem<64>::blocks : D <= 128 ? PSmem<128>::blocks : PSmem<256>::blocks) * sm_count;
    p.rows = kPRows;
    return p;
}

cudaError_t configure_tree_prefix() {
    cudaError_t e = configure_prefix<float, 64>();
    if (e == cudaSuccess) e = configure_prefix<float, 128>();
    if (e == cudaSuccess) e = configure_prefix<float, 256>();
    if (e == cudaSuccess) e = configure_prefix<__nv_bfloat16, 256>();
    // the same division of shared memory and L1 as the kernel before, or the SMs change over between the two
    if (e == cudaSuccess) e = cudaFuncSetAttribute(tree_prefix_join_kernel<float>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(tree_prefix_join_kernel<__nv_bfloat16>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    return e == cudaSuccess ? configure_tree_prefix_mma() : e;
}

cudaError_t launch_tree_prefix(TreePrefix a, const TreePrefixPlan& plan, int dtype, cudaStream_t st, int* launches) {
    cudaError_t e;
    a.joined = !plan.tensor || a.cap > plan.keys;
    if (plan.tensor) e = launch_tree_prefix_mma(a, plan.grid, st);
    else if (dtype == DBA_BF16) e = launch_prefix<__nv_bfloat16, 256>(a, plan.grid, st);
    else e = a.D <= 64 ? launch_prefix<float, 64>(a, plan.grid, st) : a.D <= 128 ? launch_prefix<float, 128>(a, plan.grid, st) : launch_prefix<float, 256>(a, plan.grid, st);
    *launches += 1;
    if (e != cudaSuccess || !a.joined) return e;
    // (an item has at most one piece from each block)
    const size_t n = (size_t)2 * plan.grid, most = (size_t)plan.grid * kPJoinManyRows, few = 2 * kPJoinRows * kPJoinFew;
    const size_t list = n * (sizeof(int4) + 2 * sizeof(int32_t)) + (most > few ? most : few) * sizeof(float);
    const int grid = plan.sm_count * 4;
    e = dtype == DBA_F32 ? launch_after(tree_prefix_join_kernel<float>, dim3(grid), dim3(kPJoinThreads), list, st, a, plan.rows, plan.grid)
                         : launch_after(tree_prefix_join_kernel<__nv_bfloat16>, dim3(grid), dim3(kPJoinThreads), list, st, a, plan.rows, plan.grid);
    *launches += 1;
    return e;
}

}  // namespace dba
