// Attention of the rows of a token tree over a paged cache on the general cores: fp32 (whose products the tensor cores would
// round to 10 bits) and head sizes over 128.  And the kernel that joins the pieces of either attention kernel.
//
// softmax over the places p a row sees:  o = sum_p 2^(x_p - m) v_p / sum_p 2^(x_p - m),  x = scale log2(e) <q, k>,  with the
// running maximum m and sum kept per row while the keys go by once; a tile's contribution is rescaled when m rises.
//
// A block of 128 threads works on 8 RI rows of one (sequence, key head): 8 row groups x 16 threads.  Thread (g, c) computes the
// scores of rows g, g+8, .. with keys c, c+16, ... of the tile, and of the output the same rows x columns 4c .. 4c+3 (+64,
// ...), so a row's statistics stay in the 16 threads that use them and the probabilities cross through shared memory
// within a warp only.  RI = 1 .. 4 by the number of rows, so that few rows are computed for nothing.  Products and sums go two
// at a time (fma.rn.f32x2), which leaves issue slots to the loads from shared memory that feed them.
// The keys of the next tile and the values of this one are on their way (cp.async) while the scores are computed.
//
// What bounds it: latency.  16 sequences of up to 1000 tokens, 16 heads of 64, 20 rows, fp32: 82 to 85 us for 104 MB read (1.3 TB/s) and
// 1 GFLOP; no unit is full (instructions issued in 39 % of the cycles, loads and stores 28 %, fma 21 %, dram 19 %): a thread's products
// follow right after the loads from shared memory that feed them (short scoreboard 1.9 and fixed latencies 1.8 of 7 cycles
// an instruction), and the 12 warps that 71 KB a block leave an SM do not cover that.  Half the tile and four blocks an SM, and
// plain instead of paired products, were no faster; more products to a load has not been tried.  bf16 heads over 128 come here
// too, widened through registers into tiles of 16 keys: 16 sequences of up to 1000 tokens, 16 heads over 4 of 256, 20 rows: 364 us, where
// their 56 MB take 9.
#include <cuda_bf16.h>

#include <type_traits>

#include "tree_device.cuh"

namespace dba {

namespace {

constexpr int kGRows = 32, kGThreads = 128;
constexpr int kGItemUnits = 1;              // what an item costs beside its tiles, in tiles

__device__ __forceinline__ void tree_store(float* p, float x) { *p = x; }
__device__ __forceinline__ void tree_store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

__device__ __forceinline__ float g_ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }     // (within 2^-22)
// (a0, a1) += (b0, b1) * (c0, c1)
__device__ __forceinline__ void pair_fma(float2& a, float b0, float b1, float c0, float c1) {
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\tfma.rn.f32x2 x, y, z, x;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a.x), "+f"(a.y) : "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}

template <int DP> struct GSmem {
    static constexpr int kt = DP == 64 ? 64 : DP == 128 ? 32 : 16;     // keys per tile: 16 KB of fp32
    static constexpr int pitch = DP + 4;                               // (16 rows at a time without a conflict of banks)
    float q[kGRows][pitch];
    float k[2][kt][pitch];
    float v[kt][pitch];
    float p[kGRows][kt + 4];
    int64_t row[2][kt];
    TreeRunShared run;
};

__device__ __forceinline__ void g_copy16(float* dst, const float* src, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(in ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void g_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void g_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// One tile of keys or values; rows at -1 and what lies beyond the head size are zeros.  fp32 is copied; bf16 is widened on the
// way, through registers.
template <int DP>
__device__ __forceinline__ void g_load(const TreeAttend& a, const float* base, const int64_t* row, float (*dst)[DP + 4]) {
    constexpr int CH = DP / 4;
#pragma unroll
    for (int i = threadIdx.x; i < GSmem<DP>::kt * CH; i += kGThreads) {
        const int r = i / CH, d = (i - r * CH) * 4;
        const bool in = row[r] >= 0 && d < a.D;
        g_copy16(&dst[r][d], in ? base + row[r] + d : base, in);
    }
}
template <int DP>
__device__ __forceinline__ void g_load(const TreeAttend& a, const __nv_bfloat16* base, const int64_t* row, float (*dst)[DP + 4]) {
    constexpr int CH = DP / 8;
#pragma unroll 4
    for (int i = threadIdx.x; i < GSmem<DP>::kt * CH; i += kGThreads) {
        const int r = i / CH, d = (i - r * CH) * 8;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (row[r] >= 0 && d < a.D) x = *reinterpret_cast<const uint4*>(base + row[r] + d);
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { dst[r][d + 2 * j] = __uint_as_float(u[j] << 16); dst[r][d + 2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
    }
}
// How many fp32 a thread brings in at a time, and whether one of them is not finite.
template <int N> struct TreeCopiedN {
    static constexpr int n = N;
    __device__ static bool not_finite(const float* p) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < N; ++i) odd = odd || (__float_as_uint(p[i]) & 0x7f800000u) == 0x7f800000u;
        return odd;
    }
};
template <typename T> struct TreeCopied;
template <> struct TreeCopied<float> : TreeCopiedN<4> {};
template <> struct TreeCopied<__nv_bfloat16> : TreeCopiedN<8> {};
__device__ __forceinline__ float g_widen(float x) { return x; }
__device__ __forceinline__ float g_widen(__nv_bfloat16 x) { return __bfloat162float(x); }

// Whether some of a sequence's rows see an arena slot; masks: the sequence's, W words a row.
__device__ __noinline__ bool g_seen(const uint32_t* masks, int rows, int W, int slot) {
    for (int i = 0; i < rows; ++i)
        if ((__ldg(masks + i * W + (slot >> 5)) >> (slot & 31)) & 1u) return true;
    return false;
}

template <typename T, int DP, int RI>
__global__ void __launch_bounds__(kGThreads, DP <= 128 ? 3 : 2) tree_attend_plain_kernel(const TreeAttend a) {
    using S = GSmem<DP>;
    constexpr int KT = S::kt, NK = KT / 16, NC = DP / 64, ROWS = 8 * RI;
    extern __shared__ __align__(16) unsigned char raw[];
    S& sm = *reinterpret_cast<S*>(raw);
    const int tid = threadIdx.x, grp = tid >> 4, c = tid & 15;
    const int M = a.n * a.G, row_blocks = (M + ROWS - 1) / ROWS;
    grid_dependency_wait();
    allow_dependents();
    TreeRun run = tree_run<kGThreads>(a, KT, a.K * row_blocks, kGItemUnits, 1, &sm.run);
    TreePiece pc;
    bool first = true;
    if (run.t >= run.t_end && tid == 0) tree_write_meta(a, run, nullptr, row_blocks, kGItemUnits);
    for (;;) {
        const bool more = tree_next_piece(a, run, KT, a.K, row_blocks, kGItemUnits, first, &pc);
        if (first && tid == 0) tree_write_meta(a, run, more ? &pc : nullptr, row_blocks, kGItemUnits);
        if (!more) break;
        first = false;
        const int rows_here = min(ROWS, M - pc.rb * ROWS);
        const T* const kb = (const T*)a.k + (int64_t)pc.h * a.pages.head_stride;
        const T* const vb = (const T*)a.v + (int64_t)pc.h * a.pages.head_stride;
        auto find_rows = [&](int t) {                      // rows of a tile in the cache
            if (t < pc.tile + pc.tiles)
                for (int i = tid; i < KT; i += kGThreads) {
                    int place, count;
                    tree_tile_span(a, pc, t, KT, &place, &count);
                    // (an arena slot that no row sees need not have a page)
                    sm.row[t & 1][i] = i >= count ? -1 : tree_row(a.pages, pc.b, place + i, [&] { return place >= a.A || g_seen(a.masks + (int64_t)pc.b * a.n * a.W, a.n, a.W, place + i); });
                }
        };
        __syncthreads();                                   // the last piece is done with
        find_rows(pc.tile);
        for (int i = tid; i < ROWS * DP; i += kGThreads) { // queries, zero beyond the rows and the head size
            const int r = i / DP, d = i - r * DP;
            float x = 0.f;
            if (r < rows_here && d < a.D) {
                const int rr = pc.rb * ROWS + r, tok = rr / a.G, head = pc.h * a.G + rr - tok * a.G;
                x = g_widen(((const T*)a.q)[(int64_t)pc.b * a.q_seq + (int64_t)tok * a.q_row + (int64_t)head * a.q_head + d]);
            }
            sm.q[r][d] = x;
        }
        __syncthreads();
        g_load<DP>(a, kb, sm.row[pc.tile & 1], sm.k[pc.tile & 1]);
        g_commit();
        find_rows(pc.tile + 1);
        float m[RI], l[RI];
        float2 o[RI][NC * 2];
        const uint32_t* mask[RI];
        bool live[RI];
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            m[i] = neg_inf(); l[i] = 0.f;
            const int r = grp + 8 * i;
            const int tok = min(pc.rb * ROWS + r, M - 1) / a.G;
            mask[i] = a.masks ? a.masks + ((int64_t)pc.b * a.n + tok) * a.W : nullptr;
            live[i] = r < rows_here;
            if (a.masks && live[i]) {                    // an empty mask closes the row
                uint32_t any = 0;
                for (int w = 0; w < (pc.top + 31) / 32; ++w) any |= __ldg(mask[i] + w);
                live[i] = any != 0;
            }
#pragma unroll
            for (int j = 0; j < NC * 2; ++j) o[i][j] = make_float2(0.f, 0.f);
        }
#pragma unroll 1
        for (int t = pc.tile; t < pc.tile + pc.tiles; ++t) {
            int place, count;
            tree_tile_span(a, pc, t, KT, &place, &count);
            const bool arena = t < pc.arena_tiles;
            g_wait<0>();
            __syncthreads();                               // this tile's keys and the next one's rows are there; the last values have been used
            g_load<DP>(a, vb, sm.row[t & 1], sm.v);
            g_commit();
            if (t + 1 < pc.tile + pc.tiles) g_load<DP>(a, kb, sm.row[(t + 1) & 1], sm.k[(t + 1) & 1]);
            g_commit();
            float2 s[RI][NK];
#pragma unroll
            for (int i = 0; i < RI; ++i)
#pragma unroll
                for (int j = 0; j < NK; ++j) s[i][j] = make_float2(0.f, 0.f);
            // A tile's keys are its first `count`: of 16 or fewer, the first of each thread's alone (121 sequences of 3 tokens and 27
            // slots, 27 rows, 14 heads over 2 of 64: 84 us, 100 with all products; full tiles as before).
            const auto products = [&](auto keys) {
#pragma unroll 4
                for (int d = 0; d < DP; d += 4) {
                    float4 qv[RI];
#pragma unroll
                    for (int i = 0; i < RI; ++i) qv[i] = *reinterpret_cast<const float4*>(&sm.q[grp + 8 * i][d]);
#pragma unroll
                    for (int j = 0; j < decltype(keys)::value; ++j) {
                        const float4 kv = *reinterpret_cast<const float4*>(&sm.k[t & 1][c + 16 * j][d]);
#pragma unroll
                        for (int i = 0; i < RI; ++i) {
                            pair_fma(s[i][j], qv[i].x, qv[i].y, kv.x, kv.y);
                            pair_fma(s[i][j], qv[i].z, qv[i].w, kv.z, kv.w);
                        }
                    }
                }
            };
            if (NK > 1 && count <= 16) products(std::integral_constant<int, 1>{});
            else if (NK > 2 && count <= 32) products(std::integral_constant<int, 2>{});
            else products(std::integral_constant<int, NK>{});
#pragma unroll
            for (int i = 0; i < RI; ++i) {
                float x[NK], top = neg_inf();
#pragma unroll
                for (int j = 0; j < NK; ++j) {
                    const int kk = c + 16 * j;
                    bool see = live[i] && kk < count && sm.row[t & 1][kk] >= 0;
                    if (arena && see) see = (__ldg(mask[i] + ((place + kk) >> 5)) >> ((place + kk) & 31)) & 1u;
                    x[j] = see ? (s[i][j].x + s[i][j].y) * a.scale_log2e : neg_inf();
                    top = fmaxf(top, x[j]);
                }
#pragma unroll
                for (int k = 8; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, k));
                const float mn = fmaxf(m[i], top);
                const float ref = mn == neg_inf() ? 0.f : mn;
                const float corr = g_ex2(m[i] - ref);          // 0 while nothing has been seen
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < NK; ++j) {
                    const float e = g_ex2(x[j] - ref);
                    sm.p[grp + 8 * i][c + 16 * j] = e;
                    sum += e;
                }
#pragma unroll
                for (int k = 8; k; k >>= 1) sum += __shfl_xor_sync(kFullMask, sum, k);
                l[i] = fmaf(l[i], corr, sum);
                m[i] = mn;
#pragma unroll
                for (int j = 0; j < NC * 2; ++j) { o[i][j].x *= corr; o[i][j].y *= corr; }
            }
            g_wait<1>();                                   // the values (the next keys may still be on their way)
            // Values of the arena, which some rows see and some do not: zero times whatever they hold has to be kept out where
            // they are not finite.  Each thread looks over what it has copied.
            bool odd = false;
            if (arena)
                for (int i = tid; i < KT * (DP / TreeCopied<T>::n); i += kGThreads)
                    odd = odd || TreeCopied<T>::not_finite(&sm.v[i / (DP / TreeCopied<T>::n)][i % (DP / TreeCopied<T>::n) * TreeCopied<T>::n]);
            odd = __syncthreads_or(odd);
            // (the tile after the next takes this one's place among the rows)
            if (odd) {
#pragma unroll 1
                for (int k = 0; k < count; ++k) {
#pragma unroll
                    for (int i = 0; i < RI; ++i) {
                        const bool see = live[i] && ((__ldg(mask[i] + ((place + k) >> 5)) >> ((place + k) & 31)) & 1u);
                        const float e = sm.p[grp + 8 * i][k];
#pragma unroll
                        for (int cc = 0; cc < NC; ++cc) {
                            const float4 vv = *reinterpret_cast<const float4*>(&sm.v[k][cc * 64 + 4 * c]);
                            if (see) { pair_fma(o[i][2 * cc], e, e, vv.x, vv.y); pair_fma(o[i][2 * cc + 1], e, e, vv.z, vv.w); }
                        }
                    }
                }
            } else {
#pragma unroll 2
                for (int k = 0; k < count; k += 4) {       // (rows that do not exist are zeros, and so are their probabilities)
                    float4 e[RI];
#pragma unroll
                    for (int i = 0; i < RI; ++i) e[i] = *reinterpret_cast<const float4*>(&sm.p[grp + 8 * i][k]);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                        for (int cc = 0; cc < NC; ++cc) {
                            const float4 vv = *reinterpret_cast<const float4*>(&sm.v[k + kk][cc * 64 + 4 * c]);
#pragma unroll
                            for (int i = 0; i < RI; ++i) {
                                const float w = kk == 0 ? e[i].x : kk == 1 ? e[i].y : kk == 2 ? e[i].z : e[i].w;
                                pair_fma(o[i][2 * cc], w, w, vv.x, vv.y); pair_fma(o[i][2 * cc + 1], w, w, vv.z, vv.w);
                            }
                        }
                }
            }
            find_rows(t + 2);
        }
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            const int r = grp + 8 * i;
            if (r >= rows_here) continue;
            if (pc.whole) {
                const int rr = pc.rb * ROWS + r, tok = rr / a.G, head = pc.h * a.G + rr - tok * a.G;
                T* out = (T*)a.out + (int64_t)pc.b * a.o_seq + (int64_t)tok * a.o_row + (int64_t)head * a.o_head;
                const float inv = l[i] > 0.f ? 1.f / l[i] : 0.f;
#pragma unroll
                for (int cc = 0; cc < NC; ++cc) {
                    const float y[4] = {o[i][2 * cc].x, o[i][2 * cc].y, o[i][2 * cc + 1].x, o[i][2 * cc + 1].y};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int d = cc * 64 + 4 * c + j;
                        if (d < a.D) tree_store(out + d, l[i] == 0.f ? 0.f : y[j] * inv);
                    }
                }
                if (a.lse && c == 0) a.lse[((int64_t)pc.b * a.n + tok) * a.H + head] = l[i] == 0.f ? neg_inf() : (m[i] + log2f(l[i])) * 0.6931471805599453f;
            } else {
                const int64_t at = (int64_t)(2 * blockIdx.x + pc.slot) * ROWS + r;
                if (c == 0) { a.part_ml[2 * at] = m[i]; a.part_ml[2 * at + 1] = l[i]; }
#pragma unroll
                for (int cc = 0; cc < NC; ++cc) {
                    const int d = cc * 64 + 4 * c;
                    if (d < a.D) *reinterpret_cast<float4*>(a.part_o + at * a.D + d) = make_float4(o[i][2 * cc].x, o[i][2 * cc].y, o[i][2 * cc + 1].x, o[i][2 * cc + 1].y);
                }
            }
        }
    }
}

// Finishes the items that several blocks worked on.  Block c of the attention names in meta[c] the item it shares with block
// c - 1 if that one was the item's first: those are the items there are.  Every block here lists them and takes every
// gridDim-th row of theirs: a warp per row where few pieces meet, all eight warps on a row (each an eighth of its pieces)
// where many do.  Pieces are added in a fixed order, so equal inputs give equal bits.  A block that gave up says so in its entry, which
// every launch writes anew: a call that is recorded once and run often (a graph) keeps no failure from one run to the next.
constexpr int kCombineThreads = 256, kCombineWarps = 8, kCombineMany = 8;

template <typename T>
__global__ void __launch_bounds__(kCombineThreads) tree_combine_kernel(const TreeAttend a, int item_rows, int blocks) {
    extern __shared__ int32_t shared_items[];              // [blocks]
    __shared__ int32_t counts[kCombineWarps], most[kCombineWarps];
    __shared__ float sums[kCombineWarps][kTreeMaxDim];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    grid_dependency_wait();
    allow_dependents();
    const int M = a.n * a.G, head_rows = item_rows / a.item_heads, row_blocks = (M + head_rows - 1) / head_rows, per_head = min(M, head_rows), rows = a.item_heads * per_head;
    int n_items = 0, n_most = 0;
    bool failed = false;
    for (int c0 = 0; c0 < blocks; c0 += kCombineThreads) {
        const int c = c0 + tid;
        const int4 meta = c < blocks ? a.meta[c] : make_int4(-1, 0, 0, 0);
        const uint32_t mine = __ballot_sync(kFullMask, meta.x >= 0);
        const int pieces = meta.x >= 0 ? meta.z - c + 2 : 0;
        if (lane == 0) counts[warp] = __popc(mine);
        const int wm = __reduce_max_sync(kFullMask, pieces);
        if (lane == 0) most[warp] = wm;
        __syncthreads();
        int before = n_items + __popc(mine & ((1u << lane) - 1u));
        for (int w = 0; w < kCombineWarps; ++w) {
            if (w < warp) before += counts[w];
            n_items += counts[w];
            n_most = max(n_most, most[w]);
        }
        if (meta.x >= 0) shared_items[before] = c;
        failed = __syncthreads_or(meta.x == -2) || failed;
    }
    if (failed) {                            // a wait of this call ran out: nothing it wrote can be trusted
        const int64_t all = (int64_t)a.B * a.n * a.H;
        for (int64_t i = (int64_t)blockIdx.x * kCombineThreads + tid; i < all * a.D; i += (int64_t)gridDim.x * kCombineThreads) {
            const int64_t r = i / a.D, tok = r / a.H, b = tok / a.n;
            tree_store((T*)a.out + b * a.o_seq + (tok - b * a.n) * a.o_row + (r - tok * a.H) * a.o_head + (i - r * a.D), __int_as_float(0x7fc00000));
            if (a.lse && i == r * a.D) a.lse[r] = __int_as_float(0x7fc00000);
        }
        return;
    }
    const bool many = n_most > kCombineMany;
    const int step = many ? gridDim.x : gridDim.x * kCombineWarps;
    for (int task = many ? blockIdx.x : blockIdx.x * kCombineWarps + warp; task < n_items * rows; task += step) {
        const int item = task / rows, r = task - item * rows, c = shared_items[item];
        const int4 meta = a.meta[c];
        const int b = meta.x, group = meta.y / row_blocks, rb = meta.y - group * row_blocks;
        const int in_item = r / per_head, in_head = r - in_item * per_head, h = group * a.item_heads + in_item, rr = rb * head_rows + in_head;
        if (rr >= M) continue;                             // (the same for all warps of a task)
        const int first = c - 1, n = meta.z - first + 1;
        auto place = [&](int i) { return (int64_t)(2 * (first + i) + (i == 0 ? meta.w : 0)) * item_rows + in_item * head_rows + in_head; };
        float m = neg_inf();
        for (int i = lane; i < n; i += 32) m = fmaxf(m, a.part_ml[2 * place(i)]);
        m = warp_max(m);
        const float ref = m == neg_inf() ? 0.f : m;
        float l = 0.f;
        for (int i = lane; i < n; i += 32) l += a.part_ml[2 * place(i) + 1] * exp2f(a.part_ml[2 * place(i)] - ref);
        l = warp_sum(l);
        const int tok = rr / a.G, head = h * a.G + rr - tok * a.G;
        T* out = (T*)a.out + (int64_t)b * a.o_seq + (int64_t)tok * a.o_row + (int64_t)head * a.o_head;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const int i0 = many ? warp : 0, di = many ? kCombineWarps : 1;
        for (int d = 4 * lane; d < a.D; d += 128) {
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
            for (int i = i0; i < n; i += di) {
                const int64_t at = place(i);
                const float w = exp2f(a.part_ml[2 * at] - ref);
                const float4 v = *reinterpret_cast<const float4*>(a.part_o + at * a.D + d);
                o.x = fmaf(w, v.x, o.x); o.y = fmaf(w, v.y, o.y); o.z = fmaf(w, v.z, o.z); o.w = fmaf(w, v.w, o.w);
            }
            const float x[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (many) sums[warp][d + j] = x[j];
                else tree_store(out + d + j, l == 0.f ? 0.f : x[j] * inv);
            }
        }
        if (many) {
            __syncthreads();
            if (tid < a.D) {
                float x = 0.f;
#pragma unroll
                for (int w = 0; w < kCombineWarps; ++w) x += sums[w][tid];
                tree_store(out + tid, l == 0.f ? 0.f : x * inv);
            }
            __syncthreads();
        }
        if (a.lse && lane == 0 && (!many || warp == 0)) a.lse[((int64_t)b * a.n + tok) * a.H + head] = l == 0.f ? neg_inf() : (m + log2f(l)) * 0.6931471805599453f;
    }
}

template <typename T, int DP, int RI>
cudaError_t configure_plain() {
    static_assert((DP <= 128 ? 3 : 2) * (sizeof(GSmem<DP>) + 1024) <= 228 * 1024, "blocks of the grid that an SM holds");
    return cudaFuncSetAttribute(tree_attend_plain_kernel<T, DP, RI>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(GSmem<DP>));
}
template <typename T, int DP>
cudaError_t configure_plain_rows() {
    cudaError_t e = configure_plain<T, DP, 1>();
    if (e == cudaSuccess) e = configure_plain<T, DP, 2>();
    if (e == cudaSuccess) e = configure_plain<T, DP, 3>();
    return e == cudaSuccess ? configure_plain<T, DP, 4>() : e;
}
template <typename T, int DP, int RI>
cudaError_t launch_plain(const TreeAttend& a, int grid, cudaStream_t st) {
    return launch_after(tree_attend_plain_kernel<T, DP, RI>, dim3(grid), dim3(kGThreads), sizeof(GSmem<DP>), st, a);
}
template <typename T, int DP>
cudaError_t launch_plain_rows(const TreeAttend& a, int rows, int grid, cudaStream_t st) {
    return rows == 8 ? launch_plain<T, DP, 1>(a, grid, st) : rows == 16 ? launch_plain<T, DP, 2>(a, grid, st)
           : rows == 24 ? launch_plain<T, DP, 3>(a, grid, st) : launch_plain<T, DP, 4>(a, grid, st);
}

}  // namespace

TreeAttendPlan plan_tree_attend(int dtype, int M, int K, int D, int sm_count) {
    TreeAttendPlan p{};
    p.combine = 6 * sm_count;
    if (tree_mma_usable(dtype, D)) {
        p.tensor = true;
        tree_mma_plan(M, K, D, sm_count, &p);
        return p;
    }
    // the fewest blocks of rows of at most 32, and of those the fewest rows
    const int blocks = (M + kGRows - 1) / kGRows;
    p.rows = ((M + blocks - 1) / blocks + 7) / 8 * 8;
    p.item_heads = 1;
    p.grid = (D <= 128 ? 3 : 2) * sm_count;         // blocks that an SM's shared memory holds (71, 73 and 86 KB each)
    return p;
}

cudaError_t configure_tree_attend() {
    cudaError_t e = configure_plain_rows<float, 64>();
    if (e == cudaSuccess) e = configure_plain_rows<float, 128>();
    if (e == cudaSuccess) e = configure_plain_rows<float, 256>();
    if (e == cudaSuccess) e = configure_plain_rows<__nv_bfloat16, 256>();
    if (e == cudaSuccess) e = configure_tree_mma();
    // the same division of shared memory and L1 as the kernel before, or the SMs change over between the two
    if (e == cudaSuccess) e = cudaFuncSetAttribute(tree_combine_kernel<float>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(tree_combine_kernel<__nv_bfloat16>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    return e;
}

// Whether items are left whole, each to one block: without pieces there is nothing to join, and no second kernel.  The lengths are on the
// device, so it goes by the most keys that a table holds (short contexts in long tables are cut: 256 x 20 rows, 16 heads of
// 64, 30 to 120 tokens and 256 slots: 40 us with tables of up to 256 context places, 51 with longer ones), in 64: up to 5
// always (one sequence of 250 tokens, 8 heads of 128: 11.2 us whole, 13.6 cut; of 440, 16 heads of 64: 16.9 whole, 14.0 cut); with
// at least a third as many items as there are blocks, up to 8 (64 sequences of 440, one row: 30.7 whole, 32.3 cut; 256 of 1200: 139
// whole, 130 cut), and up to 24 where an item has more than 32 rows, whose pieces are long to write and to join (64 sequences
// of 1100, 80 rows: 66 whole, 77 cut; of 2400: 120 whole, 116 cut).
bool stays_whole(const TreeAttend& a, const TreeAttendPlan& plan) {
    const int64_t most = ((a.masks ? a.A : 0) + 63) / 64 + ((int64_t)a.ctx_cap + 63) / 64;
    const int rows = plan.rows / plan.item_heads;
    const int64_t items = (int64_t)a.B * (a.K / plan.item_heads) * ((a.n * a.G + rows - 1) / rows);
    return most <= 5 || (3 * items >= plan.grid && most <= (rows > 32 ? 24 : 8));
}

cudaError_t launch_tree_attend(TreeAttend a, const TreeAttendPlan& plan, int dtype, cudaStream_t st, int* launches) {
    cudaError_t e;
    a.whole_items = stays_whole(a, plan);
    if (plan.tensor) e = launch_tree_mma(a, plan.rows, plan.grid, st);
    else if (dtype == DBA_BF16) e = launch_plain_rows<__nv_bfloat16, 256>(a, plan.rows, plan.grid, st);
    else if (a.D <= 64) e = launch_plain_rows<float, 64>(a, plan.rows, plan.grid, st);
    else if (a.D <= 128) e = launch_plain_rows<float, 128>(a, plan.rows, plan.grid, st);
    else e = launch_plain_rows<float, 256>(a, plan.rows, plan.grid, st);
    *launches += 1;
    if (e != cudaSuccess || a.whole_items) return e;
    const size_t list = (size_t)plan.grid * sizeof(int32_t);
    e = dtype == DBA_F32 ? launch_after(tree_combine_kernel<float>, dim3(plan.combine), dim3(kCombineThreads), list, st, a, plan.rows, plan.grid)
                         : launch_after(tree_combine_kernel<__nv_bfloat16>, dim3(plan.combine), dim3(kCombineThreads), list, st, a, plan.rows, plan.grid);
    *launches += 1;
    return e;
}

}  // namespace dba
