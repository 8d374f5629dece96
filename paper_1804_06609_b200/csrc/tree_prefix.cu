// Attention over prefixes that sequences share, on the general cores: fp32 (whose products the tensor cores would round to 10 bits) and
// head sizes over 128.  And the kernel that joins the pieces of either prefix kernel.
//
// The rows of all sequences of a prefix and of all query heads of a key head are one matrix Q [rows, D]:
//     x = scale log2(e) Q K^T,   O = sum_p 2^(x_p - m) v_p,   l = sum_p 2^(x_p - m),
// m the running maximum, so that the prefix is gone through once for 64 rows and not once for each sequence.  The rows' own
// part (context and arena) comes out of dba_tree_attend's kernels before, with its log-sum-exp; out = w_own o + w_pre O.
//
// A block of 256 threads has 64 rows: thread (ty, tx) the scores of rows ty, ty+16, .. with keys tx, tx+16, .. and the outputs of the
// same rows x columns 4 tx .. 4 tx + 3 (+64, ..); a row's statistics stay in the 16 threads that use them.  Sixteen bytes of
// queries and keys feed 4 x 4 products of pairs (fma.rn.f32x2).  The keys of the next tile and the values of this one are on their way
// (cp.async) while the scores are computed.
#include <cuda_bf16.h>

#include "tree_span.cuh"

namespace dba {

namespace {

constexpr int kPThreads = 256, kPRows = 64;

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

template <int DP> struct PSmem {
    static constexpr int kt = DP == 64 ? 64 : DP == 128 ? 32 : 16;     // keys per tile: 16 KB of fp32
    static constexpr int pitch = DP + 4;
    float q[kPRows][pitch];
    float k[2][kt][pitch];
    float v[kt][pitch];
    float p[kPRows][kt + 4];
    int64_t row[2][kt];
    SpanShared span;
};

// One tile of keys or values; rows at -1 and what lies beyond the head size are zeros.  fp32 is copied, bf16 widened through registers.
template <int DP>
__device__ __forceinline__ void p_load(int D, const float* base, const int64_t* row, float (*dst)[DP + 4]) {
    constexpr int CH = DP / 4;
#pragma unroll
    for (int i = threadIdx.x; i < PSmem<DP>::kt * CH; i += kPThreads) {
        const int r = i / CH, d = (i - r * CH) * 4;
        const bool in = row[r] >= 0 && d < D;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(&dst[r][d])), "l"(in ? base + row[r] + d : base), "r"(in ? 16u : 0u) : "memory");
    }
}
template <int DP>
__device__ __forceinline__ void p_load(int D, const __nv_bfloat16* base, const int64_t* row, float (*dst)[DP + 4]) {
    constexpr int CH = DP / 8;
#pragma unroll
    for (int i = threadIdx.x; i < PSmem<DP>::kt * CH; i += kPThreads) {
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
__device__ __forceinline__ void prefix_piece(const TreePrefix& a, PSmem<DP>& sm, const typename PrefixCut<PSmem<DP>::kt, kPRows, 0>::Piece& pc, int64_t part) {
    constexpr int KT = PSmem<DP>::kt, NK = KT / 16, NC = DP / 64;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const T* const kb = (const T*)a.k + (int64_t)pc.h * a.pages.head_stride;
    const T* const vb = (const T*)a.v + (int64_t)pc.h * a.pages.head_stride;
    auto find_rows = [&](int t) {
        if (t < pc.tile_end && tid < KT) sm.row[t & 1][tid] = t * KT + tid < pc.len ? tree_row(a.pages, pc.g, t * KT + tid) : -1;
    };
    __syncthreads();                                       // the last piece is done with
    find_rows(pc.tile);
    for (int i = tid; i < 16 * RI * DP; i += kPThreads) {  // queries, zero beyond the rows and the head size
        const int r = i / DP, d = i - r * DP;
        float x = 0.f;
        if (r < pc.rows && d < a.D) {
            const PrefixRow w = prefix_row(a, pc.lo, pc.h, pc.row0 + r);
            x = p_widen(((const T*)a.q)[(int64_t)w.b * a.q_seq + (int64_t)w.i * a.q_row + (int64_t)w.head * a.q_head + d]);
        }
        sm.q[r][d] = x;
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
                const float4 kv = *reinterpret_cast<const float4*>(&sm.k[t & 1][tx + 16 * j][d]);
#pragma unroll
                for (int i = 0; i < RI; ++i) {
                    p_fma2(s[i][j], qv[i].x, qv[i].y, kv.x, kv.y);
                    p_fma2(s[i][j], qv[i].z, qv[i].w, kv.z, kv.w);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            float x[NK], top = neg_inf();
#pragma unroll
            for (int j = 0; j < NK; ++j) {
                const int kk = tx + 16 * j;
                x[j] = sm.row[t & 1][kk] >= 0 ? (s[i][j].x + s[i][j].y) * a.scale_log2e : neg_inf();
                top = fmaxf(top, x[j]);
            }
#pragma unroll
            for (int k = 8; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, k));
            const float mn = fmaxf(m[i], top), ref = mn == neg_inf() ? 0.f : mn, corr = p_ex2(m[i] - ref);      // 0 while nothing has been seen
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NK; ++j) {
                const float e = p_ex2(x[j] - ref);
                sm.p[ty + 16 * i][tx + 16 * j] = e;
                sum += e;
            }
#pragma unroll
            for (int k = 8; k; k >>= 1) sum += __shfl_xor_sync(kFullMask, sum, k);
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
            for (int i = 0; i < RI; ++i) e[i] = *reinterpret_cast<const float4*>(&sm.p[ty + 16 * i][k]);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const float4 vv = *reinterpret_cast<const float4*>(&sm.v[k + kk][c * 64 + 4 * tx]);
#pragma unroll
                    for (int i = 0; i < RI; ++i) {
                        const float w = kk == 0 ? e[i].x : kk == 1 ? e[i].y : kk == 2 ? e[i].z : e[i].w;
                        p_fma2(o[i][2 * c], w, w, vv.x, vv.y); p_fma2(o[i][2 * c + 1], w, w, vv.z, vv.w);
                    }
                }
        }
        find_rows(t + 2);
    }
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        const int r = ty + 16 * i;
        const bool in = r < pc.rows;
        if (part >= 0) {
            if (!in) continue;
            const int64_t at = part + r;
            if (tx == 0) { a.part_ml[2 * at] = m[i]; a.part_ml[2 * at + 1] = l[i]; }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int d = c * 64 + 4 * tx;
                if (d < a.D) *reinterpret_cast<float4*>(a.part_o + at * a.D + d) = make_float4(o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y);
            }
            continue;
        }
        const PrefixRow w = prefix_row(a, pc.lo, pc.h, pc.row0 + (in ? r : 0));
        float own, w_own, w_pre, lse;
        const bool is_open = prefix_own(a, w, &own) && in;
        __syncwarp();                                      // (the row's 16 threads have read what one of them writes)
        if (!is_open || !prefix_join(own, m[i], l[i], &w_own, &w_pre, &lse)) continue;
        T* out = (T*)a.out + (int64_t)w.b * a.o_seq + (int64_t)w.i * a.o_row + (int64_t)w.head * a.o_head;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const float y[4] = {o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = c * 64 + 4 * tx + j;
                if (d < a.D) p_store(out + d, fmaf(w_own, p_widen(out[d]), w_pre * y[j]));
            }
        }
        if (tx == 0) a.own_lse[((int64_t)w.b * a.n + w.i) * a.H + w.head] = lse;
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(kPThreads, DP <= 128 ? 2 : 1) tree_prefix_kernel(const TreePrefix a) {
    using S = PSmem<DP>;
    using Cut = PrefixCut<S::kt, kPRows, 0>;
    extern __shared__ __align__(16) unsigned char praw[];
    S& sm = *reinterpret_cast<S*>(praw);
    grid_dependency_wait();
    allow_dependents();
    if (blockIdx.x == 0) prefix_check(a);
    SpanRun run = span_run<kPThreads>(a.groups, 4, &sm.span, [&](int g) { return Cut::units(a, g); });
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
}

// Finishes the items that several blocks worked on.  A block's run leaves at most two pieces of such items, in the order of the
// units, so the pieces of an item are neighbours in the list of all blocks' pieces.  Every block here reads the list and takes every
// gridDim-th row of the items on it, a warp to a row.  Pieces are added in their order: equal inputs give equal bits.  A block that gave
// up says so in its entry, which every launch writes anew.
constexpr int kPJoinThreads = 256, kPJoinWarps = kPJoinThreads / 32;

template <typename T>
__global__ void __launch_bounds__(kPJoinThreads) tree_prefix_join_kernel(const TreePrefix a, int item_rows, int blocks) {
    extern __shared__ int4 pieces[];                       // [2 * blocks], then [2 * blocks] places of items' first pieces
    int32_t* const items = reinterpret_cast<int32_t*>(pieces + 2 * blocks);
    __shared__ int counts[kPJoinWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = 2 * blocks;
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
    const auto same = [&](const int4& x, const int4& y) { return x.x == y.x && x.y == y.y && x.z == y.z; };
    int n_items = 0;
    for (int i0 = 0; i0 < n; i0 += kPJoinThreads) {
        const int i = i0 + tid;
        bool first = i < n && pieces[i].x >= 0;
        if (first) {
            int j = i - 1;
            while (j >= 0 && pieces[j].x < 0) --j;
            first = j < 0 || !same(pieces[j], pieces[i]);
        }
        const uint32_t mine = __ballot_sync(kFullMask, first);
        if (lane == 0) counts[warp] = __popc(mine);
        __syncthreads();
        int before = n_items + __popc(mine & ((1u << lane) - 1u));
        for (int w = 0; w < kPJoinWarps; ++w) {
            if (w < warp) before += counts[w];
            n_items += counts[w];
        }
        if (first) items[before] = i;
        __syncthreads();
    }
    for (int task = blockIdx.x * kPJoinWarps + warp; task < n_items * item_rows; task += gridDim.x * kPJoinWarps) {
        const int item = task / item_rows, r = task - item * item_rows, first = items[item];
        const int4 id = pieces[first];
        const PrefixGroup pg = prefix_group(a, id.x);
        const int row = id.z * item_rows + r;
        if (row >= (pg.hi - pg.lo) * a.n * a.G) continue;
        const int last = item + 1 < n_items ? items[item + 1] : n;
        const PrefixRow w = prefix_row(a, pg.lo, id.y, row);
        float own, w_own, w_pre, lse;
        if (!prefix_own(a, w, &own)) continue;
        float m = neg_inf();
        for (int i = first + lane; i < last; i += 32)
            if (pieces[i].x >= 0) m = fmaxf(m, a.part_ml[2 * ((int64_t)i * item_rows + r)]);
        m = warp_max(m);
        const float ref = m == neg_inf() ? 0.f : m;
        float l = 0.f;
        for (int i = first + lane; i < last; i += 32)
            if (pieces[i].x >= 0) l += a.part_ml[2 * ((int64_t)i * item_rows + r) + 1] * exp2f(a.part_ml[2 * ((int64_t)i * item_rows + r)] - ref);
        l = warp_sum(l);
        if (!prefix_join(own, ref, l, &w_own, &w_pre, &lse)) continue;
        T* out = (T*)a.out + (int64_t)w.b * a.o_seq + (int64_t)w.i * a.o_row + (int64_t)w.head * a.o_head;
        for (int d = 4 * lane; d < a.D; d += 128) {
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int i = first; i < last; ++i) {
                if (pieces[i].x < 0) continue;
                const int64_t at = (int64_t)i * item_rows + r;
                const float e = exp2f(a.part_ml[2 * at] - ref);
                const float4 v = *reinterpret_cast<const float4*>(a.part_o + at * a.D + d);
                o.x = fmaf(e, v.x, o.x); o.y = fmaf(e, v.y, o.y); o.z = fmaf(e, v.z, o.z); o.w = fmaf(e, v.w, o.w);
            }
            const float y[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) p_store(out + d + j, fmaf(w_own, p_widen(out[d + j]), w_pre * y[j]));
        }
        __syncwarp();                                      // (all lanes have read what one writes)
        if (lane == 0) a.own_lse[((int64_t)w.b * a.n + w.i) * a.H + w.head] = lse;
    }
}

template <typename T, int DP>
cudaError_t configure_prefix() {
    static_assert((DP <= 128 ? 2 : 1) * (sizeof(PSmem<DP>) + 1024) <= 228 * 1024, "blocks of the grid that an SM holds");
    return cudaFuncSetAttribute(tree_prefix_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PSmem<DP>));
}
template <typename T, int DP>
cudaError_t launch_prefix(const TreePrefix& a, int grid, cudaStream_t st) {
    return launch_after(tree_prefix_kernel<T, DP>, dim3(grid), dim3(kPThreads), sizeof(PSmem<DP>), st, a);
}

}  // namespace

TreePrefixPlan plan_tree_prefix(int dtype, int D, int sm_count) {
    TreePrefixPlan p{};
    if (tree_mma_usable(dtype, D)) {
        p.tensor = true;
        p.grid = sm_count;
        p.rows = tree_prefix_mma_rows();
        return p;
    }
    p.grid = (D <= 128 ? 2 : 1) * sm_count;
    p.rows = kPRows;
    return p;
}

cudaError_t configure_tree_prefix() {
    cudaError_t e = configure_prefix<float, 64>();
    if (e == cudaSuccess) e = configure_prefix<float, 128>();
    if (e == cudaSuccess) e = configure_prefix<float, 256>();
    if (e == cudaSuccess) e = configure_prefix<__nv_bfloat16, 256>();
    return e == cudaSuccess ? configure_tree_prefix_mma() : e;
}

cudaError_t launch_tree_prefix(const TreePrefix& a, const TreePrefixPlan& plan, int dtype, cudaStream_t st, int* launches) {
    cudaError_t e;
    if (plan.tensor) e = launch_tree_prefix_mma(a, plan.grid, st);
    else if (dtype == DBA_BF16) e = launch_prefix<__nv_bfloat16, 256>(a, plan.grid, st);
    else e = a.D <= 64 ? launch_prefix<float, 64>(a, plan.grid, st) : a.D <= 128 ? launch_prefix<float, 128>(a, plan.grid, st) : launch_prefix<float, 256>(a, plan.grid, st);
    *launches += 1;
    if (e != cudaSuccess) return e;
    const size_t list = (size_t)2 * plan.grid * (sizeof(int4) + sizeof(int32_t));
    const int grid = plan.grid * 2;
    e = dtype == DBA_F32 ? launch_after(tree_prefix_join_kernel<float>, dim3(grid), dim3(kPJoinThreads), list, st, a, plan.rows, plan.grid)
                         : launch_after(tree_prefix_join_kernel<__nv_bfloat16>, dim3(grid), dim3(kPJoinThreads), list, st, a, plan.rows, plan.grid);
    *launches += 1;
    return e;
}

}  // namespace dba
