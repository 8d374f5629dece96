// Attention of the rows of a token tree over a paged cache, plain kernel: every type and head size, fp32 arithmetic on the
// general cores.  It serves fp32 (whose products the tensor cores would round to 10 bits) and head sizes over 128.
//
// softmax over the places p a row sees:  o = sum_p 2^(x_p - m) v_p / sum_p 2^(x_p - m),  x = scale log2(e) <q, k>,  with the
// running maximum m and sum kept per row while the keys go by once; a tile's contribution is rescaled when m rises.
//
// A block of 128 threads works on 32 rows of one (sequence, key head): 8 row groups x 16 threads.  Thread (g, c) computes
// the scores of rows g, g+8, g+16, g+24 with keys c, c+16, ... of the tile, and of the output the same rows x columns
// 4c .. 4c+3 (+64, ...), so a row's statistics stay in the 16 threads that use them and the probabilities
// cross through shared memory within a warp only.
#include <cuda_bf16.h>

#include "tree_device.cuh"

namespace dba {

namespace {

constexpr int kGRows = 32, kGThreads = 128;

template <typename T> struct TreeVec;
template <> struct TreeVec<float> {
    static constexpr int n = 4;
    __device__ static void load(const float* p, float* r) { const float4 v = *reinterpret_cast<const float4*>(p); r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w; }
};
template <> struct TreeVec<__nv_bfloat16> {
    static constexpr int n = 8;
    __device__ static void load(const __nv_bfloat16* p, float* r) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { r[2 * i] = __uint_as_float(u[i] << 16); r[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    }
};
__device__ __forceinline__ void tree_store(float* p, float x) { *p = x; }
__device__ __forceinline__ void tree_store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <int DP> struct GSmem {
    static constexpr int kt = 8192 / DP;               // keys per tile: 32 KB of fp32 keys, as much of values
    float q[kGRows][DP + 4];
    float k[kt][DP + 4];
    float v[kt][DP + 4];
    float p[kGRows][kt + 4];
    int64_t row[kt];
    TreeRunShared run;
};

template <typename T, int DP>
__global__ void __launch_bounds__(kGThreads) tree_attend_plain_kernel(const TreeAttend a) {
    using S = GSmem<DP>;
    constexpr int KT = S::kt, NK = KT / 16, NC = DP / 64, VN = TreeVec<T>::n;
    extern __shared__ __align__(16) unsigned char raw[];
    S& sm = *reinterpret_cast<S*>(raw);
    const int tid = threadIdx.x, grp = tid >> 4, c = tid & 15;
    const int M = a.n * a.G, row_blocks = (M + kGRows - 1) / kGRows;
    grid_dependency_wait();
    allow_dependents();
    TreeRun run = tree_run<kGThreads>(a, KT, a.K * row_blocks, 0, 1, &sm.run);
    TreePiece pc;
    bool first = true;
    if (run.t >= run.t_end && tid == 0) tree_write_meta(a, run, nullptr, row_blocks, 0);
    while (tree_next_piece(a, run, KT, a.K, row_blocks, 0, first, &pc)) {
        if (first && tid == 0) tree_write_meta(a, run, &pc, row_blocks, 0);
        first = false;
        const int rows_here = min(kGRows, M - pc.rb * kGRows);
        __syncthreads();
        for (int i = tid; i < kGRows * (DP / VN); i += kGThreads) {       // queries, zero beyond the rows and the head size
            const int r = i / (DP / VN), d = (i - r * (DP / VN)) * VN;
            float x[VN];
#pragma unroll
            for (int j = 0; j < VN; ++j) x[j] = 0.f;
            if (r < rows_here && d < a.D) {
                const int rr = pc.rb * kGRows + r, tok = rr / a.G, head = pc.h * a.G + rr - tok * a.G;
                TreeVec<T>::load((const T*)a.q + (int64_t)pc.b * a.q_seq + (int64_t)tok * a.q_row + (int64_t)head * a.q_head + d, x);
            }
#pragma unroll
            for (int j = 0; j < VN; ++j) sm.q[r][d + j] = x[j];
        }
        float m[4], l[4], o[4][NC * 4];
        const uint32_t* mask[4];
        bool live[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = neg_inf(); l[i] = 0.f;
            const int r = grp + 8 * i;
            const int tok = min(pc.rb * kGRows + r, M - 1) / a.G;
            mask[i] = a.masks ? a.masks + ((int64_t)pc.b * a.n + tok) * a.W : nullptr;
            live[i] = r < rows_here;
            if (a.masks && live[i]) {                    // an empty mask closes the row
                uint32_t any = 0;
                for (int w = 0; w < (pc.top + 31) / 32; ++w) any |= __ldg(mask[i] + w);
                live[i] = any != 0;
            }
#pragma unroll
            for (int j = 0; j < NC * 4; ++j) o[i][j] = 0.f;
        }
        for (int t = pc.tile; t < pc.tile + pc.tiles; ++t) {
            int place, count;
            tree_tile_span(a, pc, t, KT, &place, &count);
            const bool arena = t < pc.arena_tiles;
            __syncthreads();                               // the last tile has been used
            for (int i = tid; i < KT; i += kGThreads)
                sm.row[i] = i < count ? tree_row(a.pages, pc.b, place + i) : -1;
            __syncthreads();
            for (int i = tid; i < KT * (DP / VN); i += kGThreads) {
                const int r = i / (DP / VN), d = (i - r * (DP / VN)) * VN;
                float x[VN], y[VN];
#pragma unroll
                for (int j = 0; j < VN; ++j) x[j] = y[j] = 0.f;
                if (sm.row[r] >= 0 && d < a.D) {
                    const int64_t at = sm.row[r] + (int64_t)pc.h * a.pages.head_stride + d;
                    TreeVec<T>::load((const T*)a.k + at, x);
                    TreeVec<T>::load((const T*)a.v + at, y);
                }
#pragma unroll
                for (int j = 0; j < VN; ++j) { sm.k[r][d + j] = x[j]; sm.v[r][d + j] = y[j]; }
            }
            __syncthreads();
            float s[4][NK];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < NK; ++j) s[i][j] = 0.f;
#pragma unroll 2
            for (int d = 0; d < DP; d += 4) {
                float4 qv[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) qv[i] = *reinterpret_cast<const float4*>(&sm.q[grp + 8 * i][d]);
#pragma unroll
                for (int j = 0; j < NK; ++j) {
                    const float4 kv = *reinterpret_cast<const float4*>(&sm.k[c + 16 * j][d]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[i][j] = fmaf(qv[i].x, kv.x, fmaf(qv[i].y, kv.y, fmaf(qv[i].z, kv.z, fmaf(qv[i].w, kv.w, s[i][j]))));
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float top = neg_inf();
#pragma unroll
                for (int j = 0; j < NK; ++j) {
                    const int kk = c + 16 * j;
                    bool see = live[i] && kk < count && sm.row[kk] >= 0;
                    if (arena && see) see = (__ldg(mask[i] + ((place + kk) >> 5)) >> ((place + kk) & 31)) & 1u;
                    s[i][j] = see ? s[i][j] * a.scale_log2e : neg_inf();
                    top = fmaxf(top, s[i][j]);
                }
#pragma unroll
                for (int k = 8; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, k));
                const float mn = fmaxf(m[i], top);
                const float ref = mn == neg_inf() ? 0.f : mn;
                const float corr = exp2f(m[i] - ref);          // 0 while nothing has been seen
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < NK; ++j) {
                    const float e = exp2f(s[i][j] - ref);
                    sm.p[grp + 8 * i][c + 16 * j] = e;
                    sum += e;
                }
#pragma unroll
                for (int k = 8; k; k >>= 1) sum += __shfl_xor_sync(kFullMask, sum, k);
                l[i] = fmaf(l[i], corr, sum);
                m[i] = mn;
#pragma unroll
                for (int j = 0; j < NC * 4; ++j) o[i][j] *= corr;
            }
            __syncwarp();
            if (arena) {        // values some row does not see: zero times whatever they hold is kept out
#pragma unroll 1
                for (int k = 0; k < count; ++k) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool see = live[i] && ((__ldg(mask[i] + ((place + k) >> 5)) >> ((place + k) & 31)) & 1u);
                        const float e = sm.p[grp + 8 * i][k];
#pragma unroll
                        for (int cc = 0; cc < NC; ++cc) {
                            const float4 vv = *reinterpret_cast<const float4*>(&sm.v[k][cc * 64 + 4 * c]);
                            if (see) {
                                o[i][4 * cc + 0] = fmaf(e, vv.x, o[i][4 * cc + 0]); o[i][4 * cc + 1] = fmaf(e, vv.y, o[i][4 * cc + 1]);
                                o[i][4 * cc + 2] = fmaf(e, vv.z, o[i][4 * cc + 2]); o[i][4 * cc + 3] = fmaf(e, vv.w, o[i][4 * cc + 3]);
                            }
                        }
                    }
                }
            } else {
#pragma unroll 4
                for (int k = 0; k < count; ++k) {
                    float e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[i] = sm.p[grp + 8 * i][k];
#pragma unroll
                    for (int cc = 0; cc < NC; ++cc) {
                        const float4 vv = *reinterpret_cast<const float4*>(&sm.v[k][cc * 64 + 4 * c]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            o[i][4 * cc + 0] = fmaf(e[i], vv.x, o[i][4 * cc + 0]); o[i][4 * cc + 1] = fmaf(e[i], vv.y, o[i][4 * cc + 1]);
                            o[i][4 * cc + 2] = fmaf(e[i], vv.z, o[i][4 * cc + 2]); o[i][4 * cc + 3] = fmaf(e[i], vv.w, o[i][4 * cc + 3]);
                        }
                    }
                }
            }
            __syncwarp();                                  // the probabilities have been read
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = grp + 8 * i;
            if (r >= rows_here) continue;
            if (pc.whole) {
                const int rr = pc.rb * kGRows + r, tok = rr / a.G, head = pc.h * a.G + rr - tok * a.G;
                T* out = (T*)a.out + (int64_t)pc.b * a.o_seq + (int64_t)tok * a.o_row + (int64_t)head * a.o_head;
                const float inv = l[i] > 0.f ? 1.f / l[i] : 0.f;
#pragma unroll
                for (int cc = 0; cc < NC; ++cc)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int d = cc * 64 + 4 * c + j;
                        if (d < a.D) tree_store(out + d, l[i] == 0.f ? 0.f : o[i][4 * cc + j] * inv);
                    }
                if (a.lse && c == 0) a.lse[((int64_t)pc.b * a.n + tok) * a.H + head] = l[i] == 0.f ? neg_inf() : (m[i] + log2f(l[i])) * 0.6931471805599453f;
            } else {
                const int64_t at = (int64_t)(2 * blockIdx.x + pc.slot) * kGRows + r;
                if (c == 0) { a.part_ml[2 * at] = m[i]; a.part_ml[2 * at + 1] = l[i]; }
#pragma unroll
                for (int cc = 0; cc < NC; ++cc) {
                    const int d = cc * 64 + 4 * c;
                    if (d < a.D) *reinterpret_cast<float4*>(a.part_o + at * a.D + d) = make_float4(o[i][4 * cc], o[i][4 * cc + 1], o[i][4 * cc + 2], o[i][4 * cc + 3]);
                }
            }
        }
    }
}

// Finishes the items that several blocks worked on.  Block c of the attention names in meta[c] the item it shares with block
// c - 1 if that one was the item's first: those are the items there are.  Every block here lists them and takes every
// gridDim-th row of theirs: a warp per row where few pieces meet, all eight warps on a row (each an eighth of its pieces)
// where many do.  Pieces are added in a fixed order, so equal inputs give equal bits.
constexpr int kCombineThreads = 256, kCombineWarps = 8, kCombineMany = 8;

template <typename T>
__global__ void __launch_bounds__(kCombineThreads) tree_combine_kernel(const TreeAttend a, int item_rows, int blocks) {
    extern __shared__ int32_t shared_items[];              // [blocks]
    __shared__ int32_t counts[kCombineWarps], most[kCombineWarps];
    __shared__ float sums[kCombineWarps][kTreeMaxDim];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    grid_dependency_wait();
    allow_dependents();
    if (a.pages.status[1] == a.call) {       // a wait of this call ran out: nothing it wrote can be trusted
        const int64_t rows = (int64_t)a.B * a.n * a.H;
        for (int64_t i = (int64_t)blockIdx.x * kCombineThreads + tid; i < rows * a.D; i += (int64_t)gridDim.x * kCombineThreads) {
            const int64_t r = i / a.D, tok = r / a.H, b = tok / a.n;
            tree_store((T*)a.out + b * a.o_seq + (tok - b * a.n) * a.o_row + (r - tok * a.H) * a.o_head + (i - r * a.D), __int_as_float(0x7fc00000));
            if (a.lse && i == r * a.D) a.lse[r] = __int_as_float(0x7fc00000);
        }
        return;
    }
    const int M = a.n * a.G, head_rows = item_rows / a.item_heads, row_blocks = (M + head_rows - 1) / head_rows, per_head = min(M, head_rows), rows = a.item_heads * per_head;
    int n_items = 0, n_most = 0;
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
        __syncthreads();
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

template <typename T, int DP>
cudaError_t configure_plain() {
    return cudaFuncSetAttribute(tree_attend_plain_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(GSmem<DP>));
}
template <typename T, int DP>
cudaError_t launch_plain(const TreeAttend& a, int grid, cudaStream_t st) {
    return launch_after(tree_attend_plain_kernel<T, DP>, dim3(grid), dim3(kGThreads), sizeof(GSmem<DP>), st, a);
}
cudaError_t launch_fp32(const TreeAttend& a, int grid, cudaStream_t st) {
    return a.D <= 64 ? launch_plain<float, 64>(a, grid, st) : a.D <= 128 ? launch_plain<float, 128>(a, grid, st) : launch_plain<float, 256>(a, grid, st);
}

}  // namespace

TreeAttendPlan plan_tree_attend(int dtype, int M, int K, int D, int sm_count) {
    TreeAttendPlan p{};
    p.combine = 2 * sm_count;
    if (tree_mma_usable(dtype, D)) {
        p.tensor = true;
        tree_mma_plan(M, K, D, sm_count, &p);
        return p;
    }
    p.rows = kGRows;
    p.item_heads = 1;
    p.grid = 2 * sm_count;                 // two blocks of up to 105 KB of shared memory share an SM
    return p;
}

cudaError_t configure_tree_attend() {
    cudaError_t e = configure_plain<float, 64>();
    if (e == cudaSuccess) e = configure_plain<float, 128>();
    if (e == cudaSuccess) e = configure_plain<float, 256>();
    if (e == cudaSuccess) e = configure_plain<__nv_bfloat16, 256>();
    if (e == cudaSuccess) e = configure_tree_mma();
    // the same division of shared memory and L1 as the kernel before, or the SMs change over between the two
    if (e == cudaSuccess) e = cudaFuncSetAttribute(tree_combine_kernel<float>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(tree_combine_kernel<__nv_bfloat16>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    return e;
}

cudaError_t launch_tree_attend(const TreeAttend& a, const TreeAttendPlan& plan, int dtype, cudaStream_t st, int* launches) {
    cudaError_t e = plan.tensor ? launch_tree_mma(a, plan.rows, plan.grid, st)
                    : dtype == DBA_F32 ? launch_fp32(a, plan.grid, st) : launch_plain<__nv_bfloat16, 256>(a, plan.grid, st);
    if (e != cudaSuccess) return e;
    const size_t list = (size_t)plan.grid * sizeof(int32_t);
    e = dtype == DBA_F32 ? launch_after(tree_combine_kernel<float>, dim3(plan.combine), dim3(kCombineThreads), list, st, a, plan.rows, plan.grid)
                         : launch_after(tree_combine_kernel<__nv_bfloat16>, dim3(plan.combine), dim3(kCombineThreads), list, st, a, plan.rows, plan.grid);
    *launches += 2;
    return e;
}

}  // namespace dba
