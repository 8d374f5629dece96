// The weight that context tokens receive from attention, on the general cores: fp32 and head sizes over 128.
//
//     w'[p] = decay w[p] + sum over rows and heads of 2^(scale log2(e) <q, k_p> - lse log2(e))
//
// for every context place of a (sequence, key head): the attention's own probabilities, once its log-sum-exps are known, so keys are
// read and values are not.  A block of 256 threads works on a tile of keys and 64 rows at a time: thread (ty, tx) rows ty, ty+16, .. and
// keys tx, tx+16, ..; a key's sum goes over the rows of a thread, then over the 16 ty in their order, so no sum depends on
// the order of anything.  The next tile's keys are on their way (cp.async; bf16, which is widened, comes through registers) while this one is
// worked on, and the page numbers of the one after it.
// Up to eight rows (a beam or one token, a query head to a key head): four or eight threads have a key, its dimensions in registers, and rows go by, so
// that keys come out of shared memory once and not once for every two rows.
//
// Measured, fp32, 8 sequences of up to 1000 tokens, 16 heads of 64 (27 MB): one row 14 us, five 17 (24 by the way of many rows), 20 rows 27, 64 rows 35; five
// rows of heads of 256 71 (101).  A tile's chain bounds few rows (some three tiles a block: page numbers, keys, products, sums), loads from shared
// memory many.
#include <cuda_bf16.h>

#include <type_traits>

#include "tree_span.cuh"

namespace dba {

namespace {

constexpr int kWThreads = 256, kWRows = 64, kWFew = 8;

__device__ __forceinline__ float w_ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }     // (within 2^-22)
__device__ __forceinline__ void w_fma2(float2& a, float b0, float b1, float c0, float c1) {
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\tfma.rn.f32x2 x, y, z, x;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a.x), "+f"(a.y) : "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ float w_widen(float x) { return x; }
__device__ __forceinline__ float w_widen(__nv_bfloat16 x) { return __bfloat162float(x); }

template <int DP> struct WSmem {
    static constexpr int kt = DP <= 128 ? 64 : 32;
    static constexpr int pitch = DP + 4;
    float q[kWRows][pitch];
    float k[2][kt][pitch];
    float sum[16][kt];                 // of a key, by rows' threads; few rows: the first is all
    float lse[kWRows];                 // in powers of two; +inf: the row counts nothing
    int64_t row[2][kt];
    SpanShared span;
};

// One tile of keys; rows at -1 and what lies beyond the head size are zeros.
template <int DP>
__device__ __forceinline__ void w_load(int D, const float* base, const int64_t* row, float (*dst)[DP + 4]) {
    constexpr int CH = DP / 4;
#pragma unroll 4
    for (int i = threadIdx.x; i < WSmem<DP>::kt * CH; i += kWThreads) {
        const int r = i / CH, d = (i - r * CH) * 4;
        const bool in = row[r] >= 0 && d < D;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(&dst[r][d])), "l"(in ? base + row[r] + d : base), "r"(in ? 16u : 0u) : "memory");
    }
}
template <int DP>
__device__ __forceinline__ void w_load(int D, const __nv_bfloat16* base, const int64_t* row, float (*dst)[DP + 4]) {
    constexpr int CH = DP / 8;
#pragma unroll 4
    for (int i = threadIdx.x; i < WSmem<DP>::kt * CH; i += kWThreads) {
        const int r = i / CH, d = (i - r * CH) * 8;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (row[r] >= 0 && d < D) x = *reinterpret_cast<const uint4*>(base + row[r] + d);
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { dst[r][d + 2 * j] = __uint_as_float(u[j] << 16); dst[r][d + 2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
    }
}

// FEW: up to kWFew rows to a key.
template <typename T, int DP, bool FEW>
__global__ void __launch_bounds__(kWThreads, DP <= 64 ? 3 : DP <= 128 ? 2 : 1) tree_weigh_kernel(const TreeWeigh a) {
    using S = WSmem<DP>;
    constexpr int KT = S::kt, NK = KT / 16, VEC = 16 / (int)sizeof(T), PT = kWThreads / KT, PV = DP / (4 * PT);
    extern __shared__ __align__(16) unsigned char wraw[];
    S& sm = *reinterpret_cast<S*>(wraw);
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, M = a.n * a.G;
    grid_dependency_wait();
    allow_dependents();
    const auto length_of = [&](int b) { return min(max(__ldg(a.ctx_len + b), 0), a.ctx_cap); };
    const auto tiles_of = [](int length) { return (int)((length + KT - 1u) / KT); };           // (a length may be as large as an int is)
    SpanRun run = span_run<kWThreads>(a.B, 1, &sm.span, [&](int b) { return (long long)a.K * (tiles_of(length_of(b))); });
    if (run.t >= run.t_end) return;
    // a tile: its sequence and key head, where it begins, how many keys it has
    struct Tile { int b, h, p0, count; };
    const auto tile_of = [&](long long t) {                // (in ascending order)
        int L = length_of(run.g), tiles = tiles_of(L);
        while (t - run.at >= (long long)a.K * tiles) { run.at += (long long)a.K * tiles; L = length_of(++run.g); tiles = tiles_of(L); }
        const int h = (int)((t - run.at) / tiles), p0 = (int)((t - run.at) - (long long)h * tiles) * KT;
        return Tile{run.g, h, p0, min(KT, L - p0)};
    };
    const auto find = [&](const Tile& u) { return tid < u.count ? tree_row(a.pages, u.b, a.A + u.p0 + tid) : (int64_t)-1; };
    const auto load = [&](const Tile& u, int buf) {
        w_load<DP>(a.D, (const T*)a.k + (int64_t)u.h * a.pages.head_stride, sm.row[buf], sm.k[buf]);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    Tile cur = tile_of(run.t), next = cur;
    if (tid < KT) sm.row[0][tid] = find(cur);
    if (run.t + 1 < run.t_end) {
        next = tile_of(run.t + 1);
        if (tid < KT) sm.row[1][tid] = find(next);
    }
    __syncthreads();
    load(cur, 0);
    int have_b = -1, have_h = -1, buf = 0;                 // whose queries (all of them) are in shared memory
#pragma unroll 1
    for (long long t = run.t, end = run.t_end; t < end; ++t, buf ^= 1) {
        // (both tiles' rows are there, and the buffer of the next one's keys is free)
        if (t + 1 < end) load(next, buf ^ 1);
        else asm volatile("cp.async.commit_group;" ::: "memory");
        Tile after = next;
        int64_t after_row = -1;
        if (t + 2 < end) {
            after = tile_of(t + 2);
            if (tid < KT) after_row = find(after);
        }
        float sum[NK];
#pragma unroll
        for (int j = 0; j < NK; ++j) sum[j] = 0.f;
        for (int r0 = 0; r0 < M; r0 += kWRows) {
            if (M > kWRows || cur.b != have_b || cur.h != have_h) {
                if (r0) __syncthreads();
                const int rows16 = M - r0 <= 16 ? 16 : M - r0 <= 32 ? 32 : kWRows;       // (those that are looked at)
#pragma unroll 4
                for (int i = tid; i < rows16 * (DP / VEC); i += kWThreads) {
                    const int r = i / (DP / VEC), d = (i - r * (DP / VEC)) * VEC, rr = r0 + r;
                    alignas(16) T x[VEC];
                    *reinterpret_cast<uint4*>(x) = make_uint4(0, 0, 0, 0);
                    if (rr < M && d < a.D) {
                        const int tok = rr / a.G, head = cur.h * a.G + rr - tok * a.G;
                        const bool is_open = a.lse[((int64_t)cur.b * a.n + tok) * a.H + head] != neg_inf();      // (else the query may hold anything)
                        if (is_open) *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>((const T*)a.q + (int64_t)cur.b * a.q_seq + (int64_t)tok * a.q_row + (int64_t)head * a.q_head + d);
                    }
#pragma unroll
                    for (int j = 0; j < VEC; ++j) sm.q[r][d + j] = w_widen(x[j]);
                }
                if (tid < kWRows) {
                    float z = __int_as_float(0x7f800000);
                    const int rr = r0 + tid;
                    if (rr < M) {
                        const int tok = rr / a.G;
                        const float lse = a.lse[((int64_t)cur.b * a.n + tok) * a.H + cur.h * a.G + rr - tok * a.G];
                        if (lse != neg_inf()) z = lse * 1.4426950408889634f;
                    }
                    sm.lse[tid] = z;
                }
                have_b = cur.b; have_h = cur.h;
            }
            if (r0 == 0) asm volatile("cp.async.wait_group 1;" ::: "memory");      // this tile's keys (the next one's may still be on their way)
            __syncthreads();
            // sixteen rows for each that a thread has: no more of them than there are rows
            const auto products = [&](auto rows) {
                constexpr int RI = decltype(rows)::value;
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
                        const float4 kv = *reinterpret_cast<const float4*>(&sm.k[buf][tx + 16 * j][d]);
#pragma unroll
                        for (int i = 0; i < RI; ++i) {
                            w_fma2(s[i][j], qv[i].x, qv[i].y, kv.x, kv.y);
                            w_fma2(s[i][j], qv[i].z, qv[i].w, kv.z, kv.w);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < RI; ++i) {
                    const float z = sm.lse[ty + 16 * i];
#pragma unroll
                    for (int j = 0; j < NK; ++j)           // (zeros times keys that are not finite are not zero)
                        if (z != __int_as_float(0x7f800000)) sum[j] += w_ex2(fmaf(s[i][j].x + s[i][j].y, a.scale_log2e, -z));
                }
            };
            // few rows: PT threads have a key, whose dimensions stay in their registers while the rows go by.  Eight neighbours read 128 bytes of shared memory
            // without a conflict (a row is 16 bytes longer than a multiple of 128, so four rows on it is 64 bytes further).
            const auto few = [&]() {
                const int in_key = tid % PT, key = PT == 8 ? tid / 8 : (tid >> 5) * 8 + ((tid >> 3) & 3) + (tid & 4);
                float few_sum = 0.f;
                float4 kv[PV];
#pragma unroll
                for (int c = 0; c < PV; ++c) kv[c] = *reinterpret_cast<const float4*>(&sm.k[buf][key][4 * (c * PT + in_key)]);
#pragma unroll 1
                for (int r = 0; r < M; r += PT) {     // PT rows: at last each thread has one of them
                    float x[PT];
#pragma unroll
                    for (int i = 0; i < PT; ++i) {
                        float2 s = make_float2(0.f, 0.f);
#pragma unroll
                        for (int c = 0; c < PV; ++c) {
                            const float4 qv = *reinterpret_cast<const float4*>(&sm.q[r + i][4 * (c * PT + in_key)]);
                            w_fma2(s, qv.x, qv.y, kv[c].x, kv[c].y);
                            w_fma2(s, qv.z, qv.w, kv[c].z, kv[c].w);
                        }
                        x[i] = s.x + s.y;
                    }
#pragma unroll
                    for (int o = PT / 2; o; o >>= 1)       // half of the rows stay, the other half's sums go to the thread that keeps those
#pragma unroll
                        for (int i = 0; i < o; ++i) {
                            const float mine = in_key & o ? x[i + o] : x[i], other = in_key & o ? x[i] : x[i + o];
                            x[i] = mine + __shfl_xor_sync(kFullMask, other, o);
                        }
                    const float z = sm.lse[r + in_key];
                    if (z != __int_as_float(0x7f800000)) few_sum += w_ex2(fmaf(x[0], a.scale_log2e, -z));
                }
#pragma unroll
                for (int o = PT / 2; o; o >>= 1) few_sum += __shfl_xor_sync(kFullMask, few_sum, o);
                if (in_key == 0) sm.sum[0][key] = few_sum;
            };
            if constexpr (FEW) few();
            else if (M - r0 <= 16) products(std::integral_constant<int, 1>{});
            else if (M - r0 <= 32) products(std::integral_constant<int, 2>{});
            else products(std::integral_constant<int, 4>{});
        }
        if (!FEW)
#pragma unroll
            for (int j = 0; j < NK; ++j) sm.sum[ty][tx + 16 * j] = sum[j];
        __syncthreads();
        if (tid < KT) {
            if (tid < cur.count) {
                float x = sm.sum[0][tid];
                if (!FEW)
#pragma unroll
                    for (int i = 1; i < 16; ++i) x += sm.sum[i][tid];
                if (sm.row[buf][tid] < 0) x = 0.f;
                const int64_t at = (int64_t)cur.b * a.w_seq + (int64_t)cur.h * a.w_head + cur.p0 + tid;
                a.out[at] = a.in ? fmaf(a.decay, a.in[at], x) : x;
            }
            sm.row[buf][tid] = after_row;
        }
        cur = next; next = after;
        __syncthreads();                                   // (the rows, and the sums have been read)
    }
}

template <typename T, int DP>
cudaError_t configure_weigh() {
    static_assert((DP <= 64 ? 3 : DP <= 128 ? 2 : 1) * (sizeof(WSmem<DP>) + 1024) <= 228 * 1024, "blocks of the grid that an SM holds");
    const cudaError_t e = cudaFuncSetAttribute(tree_weigh_kernel<T, DP, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(WSmem<DP>));
    return e == cudaSuccess ? cudaFuncSetAttribute(tree_weigh_kernel<T, DP, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(WSmem<DP>)) : e;
}
template <typename T, int DP>
cudaError_t launch_weigh(const TreeWeigh& a, int sm_count, cudaStream_t st) {
    const dim3 grid((DP <= 64 ? 3 : DP <= 128 ? 2 : 1) * sm_count);
    // (fp32, 8 sequences of up to 1000 tokens, 16 heads of 64: five rows 20 us, as 16 rows 24; sixteen rows 24.6, as few 28)
    return a.n * a.G <= kWFew ? launch_after(tree_weigh_kernel<T, DP, true>, grid, dim3(kWThreads), sizeof(WSmem<DP>), st, a)
                              : launch_after(tree_weigh_kernel<T, DP, false>, grid, dim3(kWThreads), sizeof(WSmem<DP>), st, a);
}

}  // namespace

cudaError_t configure_tree_weigh() {
    cudaError_t e = configure_weigh<float, 64>();
    if (e == cudaSuccess) e = configure_weigh<float, 128>();
    if (e == cudaSuccess) e = configure_weigh<float, 256>();
    if (e == cudaSuccess) e = configure_weigh<__nv_bfloat16, 256>();
    return e == cudaSuccess ? configure_tree_weigh_mma() : e;
}

cudaError_t launch_tree_weigh(const TreeWeigh& a, int dtype, int sm_count, cudaStream_t st, int* launches) {
    *launches += 1;
    if (tree_mma_usable(dtype, a.D)) return launch_tree_weigh_mma(a, sm_count, st);
    if (dtype == DBA_F32)
        return a.D <= 64 ? launch_weigh<float, 64>(a, sm_count, st) : a.D <= 128 ? launch_weigh<float, 128>(a, sm_count, st) : launch_weigh<float, 256>(a, sm_count, st);
    return launch_weigh<__nv_bfloat16, 256>(a, sm_count, st);
}

}  // namespace dba
