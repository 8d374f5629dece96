// The weight that context tokens receive from attention, on the general cores: fp32 and head sizes over 128.
//
//     w'[p] = decay w[p] + sum over rows and heads of 2^(scale log2(e) <q, k_p> - lse log2(e))
//
// for every context place of a (sequence, key head): the attention's own probabilities, once its log-sum-exps are known, so keys are
// read and values are not.  A block of 256 threads works on a tile of keys and 64 rows at a time: thread (ty, tx) rows ty, ty+16, .. and
// keys tx, tx+16, ..; a key's sum goes over the rows of a thread, then over the 16 ty in their order, so no sum depends on
// the order of anything.
#include <cuda_bf16.h>

#include <type_traits>

#include "tree_span.cuh"

namespace dba {

namespace {

constexpr int kWThreads = 256, kWRows = 64;

__device__ __forceinline__ float w_ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }     // (within 2^-22)
__device__ __forceinline__ void w_fma2(float2& a, float b0, float b1, float c0, float c1) {
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\tfma.rn.f32x2 x, y, z, x;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a.x), "+f"(a.y) : "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ float w_widen(float x) { return x; }
__device__ __forceinline__ float w_widen(__nv_bfloat16 x) { return __bfloat162float(x); }

template <int DP> struct WSmem {
    static constexpr int kt = DP == 64 ? 64 : DP == 128 ? 64 : 32;
    static constexpr int pitch = DP + 4;
    float q[kWRows][pitch];
    float k[kt][pitch];
    float sum[16][kt];
    float lse[kWRows];                 // in powers of two; +inf: the row counts nothing
    int64_t row[kt];
    SpanShared span;
};

template <typename T, int DP>
__global__ void __launch_bounds__(kWThreads, DP <= 64 ? 3 : DP <= 128 ? 2 : 1) tree_weigh_kernel(const TreeWeigh a) {
    using S = WSmem<DP>;
    constexpr int KT = S::kt, NK = KT / 16, VEC = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) unsigned char wraw[];
    S& sm = *reinterpret_cast<S*>(wraw);
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, M = a.n * a.G;
    grid_dependency_wait();
    allow_dependents();
    const auto tiles_of = [&](int b) { return (min(max(__ldg(a.ctx_len + b), 0), a.ctx_cap) + KT - 1) / KT; };
    SpanRun run = span_run<kWThreads>(a.B, 1, &sm.span, [&](int b) { return (long long)a.K * tiles_of(b); });
    int have_b = -1, have_h = -1;                          // whose queries (all of them) are in shared memory
#pragma unroll 1
    for (; run.t < run.t_end; ++run.t) {
        int tiles = tiles_of(run.g);
        while (run.t - run.at >= (long long)a.K * tiles) { run.at += (long long)a.K * tiles; tiles = tiles_of(++run.g); }
        const int b = run.g, h = (int)((run.t - run.at) / tiles), t = (int)((run.t - run.at) - (long long)h * tiles);
        const int L = min(max(__ldg(a.ctx_len + b), 0), a.ctx_cap), p0 = t * KT, count = min(KT, L - p0);
        __syncthreads();                                   // the last tile is done with
        if (tid < KT) sm.row[tid] = tid < count ? tree_row(a.pages, b, a.A + p0 + tid) : -1;
        __syncthreads();
#pragma unroll 4
        for (int i = tid; i < KT * (DP / VEC); i += kWThreads) {
            const int r = i / (DP / VEC), d = (i - r * (DP / VEC)) * VEC;
            alignas(16) T x[VEC];
            if (sm.row[r] >= 0 && d < a.D) *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>((const T*)a.k + sm.row[r] + (int64_t)h * a.pages.head_stride + d);
            else *reinterpret_cast<uint4*>(x) = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < VEC; ++j) sm.k[r][d + j] = w_widen(x[j]);
        }
        float sum[NK];
#pragma unroll
        for (int j = 0; j < NK; ++j) sum[j] = 0.f;
        for (int r0 = 0; r0 < M; r0 += kWRows) {
            if (M > kWRows || b != have_b || h != have_h) {
                if (r0) __syncthreads();
                const int rows16 = M - r0 <= 16 ? 16 : M - r0 <= 32 ? 32 : kWRows;       // (those that are looked at)
#pragma unroll 4
                for (int i = tid; i < rows16 * (DP / VEC); i += kWThreads) {
                    const int r = i / (DP / VEC), d = (i - r * (DP / VEC)) * VEC, rr = r0 + r;
                    alignas(16) T x[VEC];
                    *reinterpret_cast<uint4*>(x) = make_uint4(0, 0, 0, 0);
                    if (rr < M && d < a.D) {
                        const int tok = rr / a.G, head = h * a.G + rr - tok * a.G;
                        const bool is_open = a.lse[((int64_t)b * a.n + tok) * a.H + head] != neg_inf();      // (else the query may hold anything)
                        if (is_open) *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>((const T*)a.q + (int64_t)b * a.q_seq + (int64_t)tok * a.q_row + (int64_t)head * a.q_head + d);
                    }
#pragma unroll
                    for (int j = 0; j < VEC; ++j) sm.q[r][d + j] = w_widen(x[j]);
                }
                if (tid < kWRows) {
                    float z = __int_as_float(0x7f800000);
                    const int rr = r0 + tid;
                    if (rr < M) {
                        const int tok = rr / a.G;
                        const float lse = a.lse[((int64_t)b * a.n + tok) * a.H + h * a.G + rr - tok * a.G];
                        if (lse != neg_inf()) z = lse * 1.4426950408889634f;
                    }
                    sm.lse[tid] = z;
                }
                have_b = b; have_h = h;
            }
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
                        const float4 kv = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][d]);
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
                    for (int j = 0; j < NK; ++j) sum[j] += w_ex2(fmaf(s[i][j].x + s[i][j].y, a.scale_log2e, -z));
                }
            };
            if (M - r0 <= 16) products(std::integral_constant<int, 1>{});
            else if (M - r0 <= 32) products(std::integral_constant<int, 2>{});
            else products(std::integral_constant<int, 4>{});
        }
#pragma unroll
        for (int j = 0; j < NK; ++j) sm.sum[ty][tx + 16 * j] = sum[j];
        __syncthreads();
        if (tid < count) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) x += sm.sum[i][tid];
            if (sm.row[tid] < 0) x = 0.f;
            const int64_t at = (int64_t)b * a.w_seq + (int64_t)h * a.w_head + p0 + tid;
            a.out[at] = a.in ? fmaf(a.decay, a.in[at], x) : x;
        }
    }
}

template <typename T, int DP>
cudaError_t configure_weigh() {
    static_assert((DP <= 64 ? 3 : DP <= 128 ? 2 : 1) * (sizeof(WSmem<DP>) + 1024) <= 228 * 1024, "blocks of the grid that an SM holds");
    return cudaFuncSetAttribute(tree_weigh_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(WSmem<DP>));
}
template <typename T, int DP>
cudaError_t launch_weigh(const TreeWeigh& a, int sm_count, cudaStream_t st) {
    return launch_after(tree_weigh_kernel<T, DP>, dim3((DP <= 64 ? 3 : DP <= 128 ? 2 : 1) * sm_count), dim3(kWThreads), sizeof(WSmem<DP>), st, a);
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
