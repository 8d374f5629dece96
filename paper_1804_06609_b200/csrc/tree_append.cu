// Keys and values of new tokens into the paged cache, the position rotation applied on the way, and the copying of
// settled tokens into the context.  Both are copies: bound by HBM when there are many tokens, by a launch otherwise.
// Measured on the device: a prompt of 8 x 2039 tokens, 32 + 2 x 8 heads of 128, bf16, 402 MB read and written: 65 us, 6.2 TB/s
// (94 % of what a copy reaches; more units of a thread in the air cost warps, and with them 10 to 40 us); one step's 16 x 20 tokens:
// 3.8 us.  Commit of up to 9 tokens of 64 sequences in 6 layers, 14 MB: 5.4 us (9.2 with every copy looking its places up);
// 16 sequences of 2, 32 layers: 3.3 us.
#include <cuda_bf16.h>

#include "tree_device.cuh"

namespace dba {

namespace {

constexpr int kAThreads = 128, kCThreads = 256, kCopies = 4;

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) TreePack { T x[VEC]; };
__device__ __forceinline__ float tree_widen(float x) { return x; }
__device__ __forceinline__ float tree_widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void tree_narrow(float v, float* x) { *x = v; }
__device__ __forceinline__ void tree_narrow(float v, __nv_bfloat16* x) { *x = __float2bfloat16_rn(v); }

// A block per token.  A rotated head is cut into rot/2/VEC units of two packs (dimensions d.. and d + rot/2.., or 2 VEC
// neighbouring ones) and (D - rot)/(2 VEC) units that are copied; a value head into D/(2 VEC) copied units.  A unit is
// read whole before it is written, so q_out may be q.
template <typename T, int VEC, bool PAIRS>
__global__ void __launch_bounds__(kAThreads) tree_append_kernel(const dba_tree_tokens t, const TreePages pg, T* ck, T* cv, int B, int H, int K, int D) {
    using P = TreePack<T, VEC>;
    grid_dependency_wait();
    allow_dependents();
    const int tok = blockIdx.x;
    const int b = t.seq ? __ldg(t.seq + tok) : tok / (t.N / B);
    const int place = t.place ? __ldg(t.place + tok) : -1;
    int pos = t.position ? __ldg(t.position + tok) : -1;
    int64_t row = -1;
    if ((unsigned)b < (unsigned)B) {
        if (place >= 0) {
            row = tree_row(pg, b, place);
            if (row < 0 && threadIdx.x == 0) atomicOr(pg.status, (uint32_t)DBA_TREE_BAD_INDEX);
        }
    } else if (threadIdx.x == 0) atomicOr(pg.status, (uint32_t)DBA_TREE_BAD_INDEX);
    if (pos >= t.positions && t.cos) {
        if (threadIdx.x == 0) atomicOr(pg.status, (uint32_t)DBA_TREE_BAD_INDEX);
        pos = -1;
    }
    const int half = t.rot_dim / 2, per = D / (2 * VEC), turned = half / VEC;
    const float* cosr = t.cos + (int64_t)(pos < 0 ? 0 : pos) * half;
    const float* sinr = t.sin + (int64_t)(pos < 0 ? 0 : pos) * half;
    const int q_heads = t.q ? H : 0, heads = q_heads + 2 * K;
#pragma unroll 1
    for (int u = threadIdx.x; u < heads * per; u += blockDim.x) {
        const int hd = u / per, j = u - hd * per;
        const T* src; T* dst;
        if (hd < q_heads) {
            src = (const T*)t.q + (int64_t)tok * t.q_token_stride + (int64_t)hd * t.q_head_stride;
            dst = (T*)t.q_out + (int64_t)tok * t.qo_token_stride + (int64_t)hd * t.qo_head_stride;
        } else {
            if (row < 0) continue;
            const bool is_k = hd < q_heads + K;
            const int kh = hd - q_heads - (is_k ? 0 : K);
            src = is_k ? (const T*)t.k + (int64_t)tok * t.k_token_stride + (int64_t)kh * t.k_head_stride
                       : (const T*)t.v + (int64_t)tok * t.v_token_stride + (int64_t)kh * t.v_head_stride;
            dst = (is_k ? ck : cv) + row + (int64_t)kh * pg.head_stride;
        }
        const bool turn = pos >= 0 && j < turned && hd < q_heads + K;
        // the two packs of the unit
        const int d0 = j < turned ? (PAIRS ? 2 * j * VEC : j * VEC) : t.rot_dim + 2 * (j - turned) * VEC;
        const int d1 = j < turned && !PAIRS ? d0 + half : d0 + VEC;
        P x = *reinterpret_cast<const P*>(src + d0), y = *reinterpret_cast<const P*>(src + d1);
        if (turn) {
            float cs[VEC], sn[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) { cs[i] = __ldg(cosr + j * VEC + i); sn[i] = __ldg(sinr + j * VEC + i); }
            T* const e[2] = {x.x, y.x};
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                // PAIRS: elements 2i, 2i+1 of the 2 VEC neighbours; else element i of either pack
                T* p0 = PAIRS ? e[(2 * i) / VEC] + (2 * i) % VEC : x.x + i;
                T* p1 = PAIRS ? e[(2 * i + 1) / VEC] + (2 * i + 1) % VEC : y.x + i;
                const float a = tree_widen(*p0), c = tree_widen(*p1);
                tree_narrow(fmaf(a, cs[i], -(c * sn[i])), p0);
                tree_narrow(fmaf(c, cs[i], a * sn[i]), p1);
            }
        }
        *reinterpret_cast<P*>(dst + d0) = x;
        *reinterpret_cast<P*>(dst + d1) = y;
    }
}

// A block per (sequence, layer, keys or values).  The places of up to kCThreads tokens are looked up first, one to a thread,
// so that the chain of loads to a place (slot, page) is gone through once and not for every 16 bytes; then a thread has
// kCopies copies of 16 bytes in the air.
__global__ void __launch_bounds__(kCThreads) tree_commit_kernel(const TreePages pg, char* ck, char* cv, int64_t layer_bytes, int es, int K,
                                                          int head_chunks, int A, const int32_t* ctx_len, const int32_t* src, const int32_t* n) {
    __shared__ int64_t from_at[kCThreads], to_at[kCThreads];
    grid_dependency_wait();
    allow_dependents();
    const int b = blockIdx.x, tid = threadIdx.x;
    const int count = min(max(__ldg(n + b), 0), A), ctx = __ldg(ctx_len + b);
    char* base = ((blockIdx.y & 1) ? cv : ck) + (int64_t)(blockIdx.y >> 1) * layer_bytes;
    const int per = K * head_chunks;
    for (int t0 = 0; t0 < count; t0 += kCThreads) {
        const int tokens = min(kCThreads, count - t0), units = tokens * per;
        if (t0) __syncthreads();
        if (tid < tokens) {
            const int from = __ldg(src + (int64_t)b * A + t0 + tid), to = A + ctx - count + t0 + tid;
            const int64_t r0 = (unsigned)from < (unsigned)A ? tree_row(pg, b, from) : -1, r1 = to >= A ? tree_row(pg, b, to) : -1;
            const bool bad = r0 < 0 || r1 < 0;
            if (bad) atomicOr(pg.status, (uint32_t)DBA_TREE_BAD_INDEX);
            from_at[tid] = bad ? -1 : r0 * es; to_at[tid] = r1 * es;
        }
        __syncthreads();
        for (int first = tid; first < units; first += kCopies * kCThreads) {
            uint4 x[kCopies];
            char* to[kCopies];
#pragma unroll
            for (int c = 0; c < kCopies; ++c) {
                const int u = first + c * kCThreads;
                to[c] = nullptr;
                if (u < units) {
                    const int i = u / per, w = u - i * per, h = w / head_chunks, ch = w - h * head_chunks;
                    const int64_t in_head = (int64_t)h * pg.head_stride * es + ch * 16, at = from_at[i];
                    if (at >= 0) {
                        x[c] = *reinterpret_cast<const uint4*>(base + at + in_head);
                        to[c] = base + to_at[i] + in_head;
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < kCopies; ++c)
                if (to[c]) *reinterpret_cast<uint4*>(to[c]) = x[c];
        }
    }
}

template <typename T, int VEC>
cudaError_t launch_append_v(const dba_tree_tokens& t, const TreePages& pg, void* k, void* v, int B, int H, int K, int D, cudaStream_t st) {
    // Blocks of 64 threads once their number fills the machine several times over (8 x 2039 tokens of 48 heads of 128: 65.0
    // us, 128 threads 67.5, 256 81), of 128 before, where a block's own loop is what takes time (16 x 20 tokens: 4.8, 3.8, 3.6).
    const int threads = t.N >= 2048 ? 64 : kAThreads;
    return t.pairs ? launch_after(tree_append_kernel<T, VEC, true>, dim3(t.N), dim3(threads), 0, st, t, pg, (T*)k, (T*)v, B, H, K, D)
                   : launch_after(tree_append_kernel<T, VEC, false>, dim3(t.N), dim3(threads), 0, st, t, pg, (T*)k, (T*)v, B, H, K, D);
}

}  // namespace

cudaError_t launch_tree_append(const dba_tree_tokens& t, const TreePages& pg, void* k, void* v, int32_t B, int32_t H, int32_t K, int32_t D,
                               int dtype, cudaStream_t st, int* launches) {
    *launches += 1;
    // packs of 16 bytes where the two halves of a rotated head and what is left of it are whole numbers of them, else
    // the widest that divides them
    const int half = t.rot_dim / 2, rest = (D - t.rot_dim) / 2;
    int vec = dtype == DBA_F32 ? 4 : 8;
    while (half % vec || rest % vec) vec >>= 1;
    if (dtype == DBA_F32)
        return vec == 4 ? launch_append_v<float, 4>(t, pg, k, v, B, H, K, D, st) : vec == 2 ? launch_append_v<float, 2>(t, pg, k, v, B, H, K, D, st)
                                                                                              : launch_append_v<float, 1>(t, pg, k, v, B, H, K, D, st);
    return vec == 8   ? launch_append_v<__nv_bfloat16, 8>(t, pg, k, v, B, H, K, D, st)
           : vec == 4 ? launch_append_v<__nv_bfloat16, 4>(t, pg, k, v, B, H, K, D, st)
           : vec == 2 ? launch_append_v<__nv_bfloat16, 2>(t, pg, k, v, B, H, K, D, st)
                      : launch_append_v<__nv_bfloat16, 1>(t, pg, k, v, B, H, K, D, st);
}

cudaError_t launch_tree_commit(const dba_kv_cache& c, const TreePages& pg, int32_t B, int32_t K, int32_t D, int32_t A, int dtype,
                               const int32_t* ctx_len, const int32_t* src, const int32_t* n, cudaStream_t st, int* launches) {
    *launches += 1;
    const int es = dtype == DBA_F32 ? 4 : 2;
    return launch_after(tree_commit_kernel, dim3(B, 2 * c.layers), dim3(kCThreads), 0, st, pg, (char*)c.k, (char*)c.v, c.layer_stride * es, es, K,
                        D * es / 16, A, ctx_len, src, n);
}

}  // namespace dba
