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
// read whole before it is written, so q_out may be q.  offset (may be null): of the sequences' positions.
template <typename T, int VEC, bool PAIRS>
__global__ void __launch_bounds__(kAThreads) tree_append_kernel(const dba_tree_tokens t, const int32_t* offset, const TreePages pg, T* ck, T* cv, int B, int H, int K, int D) {
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
        if (offset && pos >= 0) {
            const int64_t moved = (int64_t)pos + __ldg(offset + b);
            pos = moved < 0 || moved > 0x7fffffff ? 0x7fffffff : (int)moved;           // (out of range, the one as the other)
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

// (x, y) = (a0, a1) * (b0, b1) [+ (x, y)]
__device__ __forceinline__ void norm_mul2(float& x, float& y, float a0, float a1, float b0, float b1) {
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}" : "=f"(x), "=f"(y) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void norm_fma2(float& x, float& y, float a0, float a1, float b0, float b1) {
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%0, %1};\n\tfma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "+f"(x), "+f"(y) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

// Whether a head is left to the end: the sum of its squares is not finite, or it is one without a norm and not rotated altogether (its zeros keep their sign).
__device__ __forceinline__ bool norm_is_apart(float sum, bool normed, bool all_turned) { return !(sum < __int_as_float(0x7f800000)) || (!all_turned && !normed); }

// The heads of a token that the kernel below leaves to the end: queries or keys, before which there are `before` others (a head's own lanes come back to
// it).  f: the pairs' factors; turned: units that are rotated.  What is not rotated keeps to itself, whatever its neighbours hold, and without a norm it is a copy.
template <typename T, int VEC, bool PAIRS>
__device__ __noinline__ void norm_apart(const T* src, T* dst, int64_t src_head, int64_t dst_head, int before, int heads, const float* f, bool normed, float eps, int D, int lanes, int turned, int half) {
    using P = TreePack<T, VEC>;
    constexpr int to = kTreeMaxDim / 2;
    const int per = D / (2 * VEC), sub = threadIdx.x / lanes, lane = threadIdx.x - sub * lanes, heads_at = blockDim.x / lanes;
    const auto first = [&](int j) { return PAIRS || j >= half / VEC ? 2 * j * VEC : j * VEC; };
    const auto second = [&](int j) { return j < half / VEC && !PAIRS ? j * VEC + half : first(j) + VEC; };
    for (int h0 = -(before % heads_at); h0 < heads; h0 += heads_at) {
        const int h = h0 + sub;
        const bool in = h >= 0 && h < heads;
        const T* const from = src + h * src_head;
        float sum = 0.f, sum2 = 0.f;                       // (in the kernel's order, so that both see the same heads)
        for (int j = lane; in && j < per; j += lanes) {
            const P x = *reinterpret_cast<const P*>(from + first(j)), y = *reinterpret_cast<const P*>(from + second(j));
#pragma unroll
            for (int i = 0; i < 2 * VEC; i += 2) {
                const float a = tree_widen(i < VEC ? x.x[i] : y.x[i - VEC]), b = tree_widen(i + 1 < VEC ? x.x[i + 1] : y.x[i + 1 - VEC]);
                sum = fmaf(a, a, sum); sum2 = fmaf(b, b, sum2);
            }
        }
        sum += sum2;
        for (int o = lanes >> 1; o; o >>= 1) sum += __shfl_xor_sync(kFullMask, sum, o);
        if (!in || !norm_is_apart(sum, normed, turned == per)) continue;
        const float r = normed ? rsqrtf(fmaf(sum, 1.f / (float)D, eps)) : 1.f;
        for (int j = lane; j < per; j += lanes) {
            const P x = *reinterpret_cast<const P*>(from + first(j)), y = *reinterpret_cast<const P*>(from + second(j));
            P ya = x, yb = y;
            const bool turn = j < turned;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                if (!turn && !normed) break;
                const int ia = PAIRS ? 2 * i : i, ib = PAIRS ? 2 * i + 1 : VEC + i;
                const float a = tree_widen(ia < VEC ? x.x[ia] : y.x[ia - VEC]), b = tree_widen(ib < VEC ? x.x[ib] : y.x[ib - VEC]), *g = f + j * VEC + i;
                const float va = r * (turn ? fmaf(a, g[0], b * g[to]) : a * g[0]), vb = r * (turn ? fmaf(b, g[2 * to], a * g[3 * to]) : b * g[2 * to]);
                tree_narrow(va, ia < VEC ? &ya.x[ia] : &yb.x[ia - VEC]);
                tree_narrow(vb, ib < VEC ? &ya.x[ib] : &yb.x[ib - VEC]);
            }
            *reinterpret_cast<P*>(dst + h * dst_head + first(j)) = ya;
            *reinterpret_cast<P*>(dst + h * dst_head + second(j)) = yb;
        }
    }
}

// The same for decoders that norm queries and keys: y = x / sqrt(mean(x^2) + eps) * weight per head, then the rotation.  A block per token;
// a head is the work of `lanes` lanes next to one another (the power of two from D/(2 VEC) up, 32 at most), each with UNITS units of
// it.  With r the root's inverse, a pair of dimensions (a, b) becomes
//     y_a = r (x_a w_a cos - x_b w_b sin),  y_b = r (x_b w_b cos + x_a w_a sin),
// whose four products of weights and cosines are the same for all heads of a kind: they are made once a token, in shared memory.  All of it is fp32; the
// one rounding is the store's.  Dimensions that are not rotated go the same way with a sine of 0, but not in heads where that would show: those are left to the
// end (norm_is_apart; with a branch for them in the loop the prompt below takes 9 % longer, with this no longer; one with half of its dimensions rotated and
// queries alone normed 100 us where 85 were without).  Without any norm an offset alone is left, and that is tree_append_kernel's (65 us, 77 by this kernel).
//
// Measured: 8 x 2039 tokens, 32 + 2 x 8 heads of 128 (402 MB): 78 us, 5.2 TB/s, 79 % of the rate of a copy; bound by the chain of a head (load, sum over its
// lanes, store: issue 58 %, 9 cycles of stalls on loads for an instruction).  The next head's loads ahead, or a warp to a token: 97 to 148 us.  16 x 20
// tokens: 6 us, dependent loads.
template <typename T, int VEC, bool PAIRS, int UNITS, int NT>
__global__ void __launch_bounds__(NT, UNITS > 1 ? 1 : NT == 64 ? 22 : 8) tree_append_norm_kernel(const dba_tree_tokens t, const dba_tree_norm nm, const TreePages pg, T* ck,
                                                                                                T* cv, int B, int H, int K, int D, int lanes) {
    using P = TreePack<T, VEC>;
    __shared__ alignas(16) float factor[2][4][kTreeMaxDim / 2];        // of queries, of keys: x_a to y_a, x_b to y_a, x_b to y_b, x_a to y_b, by pair
    __shared__ int turned_here;                            // units of a head that are rotated (read again at the end: the loop has no register for it)
    grid_dependency_wait();
    allow_dependents();
    const int tok = blockIdx.x, tid = threadIdx.x;
    const int b = t.seq ? __ldg(t.seq + tok) : tok / (t.N / B);
    const int place = __ldg(t.place + tok);
    int pos = t.position ? __ldg(t.position + tok) : -1;
    int64_t row = -1;
    bool bad = false;
    if ((unsigned)b < (unsigned)B) {
        if (place >= 0) {
            row = tree_row(pg, b, place);
            bad = row < 0;
        }
        if (pos >= 0 && nm.offset) {
            const int64_t moved = (int64_t)pos + __ldg(nm.offset + b);
            bad = bad || moved < 0 || moved >= t.positions;
            pos = moved < 0 || moved >= t.positions ? -1 : (int)moved;
        }
    } else bad = true;
    if (pos >= t.positions) { bad = bad || t.cos; pos = -1; }
    if (bad && tid == 0) atomicOr(pg.status, (uint32_t)DBA_TREE_BAD_INDEX);
    const int half = t.rot_dim / 2, turned = half / VEC;
    if (tid == 0) turned_here = pos >= 0 ? turned : 0;
    for (int i = tid; i < D; i += NT) {
        const int side = i >= D / 2, p = i - side * (D / 2), j = p / VEC;
        // the pair's dimensions: of unit j, element p % VEC of either pack, or two neighbours
        const int da = PAIRS ? 2 * p : j < turned ? p : p + j * VEC, db = PAIRS ? da + 1 : j < turned ? p + half : da + VEC;
        const float* const w = side ? nm.k_weight : nm.q_weight;
        const float wa = w ? __ldg(w + da) : 1.f, wb = w ? __ldg(w + db) : 1.f;
        const bool turn = pos >= 0 && j < turned;
        const float c = turn ? __ldg(t.cos + (int64_t)pos * half + p) : 1.f, s = turn ? __ldg(t.sin + (int64_t)pos * half + p) : 0.f;
        factor[side][0][p] = wa * c; factor[side][1][p] = -(wb * s); factor[side][2][p] = wb * c; factor[side][3][p] = wa * s;
    }
    __syncthreads();
    const int per = D / (2 * VEC), sub = tid / lanes, lane = tid - sub * lanes, heads_at = NT / lanes;
    int d0[UNITS], d1[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int j = lane + u * lanes;
        d0[u] = PAIRS || j >= turned ? 2 * j * VEC : j * VEC;
        d1[u] = j < turned && !PAIRS ? d0[u] + half : d0[u] + VEC;
        if (j >= per) d0[u] = -1;
    }
    // heads: the queries' (where there are any), then the keys'
    const int q_heads = t.q ? H : 0, n = q_heads + (row >= 0 ? K : 0);
    const float inv_d = 1.f / (float)D;
    const bool all_turned = pos >= 0 && turned == per;
    bool left = false;                                     // heads of these lanes, to the end
#pragma unroll 1
    for (int h0 = 0; h0 < n; h0 += heads_at) {
        const int h = h0 + sub;
        const bool is_q = h < q_heads;
        const T* const src = is_q ? (const T*)t.q + (int64_t)tok * t.q_token_stride + (int64_t)h * t.q_head_stride
                                  : (const T*)t.k + (int64_t)tok * t.k_token_stride + (int64_t)(h - q_heads) * t.k_head_stride;
        float e[UNITS][2 * VEC], sum = 0.f, sum2 = 0.f;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (h >= n || d0[u] < 0) continue;
            const P x = *reinterpret_cast<const P*>(src + d0[u]), y = *reinterpret_cast<const P*>(src + d1[u]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) { e[u][i] = tree_widen(x.x[i]); e[u][VEC + i] = tree_widen(y.x[i]); }
#pragma unroll
            for (int i = 0; i < 2 * VEC; i += 2) norm_fma2(sum, sum2, e[u][i], e[u][i + 1], e[u][i], e[u][i + 1]);
        }
        sum += sum2;
        for (int o = lanes >> 1; o; o >>= 1) sum += __shfl_xor_sync(kFullMask, sum, o);
        const float r = (is_q ? nm.q_weight : nm.k_weight) ? rsqrtf(fmaf(sum, inv_d, nm.eps)) : 1.f;
        T* const dst = is_q ? (T*)t.q_out + (int64_t)tok * t.qo_token_stride + (int64_t)h * t.qo_head_stride : ck + row + (int64_t)(h - q_heads) * pg.head_stride;
        const bool apart = norm_is_apart(sum, (is_q ? nm.q_weight : nm.k_weight) != nullptr, all_turned);
        left = left || apart;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (h >= n || d0[u] < 0 || apart) continue;
            const float* const f = factor[is_q ? 0 : 1][0] + (lane + u * lanes) * VEC;
            constexpr int to = kTreeMaxDim / 2;            // the next of the four
            P ya, yb;
            const auto put = [&](int i, float va, float vb) {
                if (PAIRS) { tree_narrow(va, 2 * i < VEC ? &ya.x[2 * i % VEC] : &yb.x[2 * i % VEC]); tree_narrow(vb, 2 * i + 1 < VEC ? &ya.x[(2 * i + 1) % VEC] : &yb.x[(2 * i + 1) % VEC]); }
                else { tree_narrow(va, &ya.x[i]); tree_narrow(vb, &yb.x[i]); }
            };
            if constexpr (VEC >= 2) {
                constexpr int FN = VEC < 4 ? VEC : 4;      // what shared memory gives at a time
                using F = TreePack<float, FN>;
#pragma unroll
                for (int i0 = 0; i0 < VEC; i0 += FN) {
                    const F aa = *reinterpret_cast<const F*>(f + i0), ba = *reinterpret_cast<const F*>(f + to + i0), bb = *reinterpret_cast<const F*>(f + 2 * to + i0),
                            ab = *reinterpret_cast<const F*>(f + 3 * to + i0);
#pragma unroll
                    for (int k = 0; k < FN; k += 2) {
                        const int i = i0 + k;
                        const float a0 = e[u][PAIRS ? 2 * i : i], a1 = e[u][PAIRS ? 2 * i + 2 : i + 1], b0 = e[u][PAIRS ? 2 * i + 1 : VEC + i], b1 = e[u][PAIRS ? 2 * i + 3 : VEC + i + 1];
                        float p0, p1, q0, q1;
                        norm_mul2(p0, p1, b0, b1, ba.x[k], ba.x[k + 1]); norm_fma2(p0, p1, a0, a1, aa.x[k], aa.x[k + 1]);
                        norm_mul2(q0, q1, a0, a1, ab.x[k], ab.x[k + 1]); norm_fma2(q0, q1, b0, b1, bb.x[k], bb.x[k + 1]);
                        norm_mul2(p0, p1, p0, p1, r, r); norm_mul2(q0, q1, q0, q1, r, r);
                        put(i, p0, q0); put(i + 1, p1, q1);
                    }
                }
            } else put(0, r * fmaf(e[u][0], f[0], e[u][1] * f[to]), r * fmaf(e[u][1], f[2 * to], e[u][0] * f[3 * to]));
            *reinterpret_cast<P*>(dst + d0[u]) = ya;
            *reinterpret_cast<P*>(dst + d1[u]) = yb;
        }
    }
    if (__any_sync(kFullMask, left)) {
        const int at = *(volatile int*)&turned_here, tok0 = blockIdx.x;
        if (t.q)
            norm_apart<T, VEC, PAIRS>((const T*)t.q + (int64_t)tok0 * t.q_token_stride, (T*)t.q_out + (int64_t)tok0 * t.qo_token_stride, t.q_head_stride, t.qo_head_stride, 0, H,
                                      factor[0][0], nm.q_weight != nullptr, nm.eps, D, lanes, at, t.rot_dim / 2);
        if (row >= 0)
            norm_apart<T, VEC, PAIRS>((const T*)t.k + (int64_t)tok0 * t.k_token_stride, ck + row, t.k_head_stride, pg.head_stride, t.q ? H : 0, K, factor[1][0], nm.k_weight != nullptr, nm.eps, D,
                                      lanes, at, t.rot_dim / 2);
    }
    if (row < 0) return;
    const int chunks = D * (int)sizeof(T) / 16;
    for (int u = tid; u < K * chunks; u += NT) {
        const int h = u / chunks, at = (u - h * chunks) * 16;
        *reinterpret_cast<uint4*>((char*)(cv + row + (int64_t)h * pg.head_stride) + at) =
            *reinterpret_cast<const uint4*>((const char*)((const T*)t.v + (int64_t)tok * t.v_token_stride + (int64_t)h * t.v_head_stride) + at);
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
cudaError_t launch_append_v(const dba_tree_tokens& t, const int32_t* offset, const TreePages& pg, void* k, void* v, int B, int H, int K, int D, cudaStream_t st) {
    // Blocks of 64 threads once their number fills the machine several times over (8 x 2039 tokens of 48 heads of 128: 65.0
    // us, 128 threads 67.5, 256 81), of 128 before, where a block's own loop is what takes time (16 x 20 tokens: 4.8, 3.8, 3.6).
    const int threads = t.N >= 2048 ? 64 : kAThreads;
    return t.pairs ? launch_after(tree_append_kernel<T, VEC, true>, dim3(t.N), dim3(threads), 0, st, t, offset, pg, (T*)k, (T*)v, B, H, K, D)
                   : launch_after(tree_append_kernel<T, VEC, false>, dim3(t.N), dim3(threads), 0, st, t, offset, pg, (T*)k, (T*)v, B, H, K, D);
}

}  // namespace

cudaError_t launch_tree_append(const dba_tree_tokens& t, const int32_t* offset, const TreePages& pg, void* k, void* v, int32_t B, int32_t H, int32_t K, int32_t D,
                               int dtype, cudaStream_t st, int* launches) {
    *launches += 1;
    // packs of 16 bytes where the two halves of a rotated head and what is left of it are whole numbers of them, else
    // the widest that divides them
    const int half = t.rot_dim / 2, rest = (D - t.rot_dim) / 2;
    int vec = dtype == DBA_F32 ? 4 : 8;
    while (half % vec || rest % vec) vec >>= 1;
    if (dtype == DBA_F32)
        return vec == 4 ? launch_append_v<float, 4>(t, offset, pg, k, v, B, H, K, D, st) : vec == 2 ? launch_append_v<float, 2>(t, offset, pg, k, v, B, H, K, D, st)
                                                                                              : launch_append_v<float, 1>(t, offset, pg, k, v, B, H, K, D, st);
    return vec == 8   ? launch_append_v<__nv_bfloat16, 8>(t, offset, pg, k, v, B, H, K, D, st)
           : vec == 4 ? launch_append_v<__nv_bfloat16, 4>(t, offset, pg, k, v, B, H, K, D, st)
           : vec == 2 ? launch_append_v<__nv_bfloat16, 2>(t, offset, pg, k, v, B, H, K, D, st)
                      : launch_append_v<__nv_bfloat16, 1>(t, offset, pg, k, v, B, H, K, D, st);
}

namespace {
template <typename T, int VEC, int UNITS>
cudaError_t launch_norm_u(const dba_tree_tokens& t, const dba_tree_norm& nm, const TreePages& pg, void* k, void* v, int B, int H, int K, int D, int lanes, cudaStream_t st) {
    // (blocks of 64 or of 128 threads as above: 8 x 2039 tokens of 48 heads of 128 78 us, with 128 threads 87; 16 x 20 tokens 6.9 and 5.8)
    const auto go = [&](auto* kernel, int threads) { return launch_after(kernel, dim3(t.N), dim3(threads), 0, st, t, nm, pg, (T*)k, (T*)v, B, H, K, D, lanes); };
    if (t.N >= 2048) return t.pairs ? go(tree_append_norm_kernel<T, VEC, true, UNITS, 64>, 64) : go(tree_append_norm_kernel<T, VEC, false, UNITS, 64>, 64);
    return t.pairs ? go(tree_append_norm_kernel<T, VEC, true, UNITS, 128>, 128) : go(tree_append_norm_kernel<T, VEC, false, UNITS, 128>, 128);
}
template <typename T, int VEC>
cudaError_t launch_norm_v(const dba_tree_tokens& t, const dba_tree_norm& nm, const TreePages& pg, void* k, void* v, int B, int H, int K, int D, cudaStream_t st) {
    const int per = D / (2 * VEC);
    int lanes = 1;
    while (lanes < 32 && lanes < per) lanes *= 2;
    // (a head of 256 in units of 2 VEC: up to 128 / VEC units)
    if (per <= 32) return launch_norm_u<T, VEC, 1>(t, nm, pg, k, v, B, H, K, D, lanes, st);
    if constexpr (VEC <= 2) {
        if (per <= 64) return launch_norm_u<T, VEC, 2>(t, nm, pg, k, v, B, H, K, D, lanes, st);
        if constexpr (VEC == 1) return launch_norm_u<T, VEC, 4>(t, nm, pg, k, v, B, H, K, D, lanes, st);
    }
    return cudaErrorInvalidValue;
}
}  // namespace

cudaError_t launch_tree_append_norm(const dba_tree_tokens& t, const dba_tree_norm& norm, const TreePages& pg, void* k, void* v, int32_t B, int32_t H,
                                    int32_t K, int32_t D, int dtype, cudaStream_t st, int* launches) {
    if (!norm.q_weight && !norm.k_weight) return launch_tree_append(t, norm.offset, pg, k, v, B, H, K, D, dtype, st, launches);
    *launches += 1;
    const int half = t.rot_dim / 2, rest = (D - t.rot_dim) / 2;       // (packs as above)
    int vec = dtype == DBA_F32 ? 4 : 8;
    while (half % vec || rest % vec) vec >>= 1;
    if (dtype == DBA_F32)
        return vec == 4 ? launch_norm_v<float, 4>(t, norm, pg, k, v, B, H, K, D, st) : vec == 2 ? launch_norm_v<float, 2>(t, norm, pg, k, v, B, H, K, D, st)
                                                                                              : launch_norm_v<float, 1>(t, norm, pg, k, v, B, H, K, D, st);
    return vec == 8   ? launch_norm_v<__nv_bfloat16, 8>(t, norm, pg, k, v, B, H, K, D, st)
           : vec == 4 ? launch_norm_v<__nv_bfloat16, 4>(t, norm, pg, k, v, B, H, K, D, st)
           : vec == 2 ? launch_norm_v<__nv_bfloat16, 2>(t, norm, pg, k, v, B, H, K, D, st)
                      : launch_norm_v<__nv_bfloat16, 1>(t, norm, pg, k, v, B, H, K, D, st);
}

cudaError_t launch_tree_commit(const dba_kv_cache& c, const TreePages& pg, int32_t B, int32_t K, int32_t D, int32_t A, int dtype,
                               const int32_t* ctx_len, const int32_t* src, const int32_t* n, cudaStream_t st, int* launches) {
    *launches += 1;
    const int es = dtype == DBA_F32 ? 4 : 2;
    return launch_after(tree_commit_kernel, dim3(B, 2 * c.layers), dim3(kCThreads), 0, st, pg, (char*)c.k, (char*)c.v, c.layer_stride * es, es, K,
                        D * es / 16, A, ctx_len, src, n);
}

}  // namespace dba
