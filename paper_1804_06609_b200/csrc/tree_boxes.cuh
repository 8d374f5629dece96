// Copies of neighbouring places of a page by tensor maps: what the kernels that read a bf16 cache tile by tile share.
// A box is up to 128 places in one instruction, where 16-byte copies are 2048 for a tile of 128 keys of 128: eight rows on 100003 shared tokens took 73 us
// with boxes and 92 without when the boxes came (now 66 with pages of 64, and 70 with pages of 5, which 16-byte copies fetch); gathers of four places at a
// time, 340 on a document of 6007 tokens where these took 157.
#pragma once
#include <cuda.h>

#include "tree_internal.h"
#include "tree_mma.cuh"

namespace dba {

namespace {

// Keys and values as tensors of (head dimension, place in a page, page, head), for copies of `rows` places of a page at a time.
struct TreeBoxes { CUtensorMap k, v; int32_t rows; };

// 64 columns from x on of neighbouring places of a page; what lies outside is zeros.
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int x, int token, int page, int head, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(token), "r"(page), "r"(head), "r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {      // (does not wait)
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Which of the 128 places of a tile there are, from the lanes' boxes: lane l < 128 / rows has `rows` places from `first` on, `there` or not, and the
// tile ends after `count`.  Lane 0 writes the four words.
__device__ __forceinline__ void boxes_seen(uint32_t* seen, int rows, int first, bool there, int count) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t mine = 0;
        if (there && lane * rows < 128) {
            const int lo = max(first - 32 * w, 0), hi = min(min(first + rows, count) - 32 * w, 32);
            if (hi > lo) mine = (hi == 32 ? 0xffffffffu : (1u << hi) - 1u) & ~((1u << lo) - 1u);
        }
        mine = __reduce_or_sync(kFullMask, mine);
        if (lane == 0) seen[w] = mine;
    }
}

typedef CUresult (*TreeEncode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                               CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline TreeEncode tree_encode_fn() {
    static const TreeEncode fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess ? (TreeEncode)f : nullptr;
    }();
    return fn;
}
inline bool tree_box_map(CUtensorMap* map, const void* base, const TreePages& pg, int K, int D, int rows) {
    const auto bytes = [](int64_t n, int64_t stride) { return (cuuint64_t)(n > 1 ? 2 * stride : 16); };      // (a dimension of one has any stride)
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)pg.page_size, (cuuint64_t)pg.num_pages, (cuuint64_t)K};
    const cuuint64_t strides[3] = {bytes(pg.page_size, pg.token_stride), bytes(pg.num_pages, pg.page_stride), bytes(K, pg.head_stride)};
    const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
    const TreeEncode fn = tree_encode_fn();
    return fn && fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Boxes of 8 to 128 places, the most that divide a page, a tile and where the first tile begins.  False: pages are not made of eights, or the strides
// are such as no tensor map has (there are few); then the tiles come by copies of 16 bytes.
inline bool tree_boxes(TreeBoxes* m, const void* k, const void* v, const TreePages& pg, int K, int D, int first) {
    m->rows = 128;
    while (pg.page_size % m->rows || first % m->rows) m->rows /= 2;
    return m->rows >= 8 && tree_box_map(&m->k, k, pg, K, D, m->rows) && (!v || tree_box_map(&m->v, v, pg, K, D, m->rows));
}

}  // namespace

}  // namespace dba
