// Internal declarations of the token tree over a paged cache (dba_tree_*).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "dba_internal.h"

namespace dba {

constexpr int kTreeMaxRows = 64;       // rows per sequence (one bit each in a 64-bit mask of ancestors)
constexpr int kTreeMaxWords = 128;     // arena words per sequence
constexpr int kTreeMaxDim = 256;
constexpr int kTreeTurns = 256;        // SMs told apart by number

// What a kernel needs to find the rows of one layer's cache.
struct TreePages {
    const int32_t* table;
    int64_t table_stride;
    int32_t num_pages, max_pages, page_size;
    int64_t page_stride, token_stride, head_stride;   // elements
    uint32_t* status;
    uint32_t page_mul;                                // page_size's multiplier and shift (see tree_page)
    int32_t page_shift;
};

// Attention, all sizes of one call.
struct TreeAttend {
    TreePages pages;
    const void *k, *v, *q;
    void* out;
    float* lse;
    const int32_t* ctx_len;
    const uint32_t* masks;             // null: no arena is looked at, every row sees the context
    const int32_t* top;
    int32_t B, n, H, K, G, D;          // G = H / K query heads per key head; M = n * G rows per (sequence, key head)
    int32_t item_heads;                // key heads an item has, each a share of its rows
    int32_t W, A, ctx_cap;             // arena words and slots, context places the table holds
    int64_t q_seq, q_row, q_head, o_seq, o_row, o_head;
    float scale_log2e;                 // softmax in powers of two
    // split work: the tiles of all items are dealt out in equal contiguous runs
    float* part_o;                     // [2 * grid][rows of an item][D]: unfinished first and last items of a block's run
    float* part_ml;                    // [2 * grid][rows of an item][2]: their maxima (of the scaled scores, in powers of two) and sums
    uint32_t* turns;                   // [kTreeTurns] a counter per SM, which goes on from call to call: blocks on an SM take turns by it
    int4* meta;                        // [grid] item shared with the block before this one, if that block is the first on it (x = -1: none,
                                       // -2: the block gave up)
    int whole_items;                   // items are not cut (short ones: no second kernel then)
    long long wait_clocks;
    int drop_item;
};

struct TreeAttendPlan {
    int grid, combine;                 // blocks of the attention kernel and of the one that joins its pieces
    int rows, item_heads;              // rows of an item (all its key heads together), and its key heads
    bool tensor;                       // tcgen05 kernel
};

// The most an item's partial results take, for the workspace.
TreeAttendPlan plan_tree_attend(int dtype, int M, int K, int D, int sm_count);
cudaError_t configure_tree_attend();
// the tensor-core kernel (tree_attend_mma.cu)
bool tree_mma_usable(int dtype, int D);
void tree_mma_plan(int M, int K, int D, int sm_count, TreeAttendPlan* p);
cudaError_t configure_tree_mma();
cudaError_t launch_tree_mma(const TreeAttend& a, int rows, int grid, cudaStream_t st);
cudaError_t launch_tree_attend(TreeAttend a, const TreeAttendPlan& plan, int dtype, cudaStream_t st, int* launches);
cudaError_t launch_tree_append(const dba_tree_tokens& t, const int32_t* offset, const TreePages& pg, void* k, void* v, int32_t B, int32_t H, int32_t K,
                               int32_t D, int dtype, cudaStream_t st, int* launches);
cudaError_t launch_tree_commit(const dba_kv_cache& c, const TreePages& pg, int32_t B, int32_t K, int32_t D, int32_t A, int dtype,
                               const int32_t* ctx_len, const int32_t* src, const int32_t* n, cudaStream_t st, int* launches);
struct TreeAdvance {
    int32_t B, rows_in, rows_out, W, ctx_cap, eos_id;
    const uint32_t* masks_in;
    const int32_t *backptr, *token, *ctx_len;
    const float* score;
    int32_t* slot_pos;
    int64_t slot_pos_stride;
    dba_tree_next next;
    uint32_t* status;
};
// Attention over prefixes that sequences share, joined with the rows' own part.
struct TreePrefix {
    TreePages pages;                   // of the prefixes' table
    const int32_t *first, *len;
    int32_t groups, cap;               // prefixes, places that a table row holds
    const void *k, *v, *q;
    void* out;                         // the rows' own part, and then their whole
    float* own_lse;                    // [B, n, H] of the own part, and then of the whole
    const uint32_t* masks;             // null: every row is open
    int32_t B, n, H, K, G, D, W;       // G = H / K query heads per key head
    int64_t q_seq, q_row, q_head, o_seq, o_row, o_head;
    float scale_log2e;
    float* part_o;                     // [2 * grid][item rows][D]: first and last pieces of a block's run that are part of an item
    float* part_ml;                    // [2 * grid][item rows][2]: maximum (powers of two) and sum
    int4* meta;                        // [2 * grid] prefix, key head and block of rows of the piece there (x = -1: none, -2: the block gave up)
    bool joined;                       // the joining kernel follows (prefixes of one tile cannot be cut)
    long long wait_clocks;
    int drop_item;
};
struct TreePrefixPlan { int grid, rows, keys, sm_count; bool tensor; };        // blocks of the kernel, rows of an item, keys of a tile (tensor)
TreePrefixPlan plan_tree_prefix(int dtype, int D, int sm_count);
cudaError_t configure_tree_prefix();
// the tensor-core kernel (tree_prefix_mma.cu); usable where tree_mma_usable
int tree_prefix_mma_rows();
int tree_prefix_mma_keys();
cudaError_t configure_tree_prefix_mma();
cudaError_t launch_tree_prefix_mma(const TreePrefix& a, int grid, cudaStream_t st);
cudaError_t launch_tree_prefix(TreePrefix a, const TreePrefixPlan& plan, int dtype, cudaStream_t st, int* launches);

// The weight that context tokens receive.
struct TreeWeigh {
    TreePages pages;
    const void *k, *q;
    const float *lse, *in;
    float* out;
    const int32_t* ctx_len;
    int32_t B, n, H, K, G, D, A, ctx_cap;
    int64_t q_seq, q_row, q_head, w_seq, w_head;
    float scale_log2e, decay;
    long long wait_clocks;
    int drop_item;
};
cudaError_t configure_tree_weigh();
// the tensor-core kernel (tree_weigh_mma.cu); usable where tree_mma_usable
cudaError_t configure_tree_weigh_mma();
cudaError_t launch_tree_weigh_mma(const TreeWeigh& a, int grid, cudaStream_t st);
cudaError_t launch_tree_weigh(const TreeWeigh& a, int dtype, int sm_count, cudaStream_t st, int* launches);
struct TreeEvict {
    TreePages from, to;
    char *k, *v;
    int64_t layer_bytes;
    int32_t es, layers, B, K, D, A, ctx_cap, sm_count;
    const int32_t* ctx_len;
    dba_tree_evicted e;
};
cudaError_t configure_tree_evict();
cudaError_t launch_tree_evict(const TreeEvict& a, cudaStream_t st, int* launches);
cudaError_t launch_tree_append_norm(const dba_tree_tokens& t, const dba_tree_norm& norm, const TreePages& pg, void* k, void* v, int32_t B, int32_t H,
                                    int32_t K, int32_t D, int dtype, cudaStream_t st, int* launches);
cudaError_t configure_tree_advance();
cudaError_t launch_tree_advance(const TreeAdvance& a, cudaStream_t st, int* launches);

}  // namespace dba
