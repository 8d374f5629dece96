// Host side of the token tree declared in include/dba.h: argument checks, workspace, launches.
#include <new>

#include "tree_internal.h"

using namespace dba;

struct dba_tree {
    dba_tree_config c;
    int device, sm_count;
    cudaStream_t stream;
    int64_t ctx_cap;               // context places a table row holds
    uint32_t* status;
    uint32_t* turns;
    int4* meta;
    float *part_ml, *part_o;
    long long wait_clocks;
    int drop_item;
    uint64_t launches;
};

namespace {

inline int elem_size(int dtype) { return dtype == DBA_F32 ? 4 : 2; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

dba_status check_tree_config(const dba_tree_config* c) {
    if (!c) return DBA_ERR_INVALID_ARG;
    if (c->B < 1 || c->rows < 1 || c->heads < 1 || c->kv_heads < 1 || c->head_dim < 1 || c->page_size < 1 || c->max_pages < 1 || c->words < 0)
        return DBA_ERR_INVALID_ARG;
    if (c->dtype != DBA_F32 && c->dtype != DBA_BF16) return DBA_ERR_INVALID_ARG;
    if (c->heads % c->kv_heads) return DBA_ERR_INVALID_ARG;
    const int64_t places = (int64_t)c->max_pages * c->page_size;
    if (places < 32 * (int64_t)c->words) return DBA_ERR_INVALID_ARG;          // the arena's places are the table's first
    if (c->rows > kTreeMaxRows || c->words > kTreeMaxWords || c->head_dim > kTreeMaxDim) return DBA_ERR_UNSUPPORTED;
    if ((c->head_dim * elem_size(c->dtype)) & 15) return DBA_ERR_UNSUPPORTED;
    if (places >= (int64_t)1 << 31 || (int64_t)c->B * c->rows >= (int64_t)1 << 27 || c->heads > 4096) return DBA_ERR_UNSUPPORTED;
    return DBA_OK;
}

struct TreeCarver {
    char* base;
    size_t off = 0;
    template <typename T> T* take(size_t n) {
        off = (off + 255) / 256 * 256;
        T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
        off += n * sizeof(T);
        return p;
    }
};

size_t carve_tree(dba_tree* h, void* base) {
    TreeCarver cv{(char*)base};
    const dba_tree_config& c = h->c;
    const TreeAttendPlan p = plan_tree_attend(c.dtype, c.rows * (c.heads / c.kv_heads), c.kv_heads, c.head_dim, h->sm_count);
    h->status = cv.take<uint32_t>(64);
    h->turns = cv.take<uint32_t>(kTreeTurns);
    h->meta = cv.take<int4>(p.grid);
    h->part_ml = cv.take<float>((size_t)2 * p.grid * p.rows * 2);
    h->part_o = cv.take<float>((size_t)2 * p.grid * p.rows * c.head_dim);
    return (cv.off + 255) / 256 * 256;
}

dba_status device_of(dba_tree* h) {
    if (cudaGetDevice(&h->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, h->device) != cudaSuccess)
        return DBA_ERR_CUDA;
    return DBA_OK;
}

// A cache and the sequences' tables; *pg is filled where both are usable.
dba_status check_cache(const dba_tree* h, const dba_kv_cache* c, const int32_t* table, int64_t table_stride, TreePages* pg) {
    if (!c || !c->k || !c->v || !table || c->num_pages < 1 || c->layers < 1 || table_stride < h->c.max_pages) return DBA_ERR_INVALID_ARG;
    if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0 || c->layer_stride < 0) return DBA_ERR_INVALID_ARG;
    const int chunk = 16 / elem_size(h->c.dtype);                            // elements in 16 bytes
    if (!aligned16(c->k) || !aligned16(c->v) || c->page_stride % chunk || c->token_stride % chunk || c->head_stride % chunk || c->layer_stride % chunk)
        return DBA_ERR_UNSUPPORTED;
    // kernels count a layer's rows in 16 bytes and 32 bits, of which the highest number stands for no row
    const uint64_t page16 = c->num_pages > 1 ? (uint64_t)(c->page_stride / chunk) : 0, token16 = h->c.page_size > 1 ? (uint64_t)(c->token_stride / chunk) : 0;
    if (page16 >= 0xffffffffu || token16 >= 0xffffffffu) return DBA_ERR_UNSUPPORTED;         // (and the sum of products below 2^64)
    if ((uint64_t)(c->num_pages - 1) * page16 + (uint64_t)(h->c.page_size - 1) * token16 >= 0xffffffffu) return DBA_ERR_UNSUPPORTED;
    // n / d for n < 2^31: with 2^s >= d and m = ceil(2^(31+s) / d), m d - 2^(31+s) < d <= 2^s, so n m / 2^(31+s) exceeds n / d by less than 1 / d
    int s = 1;
    while ((1LL << s) < h->c.page_size) ++s;
    const uint64_t m = (((uint64_t)1 << (31 + s)) + (uint64_t)h->c.page_size - 1) / (uint64_t)h->c.page_size;
    *pg = TreePages{table, table_stride, c->num_pages, h->c.max_pages, h->c.page_size, c->page_stride, c->token_stride, c->head_stride, h->status,
                    (uint32_t)m, s - 1};
    return DBA_OK;
}

inline bool strides_ok(const dba_tree* h, int64_t a, int64_t b, int64_t c) {
    const int es = elem_size(h->c.dtype);
    return !((a * es) & 15) && !((b * es) & 15) && !((c * es) & 15);
}

inline dba_status launched(cudaError_t e) { return e == cudaSuccess ? DBA_OK : DBA_ERR_CUDA; }

}  // namespace

extern "C" {

dba_status dba_tree_workspace_bytes(const dba_tree_config* cfg, size_t* bytes) {
    if (!bytes) return DBA_ERR_INVALID_ARG;
    dba_status st = check_tree_config(cfg);
    if (st != DBA_OK) return st;
    dba_tree tmp{};
    tmp.c = *cfg;
    if ((st = device_of(&tmp)) != DBA_OK) return st;
    *bytes = carve_tree(&tmp, nullptr);
    return DBA_OK;
}

dba_status dba_tree_init(const dba_tree_config* cfg, void* workspace_dev, size_t workspace_bytes, void* cuda_stream, dba_tree** out) {
    if (!out) return DBA_ERR_INVALID_ARG;
    *out = nullptr;
    dba_status st = check_tree_config(cfg);
    if (st != DBA_OK) return st;
    if (!workspace_dev || ((uintptr_t)workspace_dev & 255u)) return DBA_ERR_WORKSPACE;
    dba_tree* h = new (std::nothrow) dba_tree{};
    if (!h) return DBA_ERR_INVALID_ARG;
    h->c = *cfg;
    h->drop_item = -1;
    if ((st = device_of(h)) != DBA_OK) { delete h; return st; }
    if (workspace_bytes < carve_tree(h, workspace_dev)) { delete h; return DBA_ERR_WORKSPACE; }
    h->ctx_cap = (int64_t)cfg->max_pages * cfg->page_size - 32 * (int64_t)cfg->words;
    h->stream = (cudaStream_t)cuda_stream;
    cudaError_t e = configure_tree_attend();
    if (e == cudaSuccess) e = configure_tree_advance();
    if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, 256 + 4 * kTreeTurns, h->stream);     // (the turns lie behind it)
    if (e != cudaSuccess) { delete h; return DBA_ERR_CUDA; }
    *out = h;
    return DBA_OK;
}

dba_status dba_tree_append(dba_tree* h, const dba_tree_tokens* t, const dba_kv_cache* cache, const int32_t* table_dev, int64_t table_stride) {
    if (!h || !t || t->N < 0) return DBA_ERR_INVALID_ARG;
    if (t->N == 0) return DBA_OK;                              // (an empty array has no address)
    if (!t->k || !t->v || !t->place || (t->q && !t->q_out)) return DBA_ERR_INVALID_ARG;
    TreePages pg;
    dba_status st = check_cache(h, cache, table_dev, table_stride, &pg);
    if (st != DBA_OK) return st;
    if (!t->seq && t->N % h->c.B) return DBA_ERR_INVALID_ARG;
    if (t->rot_dim < 0 || t->rot_dim > h->c.head_dim || (t->rot_dim & 1)) return DBA_ERR_INVALID_ARG;
    if (t->position && t->rot_dim > 0 && (!t->cos || !t->sin || t->positions < 1)) return DBA_ERR_INVALID_ARG;
    if (!aligned16(t->k) || !aligned16(t->v) || !strides_ok(h, t->k_token_stride, t->k_head_stride, 0) ||
        !strides_ok(h, t->v_token_stride, t->v_head_stride, 0))
        return DBA_ERR_UNSUPPORTED;
    if (t->q && (!aligned16(t->q) || !aligned16(t->q_out) || !strides_ok(h, t->q_token_stride, t->q_head_stride, 0) ||
                 !strides_ok(h, t->qo_token_stride, t->qo_head_stride, 0)))
        return DBA_ERR_UNSUPPORTED;
    int n = 0;
    dba_tree_tokens tt = *t;
    if (!tt.position || tt.rot_dim == 0) { tt.position = nullptr; tt.rot_dim = 0; tt.cos = tt.sin = nullptr; tt.positions = 0; }
    const cudaError_t e = launch_tree_append(tt, pg, cache->k, cache->v, h->c.B, h->c.heads, h->c.kv_heads, h->c.head_dim, h->c.dtype, h->stream, &n);
    h->launches += n;
    return launched(e);
}

dba_status dba_tree_attend(dba_tree* h, const dba_tree_query* q, const dba_kv_cache* cache, const int32_t* table_dev, int64_t table_stride,
                           const int32_t* ctx_len_dev, const int32_t* masks_dev, const int32_t* top_dev) {
    if (!h || !q || !q->q || !q->out || !ctx_len_dev || q->rows < 1 || q->rows > h->c.rows || q->scale != q->scale) return DBA_ERR_INVALID_ARG;
    if (masks_dev && h->c.words == 0) return DBA_ERR_INVALID_ARG;
    TreeAttend a{};
    dba_status st = check_cache(h, cache, table_dev, table_stride, &a.pages);
    if (st != DBA_OK) return st;
    if (!aligned16(q->q) || !aligned16(q->out) || !strides_ok(h, q->q_seq_stride, q->q_row_stride, q->q_head_stride) ||
        !strides_ok(h, q->out_seq_stride, q->out_row_stride, q->out_head_stride))
        return DBA_ERR_UNSUPPORTED;
    const dba_tree_config& c = h->c;
    a.k = cache->k; a.v = cache->v; a.q = q->q; a.out = q->out; a.lse = q->lse;
    a.ctx_len = ctx_len_dev; a.masks = (const uint32_t*)masks_dev; a.top = top_dev;
    a.B = c.B; a.n = q->rows; a.H = c.heads; a.K = c.kv_heads; a.G = c.heads / c.kv_heads; a.D = c.head_dim;
    a.W = c.words; a.A = 32 * c.words; a.ctx_cap = (int32_t)h->ctx_cap;
    a.q_seq = q->q_seq_stride; a.q_row = q->q_row_stride; a.q_head = q->q_head_stride;
    a.o_seq = q->out_seq_stride; a.o_row = q->out_row_stride; a.o_head = q->out_head_stride;
    a.scale_log2e = (float)((double)q->scale * 1.4426950408889634);
    if (a.scale_log2e == 0.f) a.scale_log2e = 1e-37f;         // all scores alike; the kernels multiply -inf by it
    a.part_o = h->part_o; a.part_ml = h->part_ml; a.meta = h->meta; a.turns = h->turns;
    a.wait_clocks = h->wait_clocks; a.drop_item = h->drop_item;
    int n = 0;
    // (planned for the configuration's rows: the workspace was sized for that)
    const TreeAttendPlan plan = plan_tree_attend(c.dtype, c.rows * a.G, c.kv_heads, c.head_dim, h->sm_count);
    a.item_heads = plan.item_heads;
    const cudaError_t e = launch_tree_attend(a, plan, c.dtype, h->stream, &n);
    h->launches += n;
    return launched(e);
}

dba_status dba_tree_advance(dba_tree* h, int32_t rows_in, const int32_t* masks_in_dev, int32_t rows_out, const int32_t* backptr_dev,
                            const float* score_dev, const int32_t* token_dev, int32_t eos_id, int32_t* slot_pos_dev,
                            int64_t slot_pos_stride, const int32_t* ctx_len_dev, const dba_tree_next* next) {
    if (!h || !masks_in_dev || !backptr_dev || !slot_pos_dev || !ctx_len_dev || !next || !next->masks || rows_in < 1 || rows_out < 1)
        return DBA_ERR_INVALID_ARG;
    if (h->c.words == 0 || rows_in > h->c.rows || rows_out > h->c.rows || slot_pos_stride < 32 * h->c.words) return DBA_ERR_INVALID_ARG;
    // one sequence's new masks must not be another's old ones
    const uintptr_t in = (uintptr_t)masks_in_dev, out = (uintptr_t)next->masks, row = (uintptr_t)h->c.B * h->c.words * sizeof(int32_t);
    if (in < out + rows_out * row && out < in + rows_in * row) return DBA_ERR_INVALID_ARG;
    TreeAdvance a{};
    a.B = h->c.B; a.rows_in = rows_in; a.rows_out = rows_out; a.W = h->c.words; a.ctx_cap = (int32_t)h->ctx_cap; a.eos_id = eos_id;
    a.masks_in = (const uint32_t*)masks_in_dev; a.backptr = backptr_dev; a.token = token_dev; a.ctx_len = ctx_len_dev; a.score = score_dev;
    a.slot_pos = slot_pos_dev; a.slot_pos_stride = slot_pos_stride; a.next = *next; a.status = h->status;
    int n = 0;
    const cudaError_t e = launch_tree_advance(a, h->stream, &n);
    h->launches += n;
    return launched(e);
}

dba_status dba_tree_commit(dba_tree* h, const dba_kv_cache* cache, const int32_t* table_dev, int64_t table_stride, const int32_t* ctx_len_dev,
                           const int32_t* src_dev, const int32_t* n_dev) {
    if (!h || !ctx_len_dev || !src_dev || !n_dev || h->c.words == 0) return DBA_ERR_INVALID_ARG;
    TreePages pg;
    dba_status st = check_cache(h, cache, table_dev, table_stride, &pg);
    if (st != DBA_OK) return st;
    if (cache->layers > 32767) return DBA_ERR_UNSUPPORTED;         // two blocks a layer in a grid's second dimension
    int n = 0;
    const cudaError_t e = launch_tree_commit(*cache, pg, h->c.B, h->c.kv_heads, h->c.head_dim, 32 * h->c.words, h->c.dtype, ctx_len_dev, src_dev,
                                             n_dev, h->stream, &n);
    h->launches += n;
    return launched(e);
}

dba_status dba_tree_status(dba_tree* h, uint32_t* bits) {
    if (!h || !bits) return DBA_ERR_INVALID_ARG;
    uint32_t word = 0;
    cudaError_t e = cudaMemcpyAsync(&word, h->status, 4, cudaMemcpyDeviceToHost, h->stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, 4, h->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return DBA_ERR_CUDA;
    *bits = word;
    return DBA_OK;
}

uint64_t dba_tree_launch_count(const dba_tree* h) { return h ? h->launches : 0; }

dba_status dba_tree_test_hook(dba_tree* h, int64_t wait_clocks, int32_t drop_item) {
    if (!h) return DBA_ERR_INVALID_ARG;
    h->wait_clocks = wait_clocks > 0 ? (long long)wait_clocks : 0;
    h->drop_item = drop_item >= 0 ? drop_item : -1;
    return DBA_OK;
}

void dba_tree_destroy(dba_tree* h) { delete h; }

}  // extern "C"
