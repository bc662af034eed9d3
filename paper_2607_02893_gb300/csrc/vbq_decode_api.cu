// vbq_decode_api.cu — the C ABI of the decode step's other operators
// (include/vbq.h): argument checks and dispatch on the caller's stream.
#include <cmath>

#include "vbq_decode.h"

namespace {

using vbq::fail;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

#define VBQ_CUDA(call)                                                                                       \
    do {                                                                                                     \
        cudaError_t e_ = (call);                                                                             \
        if (e_ != cudaSuccess)                                                                               \
            return fail(e_ == cudaErrorMemoryAllocation ? VBQ_ERR_NOMEM : VBQ_ERR_CUDA, "%s: %s (%s:%d)",    \
                        #call, cudaGetErrorString(e_), __FILE__, __LINE__);                                  \
    } while (0)

vbq_status_t check_shape(int kv_heads, int head_dim) {
    if (kv_heads < 1 || kv_heads > 1024) return fail(VBQ_ERR_SHAPE, "kv_heads must be in 1..1024, got %d", kv_heads);
    if (head_dim != 64 && head_dim != 128 && head_dim != 256)
        return fail(VBQ_ERR_SHAPE, "head_dim must be 64, 128 or 256, got %d", head_dim);
    return VBQ_OK;
}

vbq_status_t check_cache(const vbq_kv_cache* c) {
    if (!c || !c->pages) return fail(VBQ_ERR_ARG, "the cache and its pages must be non-NULL");
    if (c->n_pages < 1 || c->n_pages > (1ll << 31) - 1)
        return fail(VBQ_ERR_ARG, "n_pages must be in 1..2^31 - 1, got %lld", (long long)c->n_pages);
    const vbq_status_t st = check_shape(c->kv_heads, c->head_dim);
    if (st) return st;
    if (!aligned(c->pages, 16)) return fail(VBQ_ERR_ALIGN, "the cache's pages must be 16-byte aligned");
    return VBQ_OK;
}

// The parts of a cache call: the table and the rows.
vbq_status_t check_rows(const int32_t* table, int64_t table_stride, int table_pages, const int32_t* pos, int batch,
                        int rows) {
    if (batch < 0 || rows < 0) return fail(VBQ_ERR_ARG, "batch and rows must not be negative");
    if ((int64_t)batch * rows >= (1ll << 31)) return fail(VBQ_ERR_UNSUPPORTED, "batch x rows must be below 2^31");
    if (batch == 0 || rows == 0) return VBQ_OK;
    if (!table || !pos) return fail(VBQ_ERR_ARG, "table and pos must be non-NULL");
    if (table_pages < 1 || table_stride < 0) return fail(VBQ_ERR_ARG, "table_pages must be positive, table_stride not negative");
    if (!aligned(table, 4) || !aligned(pos, 4)) return fail(VBQ_ERR_ALIGN, "table and pos must be 4-byte aligned");
    return VBQ_OK;
}

vbq_status_t check_type(int type) {
    if (type != VBQ_BF16 && type != VBQ_F32) return fail(VBQ_ERR_ARG, "type must be VBQ_BF16 or VBQ_F32, got %d", type);
    return VBQ_OK;
}

vbq::KvView view_of(const vbq_kv_cache* c, const int32_t* table, int64_t table_stride, int table_pages) {
    vbq::KvView v;
    v.pages = static_cast<uint8_t*>(c->pages);
    v.table = table;
    v.table_stride = table_stride;
    v.n_pages = c->n_pages;
    v.table_pages = table_pages;
    v.kv_heads = c->kv_heads;
    v.head_dim = c->head_dim;
    return v;
}

vbq_status_t check_heads(int heads, int kv_heads) {
    if (heads < 1 || heads % kv_heads != 0)
        return fail(VBQ_ERR_SHAPE, "heads (%d) must be a positive multiple of kv_heads (%d)", heads, kv_heads);
    if (heads / kv_heads > 64)
        return fail(VBQ_ERR_UNSUPPORTED, "at most 64 query heads per key-value head, got %d", heads / kv_heads);
    return VBQ_OK;
}

vbq_status_t check_attend(const vbq_kv_cache* c, int batch, int rows, int heads) {
    const vbq_status_t st = check_heads(heads, c->kv_heads);
    if (st) return st;
    if (batch > vbq::KV_MAX_BATCH) return fail(VBQ_ERR_UNSUPPORTED, "batch must be at most %d, got %d", vbq::KV_MAX_BATCH, batch);
    if (rows < 1 || rows > vbq::KV_MAX_ROWS)
        return fail(VBQ_ERR_UNSUPPORTED, "rows must be in 1..%d, got %d", vbq::KV_MAX_ROWS, rows);
    return VBQ_OK;
}

}  // namespace

extern "C" {

vbq_status_t vbq_kv_page_bytes(int kv_heads, int head_dim, size_t* bytes) {
    vbq::clear_error();
    if (!bytes) return fail(VBQ_ERR_ARG, "bytes is NULL");
    const vbq_status_t st = check_shape(kv_heads, head_dim);
    if (st) return st;
    *bytes = (size_t)kv_heads * (size_t)vbq::kv_blob_bytes(head_dim);
    return VBQ_OK;
}

vbq_status_t vbq_kv_append(const vbq_kv_cache* cache, const int32_t* table, int64_t table_stride, int table_pages,
                           const int32_t* pos, int batch, int rows, const void* q, int64_t q_stride, int heads,
                           const void* k, int64_t k_stride, const void* v, int64_t v_stride, int type,
                           const float* rot_cos, const float* rot_sin, int rot_dim, int64_t rot_rows,
                           uint16_t* q_out, void* stream) {
    vbq::clear_error();
    vbq_status_t st = check_cache(cache);
    if (!st) st = check_type(type);
    if (!st) st = check_rows(table, table_stride, table_pages, pos, batch, rows);
    if (st) return st;
    if (batch == 0 || rows == 0) return VBQ_OK;
    if (!k || !v) return fail(VBQ_ERR_ARG, "k and v must be non-NULL");
    if (!q != !q_out) return fail(VBQ_ERR_ARG, "q and q_out go together");
    if (q && (heads < 1 || heads > (1 << 20))) return fail(VBQ_ERR_SHAPE, "heads must be in 1..2^20, got %d", heads);
    if (!rot_cos != !rot_sin) return fail(VBQ_ERR_ARG, "rot_cos and rot_sin go together");
    if (rot_cos) {
        if (rot_dim < 16 || rot_dim > cache->head_dim || rot_dim % 16 != 0)
            return fail(VBQ_ERR_SHAPE, "rot_dim must be a multiple of 16 up to head_dim, got %d", rot_dim);
        if (rot_rows < 1) return fail(VBQ_ERR_ARG, "rot_rows must be positive");
    }
    const int64_t per = 16 / (type == VBQ_F32 ? 4 : 2), kvw = (int64_t)cache->kv_heads * cache->head_dim;
    const bool many = (int64_t)batch * rows > 1;
    if (many && (k_stride < kvw || v_stride < kvw || (q && q_stride < (int64_t)heads * cache->head_dim)))
        return fail(VBQ_ERR_ARG, "a row stride is smaller than its row");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(rot_cos, 16) ||
        !aligned(rot_sin, 16) || (many && (k_stride % per || v_stride % per || (q && q_stride % per))))
        return fail(VBQ_ERR_ALIGN, "q, k, v, their rows, q_out, rot_cos and rot_sin must be 16-byte aligned");
    vbq::KvAppend a = {};
    a.pos = pos; a.batch = batch; a.rows = rows;
    a.q = q; a.k = k; a.v = v;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.heads = heads; a.f32 = type == VBQ_F32;
    a.cos = rot_cos; a.sin = rot_sin; a.rot_dim = rot_cos ? rot_dim : 0; a.rot_rows = rot_rows;
    a.q_out = q_out;
    VBQ_CUDA(vbq::launch_kv_append(view_of(cache, table, table_stride, table_pages), a, static_cast<cudaStream_t>(stream)));
    return VBQ_OK;
}

vbq_status_t vbq_kv_read(const vbq_kv_cache* cache, const int32_t* table, int64_t table_stride, int table_pages,
                         const int32_t* pos, int batch, int rows, float* k_out, float* v_out, void* stream) {
    vbq::clear_error();
    vbq_status_t st = check_cache(cache);
    if (!st) st = check_rows(table, table_stride, table_pages, pos, batch, rows);
    if (st) return st;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return fail(VBQ_ERR_ALIGN, "k_out and v_out must be 16-byte aligned");
    if (batch == 0 || rows == 0 || (!k_out && !v_out)) return VBQ_OK;
    VBQ_CUDA(vbq::launch_kv_read(view_of(cache, table, table_stride, table_pages), pos, batch, rows, k_out, v_out,
                                 static_cast<cudaStream_t>(stream)));
    return VBQ_OK;
}

vbq_status_t vbq_kv_workspace_bytes(const vbq_kv_cache* cache, int batch, int rows, int heads, size_t* bytes) {
    vbq::clear_error();
    if (!bytes) return fail(VBQ_ERR_ARG, "bytes is NULL");
    vbq_status_t st = check_cache(cache);
    if (!st && batch < 0) st = fail(VBQ_ERR_ARG, "batch must not be negative");
    if (!st) st = check_attend(cache, batch, rows, heads);
    if (st) return st;
    int dev = 0, sms = 0;
    VBQ_CUDA(cudaGetDevice(&dev));
    VBQ_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    *bytes = vbq::kv_workspace_bytes(batch, rows, heads, cache->kv_heads, sms);
    return VBQ_OK;
}

vbq_status_t vbq_kv_attend(const vbq_kv_cache* cache, const int32_t* table, int64_t table_stride, int table_pages,
                           const int32_t* pos, int batch, int rows, const uint16_t* q, int heads, float scale,
                           int window, uint16_t* out, void* workspace, size_t workspace_bytes, void* stream) {
    vbq::clear_error();
    vbq_status_t st = check_cache(cache);
    if (!st) st = check_rows(table, table_stride, table_pages, pos, batch, rows);
    if (!st) st = check_attend(cache, batch, rows, heads);
    if (st) return st;
    if (!std::isfinite(scale)) return fail(VBQ_ERR_ARG, "scale must be finite");
    if (window < 0) return fail(VBQ_ERR_ARG, "window must not be negative");
    if (batch == 0) return VBQ_OK;
    if (!q || !out || !workspace) return fail(VBQ_ERR_ARG, "q, out and workspace must be non-NULL");
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16))
        return fail(VBQ_ERR_ALIGN, "q, out and workspace must be 16-byte aligned");
    vbq::KvAttend a = {};
    a.pos = pos; a.batch = batch; a.rows = rows;
    a.q = q; a.heads = heads; a.scale = scale; a.window = window;
    a.out = out; a.workspace = workspace; a.workspace_bytes = workspace_bytes;
    int dev = 0, sms = 0;
    VBQ_CUDA(cudaGetDevice(&dev));
    VBQ_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const size_t need = vbq::kv_workspace_bytes(batch, rows, heads, cache->kv_heads, sms);
    if (workspace_bytes < need)
        return fail(VBQ_ERR_ARG, "the workspace has %zu bytes, this call needs %zu", workspace_bytes, need);
    VBQ_CUDA(vbq::launch_kv_attend(view_of(cache, table, table_stride, table_pages), a, static_cast<cudaStream_t>(stream)));
    return VBQ_OK;
}

vbq_status_t vbq_residual_norm(const void* x, int x_type, const void* residual, int residual_type,
                               const float* weight, float eps, int64_t rows, int width, uint16_t* out,
                               void* residual_out, void* stream) {
    vbq::clear_error();
    vbq_status_t st = check_type(x_type);
    if (!st && residual) st = check_type(residual_type);
    if (st) return st;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(VBQ_ERR_ARG, "eps must be finite and not negative");
    if (rows < 0 || width < 1) return fail(VBQ_ERR_SHAPE, "need rows >= 0 and width >= 1");
    if (width > (1 << 20) || rows > (1ll << 40) / width) return fail(VBQ_ERR_UNSUPPORTED, "width above 2^20 or rows x width above 2^40");
    if (rows == 0) return VBQ_OK;
    if (!x || !weight || !out) return fail(VBQ_ERR_ARG, "x, weight and out must be non-NULL");
    if (!residual != !residual_out) return fail(VBQ_ERR_ARG, "residual and residual_out go together");
    if (!aligned(x, 16) || !aligned(residual, 16) || !aligned(weight, 16) || !aligned(out, 16) || !aligned(residual_out, 16))
        return fail(VBQ_ERR_ALIGN, "device arrays must be 16-byte aligned");
    vbq::Norm n = {};
    n.x = x; n.residual = residual;
    n.x_f32 = x_type == VBQ_F32; n.residual_f32 = residual_type == VBQ_F32;
    n.weight = weight; n.eps = eps; n.rows = rows; n.width = width; n.out = out; n.residual_out = residual_out;
    VBQ_CUDA(vbq::launch_residual_norm(n, static_cast<cudaStream_t>(stream)));
    return VBQ_OK;
}

vbq_status_t vbq_sample(const void* logits, int64_t stride, int type, int batch, int vocab, const float* temperature,
                        const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                        int32_t* tokens, float* probs, int32_t* kept, void* stream) {
    vbq::clear_error();
    const vbq_status_t st = check_type(type);
    if (st) return st;
    if (batch < 0) return fail(VBQ_ERR_ARG, "batch must not be negative");
    if (batch > 65535) return fail(VBQ_ERR_UNSUPPORTED, "batch must be at most 65535, got %d", batch);
    if (vocab < 1) return fail(VBQ_ERR_SHAPE, "vocab must be positive");
    if (vocab > vbq::SAMPLE_MAX_VOCAB) return fail(VBQ_ERR_UNSUPPORTED, "vocab must be at most %d, got %d", vbq::SAMPLE_MAX_VOCAB, vocab);
    if (batch == 0) return VBQ_OK;
    if (!logits || !temperature || !top_k || !top_p || !min_p || !u || !tokens)
        return fail(VBQ_ERR_ARG, "logits, the per-row parameters and tokens must be non-NULL");
    if (batch > 1 && stride < vocab) return fail(VBQ_ERR_ARG, "stride %lld is smaller than vocab", (long long)stride);
    if (!aligned(logits, type == VBQ_F32 ? 4 : 2) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
        !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(u, 4) || !aligned(tokens, 4) || !aligned(probs, 4) ||
        !aligned(kept, 4))
        return fail(VBQ_ERR_ALIGN, "an array is not aligned to its elements");
    vbq::Sample p = {};
    p.logits = logits; p.stride = stride; p.f32 = type == VBQ_F32;
    p.batch = batch; p.vocab = vocab;
    p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.u = u;
    p.tokens = tokens; p.probs = probs; p.kept = kept;
    VBQ_CUDA(vbq::launch_sample(p, static_cast<cudaStream_t>(stream)));
    return VBQ_OK;
}

}  // extern "C"
