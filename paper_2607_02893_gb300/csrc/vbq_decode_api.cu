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

vbq_status_t check_sequences(const vbq_sequences* q) {
    if (!q) return fail(VBQ_ERR_ARG, "the sequences must be non-NULL");
    if (q->batch < 0 || q->rows < 0 || q->tokens < 0) return fail(VBQ_ERR_ARG, "batch, rows and tokens must not be negative");
    if (q->batch > 65535) return fail(VBQ_ERR_UNSUPPORTED, "batch must be at most 65535, got %d", q->batch);
    if (q->tokens >= (1ll << 31)) return fail(VBQ_ERR_UNSUPPORTED, "tokens must be below 2^31, got %lld", (long long)q->tokens);
    if (!q->starts && q->tokens != (int64_t)q->batch * q->rows)
        return fail(VBQ_ERR_ARG, "without starts, tokens (%lld) must be batch x rows (%d x %d)", (long long)q->tokens, q->batch, q->rows);
    if (!aligned(q->starts, 4) || !aligned(q->slots, 4) || !aligned(q->fresh, 4))
        return fail(VBQ_ERR_ALIGN, "starts, slots and fresh must be 4-byte aligned");
    return VBQ_OK;
}

vbq_status_t check_slots(int64_t n_slots) {
    if (n_slots < 1 || n_slots > (1ll << 31) - 1)
        return fail(VBQ_ERR_ARG, "n_slots must be in 1..2^31 - 1, got %lld", (long long)n_slots);
    return VBQ_OK;
}

// Rows of `width` elements of `type`, 16-byte aligned, `stride` apart.
vbq_status_t check_strided(const char* name, const void* p, int64_t rows, int64_t width, int64_t stride, int type) {
    if (!p) return fail(VBQ_ERR_ARG, "%s must be non-NULL", name);
    if (rows > 1 && stride < width) return fail(VBQ_ERR_ARG, "%s's row stride is smaller than its row", name);
    if (!aligned(p, 16) || (rows > 1 && stride % (type == VBQ_F32 ? 4 : 8)))
        return fail(VBQ_ERR_ALIGN, "%s's rows must be 16-byte aligned", name);
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

vbq_status_t vbq_causal_conv(const vbq_sequences* seq, const void* x, int64_t x_stride, int type, const float* weight,
                             const float* bias, int taps, int channels, float* state, int64_t n_slots, int silu,
                             uint16_t* out, void* stream) {
    vbq::clear_error();
    vbq_status_t st = check_sequences(seq);
    if (!st) st = check_type(type);
    if (!st) st = check_slots(n_slots);
    if (st) return st;
    if (taps < 2 || taps > vbq::CONV_MAX_TAPS)
        return fail(VBQ_ERR_UNSUPPORTED, "taps must be in 2..%d, got %d", vbq::CONV_MAX_TAPS, taps);
    if (channels < 8 || channels % 8 || channels > (1 << 20))
        return fail(VBQ_ERR_SHAPE, "channels must be a multiple of 8 up to 2^20, got %d", channels);
    if (silu != 0 && silu != 1) return fail(VBQ_ERR_ARG, "silu must be 0 or 1, got %d", silu);
    if (seq->batch == 0 || seq->tokens == 0) return VBQ_OK;
    if (!weight || !state || !out) return fail(VBQ_ERR_ARG, "weight, state and out must be non-NULL");
    st = check_strided("x", x, seq->tokens, channels, x_stride, type);
    if (st) return st;
    if (!aligned(weight, 16) || !aligned(bias, 16) || !aligned(state, 16) || !aligned(out, 16))
        return fail(VBQ_ERR_ALIGN, "weight, bias, state and out must be 16-byte aligned");
    vbq::Conv c = {};
    c.seq = *seq;
    c.x = x; c.x_stride = x_stride; c.f32 = type == VBQ_F32;
    c.weight = weight; c.bias = bias; c.taps = taps; c.channels = channels;
    c.state = state; c.n_slots = n_slots; c.silu = silu; c.out = out;
    VBQ_CUDA(vbq::sequence_status(&c.status));
    VBQ_CUDA(vbq::launch_causal_conv(c, static_cast<cudaStream_t>(stream)));
    return VBQ_OK;
}

vbq_status_t vbq_delta_rule(const vbq_sequences* seq, float* state, int64_t n_slots, const void* q, int64_t q_stride,
                            const void* k, int64_t k_stride, const void* v, int64_t v_stride, int type, int k_heads,
                            int head_k, int heads, int head_v, const void* decay, int64_t decay_stride,
                            const void* beta, int64_t beta_stride, int gate_type, const float* a_log,
                            const float* dt_bias, float scale, int normalize, uint16_t* out, void* stream) {
    vbq::clear_error();
    vbq_status_t st = check_sequences(seq);
    if (!st) st = check_type(type);
    if (!st) st = check_type(gate_type);
    if (!st) st = check_slots(n_slots);
    if (st) return st;
    if (head_k != 64 && head_k != 128) return fail(VBQ_ERR_SHAPE, "head_k must be 64 or 128, got %d", head_k);
    if (head_v != 64 && head_v != 128 && head_v != 256) return fail(VBQ_ERR_SHAPE, "head_v must be 64, 128 or 256, got %d", head_v);
    if (k_heads < 1 || heads < 1 || heads > 1024 || heads % k_heads)
        return fail(VBQ_ERR_SHAPE, "heads (%d) must be a positive multiple of k_heads (%d), at most 1024", heads, k_heads);
    if (!std::isfinite(scale)) return fail(VBQ_ERR_ARG, "scale must be finite");
    if (normalize != 0 && normalize != 1) return fail(VBQ_ERR_ARG, "normalize must be 0 or 1, got %d", normalize);
    if (!a_log != !dt_bias) return fail(VBQ_ERR_ARG, "a_log and dt_bias go together");
    if (seq->tokens > vbq::DELTA_MAX_TOKENS)
        return fail(VBQ_ERR_UNSUPPORTED, "tokens must be at most 2^31 - 64, got %lld", (long long)seq->tokens);
    if (seq->batch == 0 || seq->tokens == 0) return VBQ_OK;
    if (!state || !decay || !beta || !out) return fail(VBQ_ERR_ARG, "state, decay, beta and out must be non-NULL");
    st = check_strided("q", q, seq->tokens, (int64_t)k_heads * head_k, q_stride, type);
    if (!st) st = check_strided("k", k, seq->tokens, (int64_t)k_heads * head_k, k_stride, type);
    if (!st) st = check_strided("v", v, seq->tokens, (int64_t)heads * head_v, v_stride, type);
    if (st) return st;
    if (seq->tokens > 1 && (decay_stride < heads || beta_stride < heads))
        return fail(VBQ_ERR_ARG, "decay's or beta's row stride is smaller than its row");
    const int size = gate_type == VBQ_F32 ? 4 : 2;
    if (!aligned(state, 16) || !aligned(out, 16) || !aligned(decay, size) || !aligned(beta, size) || !aligned(a_log, 4) ||
        !aligned(dt_bias, 4))
        return fail(VBQ_ERR_ALIGN, "state and out must be 16-byte aligned, the gates to their elements");
    vbq::Delta d = {};
    d.seq = *seq;
    d.state = state; d.n_slots = n_slots;
    d.q = q; d.k = k; d.v = v;
    d.q_stride = q_stride; d.k_stride = k_stride; d.v_stride = v_stride; d.f32 = type == VBQ_F32;
    d.k_heads = k_heads; d.head_k = head_k; d.heads = heads; d.head_v = head_v;
    d.decay = decay; d.beta = beta; d.decay_stride = decay_stride; d.beta_stride = beta_stride;
    d.gate_f32 = gate_type == VBQ_F32;
    d.a_log = a_log; d.dt_bias = dt_bias; d.scale = scale; d.normalize = normalize; d.out = out;
    VBQ_CUDA(vbq::sequence_status(&d.status));
    VBQ_CUDA(vbq::launch_delta_rule(d, static_cast<cudaStream_t>(stream)));
    return VBQ_OK;
}

vbq_status_t vbq_gated_norm(const void* x, int64_t x_stride, int x_type, const void* gate, int64_t gate_stride,
                            int gate_type, const float* weight, float eps, int64_t rows, int heads, int width,
                            uint16_t* out, void* stream) {
    vbq::clear_error();
    vbq_status_t st = check_type(x_type);
    if (!st && gate) st = check_type(gate_type);
    if (st) return st;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(VBQ_ERR_ARG, "eps must be finite and not negative");
    if (width < 8 || width % 8 || width > 256) return fail(VBQ_ERR_SHAPE, "width must be a multiple of 8 up to 256, got %d", width);
    if (heads < 1 || heads > 1024) return fail(VBQ_ERR_SHAPE, "heads must be in 1..1024, got %d", heads);
    if (rows < 0) return fail(VBQ_ERR_SHAPE, "rows must not be negative");
    if (rows >= (1ll << 31)) return fail(VBQ_ERR_UNSUPPORTED, "rows must be below 2^31, got %lld", (long long)rows);
    if (rows == 0) return VBQ_OK;
    if (!weight || !out) return fail(VBQ_ERR_ARG, "weight and out must be non-NULL");
    st = check_strided("x", x, rows, (int64_t)heads * width, x_stride, x_type);
    if (!st && gate) st = check_strided("gate", gate, rows, (int64_t)heads * width, gate_stride, gate_type);
    if (st) return st;
    if (!aligned(weight, 16) || !aligned(out, 16)) return fail(VBQ_ERR_ALIGN, "weight and out must be 16-byte aligned");
    vbq::GatedNorm n = {};
    n.x = x; n.gate = gate; n.x_stride = x_stride; n.gate_stride = gate_stride;
    n.x_f32 = x_type == VBQ_F32; n.gate_f32 = gate_type == VBQ_F32;
    n.weight = weight; n.eps = eps; n.rows = rows; n.heads = heads; n.width = width; n.out = out;
    VBQ_CUDA(vbq::launch_gated_norm(n, static_cast<cudaStream_t>(stream)));
    return VBQ_OK;
}

}  // extern "C"
