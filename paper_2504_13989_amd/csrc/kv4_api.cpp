// C ABI of the 4-bit paged cache: argument checks and dispatch.
#include <atomic>
#include <cmath>
#include <utility>

#include "kv4_layout.h"

namespace {

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// 0 where there is no such page.
size_t page_bytes(int kv_heads, int head_dim, int page_size) {
    if (kv_heads < 1 || kv_heads > RQ_KV4_MAX_HEADS || (head_dim != 64 && head_dim != 128)) return 0;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1))) return 0;
    return (size_t)kv_heads * page_size * (head_dim + 8);
}

int cache_of(const rq_kv4_t* c, rq::Kv4* out) {
    if (!c || c->pages < 0 || c->pages > INT32_MAX) return RQ_ERR_ARG;
    const size_t bytes = page_bytes(c->kv_heads, c->head_dim, c->page_size);
    if (!bytes || (c->pages > 0 && !c->data) || !aligned(c->data, 16)) return RQ_ERR_ARG;
    *out = rq::Kv4{static_cast<uint8_t*>(c->data), c->pages, (int64_t)bytes, c->kv_heads, c->head_dim, __builtin_ctz(c->page_size)};
    return RQ_OK;
}

// The rotation of the heads: none, or the Sylvester matrix of their width.
bool rotation_ok(const rq_hadamard_t* h, int head_dim) { return !h || (h->f.n == head_dim && h->f.p == 1); }

// Compute units of the current device, asked for once.
int num_cu() {
    static std::atomic<int> known[64];
    int dev = -1, n = 0;
    if (hipGetDevice(&dev) != hipSuccess) {
        (void)hipGetLastError();
        return 0;
    }
    if (dev >= 0 && dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) {
        (void)hipGetLastError();
        return 0;
    }
    if (dev >= 0 && dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

const int32_t kRagged = 0;                        // q_start of a call that is only planned: asked for being there

// The checks that rq_kv4_attention and its workspace share.
int shape_ok(const rq::Kv4& c, int64_t tokens, int heads, int batch, int window, int64_t max_len) {
    if (tokens < 0 || tokens > (1 << 24) || heads < 1 || heads % c.kv_heads != 0 || heads / c.kv_heads > 256) return RQ_ERR_ARG;
    if (batch < 0 || batch > (1 << 20) || window < 0 || max_len < 0 || max_len > (1 << 30)) return RQ_ERR_ARG;
    // row tiles and rows are counted in 32 bits
    if (tokens * (heads / c.kv_heads) > INT32_MAX / 2) return RQ_ERR_ARG;
    return RQ_OK;
}

// Rows of weights [..][batch][kv_heads][n] that a call writes: none of them over another.
bool rows_apart(int64_t n, int64_t outer, int64_t outer_stride, int64_t seqs, int64_t seq_stride, int64_t heads, int64_t head_stride) {
    // strides from the smallest on, each at least what the ones below it span
    struct Dim {
        int64_t size, stride;
    } d[3] = {{heads, head_stride}, {seqs, seq_stride}, {outer, outer_stride}};
    for (int i = 1; i < 3; ++i)
        for (int j = i; j > 0 && d[j].stride < d[j - 1].stride; --j) std::swap(d[j], d[j - 1]);
    int64_t span = n;
    for (const Dim& x : d) {
        if (x.size <= 1) continue;
        if (x.stride < span || x.stride > ((int64_t)1 << 60) / x.size) return false;
        span += (x.size - 1) * x.stride;
    }
    return true;
}

// A window that reaches back over the longest sequence hides nothing: 0, as without one.  Others are below 2^30, so that a position (above
// -2^24 where there are more queries than positions) less a window fits 32 bits.
int window_of(int window, int64_t max_len) { return window < max_len ? window : 0; }

}  // namespace

extern "C" {

size_t rq_kv4_page_bytes(int kv_heads, int head_dim, int page_size) { return page_bytes(kv_heads, head_dim, page_size); }

int rq_kv4_append(const rq_hadamard_t* h, const rq_kv4_t* cache, const void* K, const void* V, int dtype, int64_t tokens,
                  int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                  const int64_t* slots, float clip, void* stream) {
    rq::Kv4 c;
    const int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if (!rotation_ok(h, c.head_dim) || (dtype != RQ_BF16 && dtype != RQ_F32 && dtype != RQ_F16)) return RQ_ERR_ARG;
    if (tokens < 0 || !(clip > 0.0f && clip <= 1.0f)) return RQ_ERR_ARG;
    if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0) return RQ_ERR_ARG;
    if (tokens == 0) return RQ_OK;
    const size_t size = dtype == RQ_F32 ? 4 : 2;
    if (!K || !V || !slots || !aligned(K, size) || !aligned(V, size) || !aligned(slots, 8)) return RQ_ERR_ARG;
    return rq::kv4_append(c, rq::Kv4Append{K, V, dtype, tokens, k_token_stride, k_head_stride, v_token_stride, v_head_stride, slots, clip, h != nullptr},
                          static_cast<hipStream_t>(stream));
}

int rq_kv4_read(const rq_hadamard_t* h, const rq_kv4_t* cache, const int64_t* slots, int64_t rows, void* K, void* V, int out_dtype,
                void* stream) {
    rq::Kv4 c;
    const int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if (!rotation_ok(h, c.head_dim) || (out_dtype != RQ_BF16 && out_dtype != RQ_F32 && out_dtype != RQ_F16) || rows < 0) return RQ_ERR_ARG;
    if (rows == 0) return RQ_OK;
    if (!K || !V || !slots || !aligned(K, 16) || !aligned(V, 16) || !aligned(slots, 8)) return RQ_ERR_ARG;
    return rq::kv4_read(c, rq::Kv4Read{K, V, out_dtype, rows, slots, h != nullptr}, static_cast<hipStream_t>(stream));
}

int rq_kv4_copy_pages(const rq_kv4_t* cache, int layers, int64_t layer_stride, const int32_t* src, const int32_t* dst, int64_t pairs,
                      void* stream) {
    rq::Kv4 c;
    const int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if (layers < 0 || layers > (1 << 16) || pairs < 0 || pairs > INT32_MAX) return RQ_ERR_ARG;
    if (layers > 1 && (layer_stride < c.pages * c.page_bytes || layer_stride % 16 != 0)) return RQ_ERR_ARG;
    if (layers == 0 || pairs == 0) return RQ_OK;
    if (!src || !dst || !aligned(src, 4) || !aligned(dst, 4)) return RQ_ERR_ARG;
    // (a workgroup for every 16 KB, of which a grid holds fewer than 2^35)
    if ((double)layers * (double)pairs * (double)(c.page_bytes / 16384 + 1) >= (double)((int64_t)1 << 35)) return RQ_ERR_ARG;
    return rq::kv4_copy_pages(c, layers, layer_stride, src, dst, pairs, static_cast<hipStream_t>(stream));
}

size_t rq_kv4_attention_workspace(const rq_kv4_t* cache, int64_t tokens, int heads, int batch, int decode, int window, int64_t max_len) {
    rq::Kv4 c;
    if (cache_of(cache, &c) != RQ_OK || shape_ok(c, tokens, heads, batch, window, max_len) != RQ_OK || tokens == 0 || batch == 0) return 0;
    const int cu = num_cu();
    if (cu <= 0) return 0;
    rq::Kv4Attention a{};
    a.tokens = (int)tokens;
    a.heads = heads;
    a.batch = batch;
    a.window = window_of(window, max_len);
    a.max_len = max_len;
    a.q_start = decode ? nullptr : &kRagged;
    return rq::kv4_attention_workspace(c, a, cu);
}

int rq_kv4_attention_plan(const rq_kv4_t* cache, int dtype, int64_t tokens, int heads, int batch, int decode, int causal, int window,
                          int64_t max_len, int compute_units, rq_kv4_plan_t* plan) {
    rq::Kv4 c;
    int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if ((rc = shape_ok(c, tokens, heads, batch, window, max_len)) != RQ_OK) return rc;
    if (!plan || (dtype != RQ_BF16 && dtype != RQ_F16) || (causal != 0 && causal != 1) || compute_units < 0) return RQ_ERR_ARG;
    if (tokens == 0 || batch == 0 || (decode && tokens != batch)) return RQ_ERR_ARG;
    const int cu = compute_units ? compute_units : num_cu();
    if (cu <= 0) return RQ_ERR_HIP;
    rq::Kv4Attention a{};
    a.dtype = dtype;
    a.tokens = (int)tokens;
    a.heads = heads;
    a.batch = batch;
    a.causal = causal != 0;
    a.window = window_of(window, max_len);
    a.max_len = max_len;
    a.q_start = decode ? nullptr : &kRagged;
    *plan = rq::kv4_attention_plan(c, a, cu);
    return RQ_OK;
}

int rq_kv4_attention(const rq_hadamard_t* h, const rq_kv4_t* cache, const void* Q, int dtype, int64_t tokens, int heads,
                     int64_t q_token_stride, int64_t q_head_stride, const int32_t* table, int batch, int width, const int32_t* kv_lens,
                     const int32_t* q_start, float scale, int causal, int window, int64_t max_len, void* O, int64_t o_token_stride,
                     int64_t o_head_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    rq::Kv4 c;
    int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if (!rotation_ok(h, c.head_dim) || (dtype != RQ_BF16 && dtype != RQ_F16)) return RQ_ERR_ARG;
    if ((rc = shape_ok(c, tokens, heads, batch, window, max_len)) != RQ_OK) return rc;
    if (width < 0 || (causal != 0 && causal != 1) || !(scale > 0.0f) || !std::isfinite(scale)) return RQ_ERR_ARG;
    if (q_token_stride < 0 || q_head_stride < 0 || o_token_stride < 0 || o_head_stride < 0) return RQ_ERR_ARG;
    // (rows of results that share elements would be written over each other)
    if ((tokens > 1 && o_token_stride < c.head_dim) || (heads > 1 && o_head_stride < c.head_dim)) return RQ_ERR_ARG;
    if (!q_start && tokens != batch) return RQ_ERR_ARG;                    // a token a sequence
    if (tokens == 0) return RQ_OK;
    if (batch == 0 || !Q || !O || !kv_lens || (width > 0 && (!table || c.pages == 0))) return RQ_ERR_ARG;
    if (!aligned(Q, 2) || !aligned(O, 2) || !aligned(table, 4) || !aligned(kv_lens, 4) || !aligned(q_start, 4) || !aligned(lse, 4)) return RQ_ERR_ARG;
    if (max_len > (int64_t)width << c.page_shift) return RQ_ERR_ARG;
    const rq::Kv4Attention a{Q, O, lse, dtype, (int)tokens, heads, batch, width, q_token_stride, q_head_stride, o_token_stride, o_head_stride,
                             table, kv_lens, q_start, scale, causal != 0, h != nullptr, window_of(window, max_len), max_len};
    const int cu = num_cu();
    if (cu <= 0) return RQ_ERR_HIP;
    const size_t need = rq::kv4_attention_workspace(c, a, cu);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return RQ_ERR_ARG;
    return rq::kv4_attention(c, a, cu, static_cast<float*>(workspace), static_cast<hipStream_t>(stream));
}

size_t rq_kv4_attention_weights_workspace(const rq_kv4_t* cache, int64_t tokens, int heads, int batch, int decode, int window, int64_t max_len) {
    rq::Kv4 c;
    if (cache_of(cache, &c) != RQ_OK || shape_ok(c, tokens, heads, batch, window, max_len) != RQ_OK || tokens == 0 || batch == 0 || max_len == 0) return 0;
    const int cu = num_cu();
    if (cu <= 0) return 0;
    rq::Kv4Attention a{};
    a.tokens = (int)tokens;
    a.heads = heads;
    a.batch = batch;
    a.window = window_of(window, max_len);
    a.max_len = max_len;
    a.q_start = decode ? nullptr : &kRagged;
    return rq::kv4_weights_workspace(c, a, cu);
}

int rq_kv4_attention_weights(const rq_hadamard_t* h, const rq_kv4_t* cache, const void* Q, int dtype, int64_t tokens, int heads,
                             int64_t q_token_stride, int64_t q_head_stride, const float* lse, const int32_t* table, int batch, int width,
                             const int32_t* kv_lens, const int32_t* q_start, float scale, int causal, int window, int64_t max_len, float decay,
                             float* weights, int64_t w_seq_stride, int64_t w_head_stride, void* workspace, size_t workspace_bytes, void* stream) {
    rq::Kv4 c;
    int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if (!rotation_ok(h, c.head_dim) || (dtype != RQ_BF16 && dtype != RQ_F16)) return RQ_ERR_ARG;
    if ((rc = shape_ok(c, tokens, heads, batch, window, max_len)) != RQ_OK) return rc;
    if (width < 0 || (causal != 0 && causal != 1) || !(scale > 0.0f) || !std::isfinite(scale) || !(decay >= 0.0f && decay <= 1.0f)) return RQ_ERR_ARG;
    if (q_token_stride < 0 || q_head_stride < 0 || w_seq_stride < 0 || w_head_stride < 0) return RQ_ERR_ARG;
    // (a workgroup for every 256 positions, counted in 32 bits)
    if (batch * (max_len / 256 + 1) > (1 << 30)) return RQ_ERR_ARG;
    if (!rows_apart(max_len, 1, 0, batch, w_seq_stride, c.kv_heads, w_head_stride)) return RQ_ERR_ARG;
    if (!q_start && tokens != batch) return RQ_ERR_ARG;                    // a token a sequence
    if (max_len > (int64_t)width << c.page_shift) return RQ_ERR_ARG;
    if (batch == 0 || max_len == 0) return RQ_OK;
    if (!kv_lens || !table || c.pages == 0 || !weights || (tokens > 0 && (!Q || !lse))) return RQ_ERR_ARG;
    if (!aligned(Q, 2) || !aligned(lse, 4) || !aligned(table, 4) || !aligned(kv_lens, 4) || !aligned(q_start, 4) || !aligned(weights, 4)) return RQ_ERR_ARG;
    const rq::Kv4Attention a{Q, nullptr, const_cast<float*>(lse), dtype, (int)tokens, heads, batch, width, q_token_stride, q_head_stride, 0, 0,
                             table, kv_lens, q_start, scale, causal != 0, h != nullptr, window_of(window, max_len), max_len};
    const int cu = num_cu();
    if (cu <= 0) return RQ_ERR_HIP;
    const size_t need = tokens ? rq::kv4_weights_workspace(c, a, cu) : 0;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return RQ_ERR_ARG;
    return rq::kv4_weights(c, rq::Kv4Weights{a, weights, w_seq_stride, w_head_stride, decay}, cu, workspace, static_cast<hipStream_t>(stream));
}

int rq_kv4_select(const float* weights, int layers, int batch, int kv_heads, int64_t n, int64_t w_layer_stride, int64_t w_seq_stride,
                  int64_t w_head_stride, const int32_t* kv_lens, int64_t keep, int64_t sinks, int64_t recent, int32_t* index, void* stream) {
    if (layers < 0 || layers > (1 << 16) || batch < 0 || batch > (1 << 20) || kv_heads < 1 || kv_heads > RQ_KV4_MAX_HEADS) return RQ_ERR_ARG;
    if (n < 0 || n > (1 << 30) || keep < 0 || keep > (1 << 30) || sinks < 0 || recent < 0 || recent > keep || sinks > keep - recent) return RQ_ERR_ARG;
    if (w_layer_stride < 0 || w_seq_stride < 0 || w_head_stride < 0) return RQ_ERR_ARG;
    if ((int64_t)layers * batch * kv_heads >= (int64_t)1 << 31) return RQ_ERR_ARG;
    if (layers == 0 || batch == 0 || keep == 0) return RQ_OK;
    if ((n > 0 && !weights) || !kv_lens || !index || !aligned(weights, 4) || !aligned(kv_lens, 4) || !aligned(index, 4)) return RQ_ERR_ARG;
    return rq::kv4_select(rq::Kv4Select{weights, w_layer_stride, w_seq_stride, w_head_stride, kv_lens, layers, batch, kv_heads, (int)n, (int)keep,
                                        (int)sinks, (int)recent, index}, static_cast<hipStream_t>(stream));
}

int rq_kv4_evict(const rq_kv4_t* cache, int layers, int64_t layer_stride, const int32_t* index, int64_t keep, const int32_t* table, int batch, int width,
                 const int32_t* new_table, int new_width, float* weights, int64_t n, int64_t w_layer_stride, int64_t w_seq_stride,
                 int64_t w_head_stride, void* stream) {
    rq::Kv4 c;
    const int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if (layers < 0 || layers > (1 << 16) || batch < 0 || batch > (1 << 20) || keep < 0 || keep > (1 << 30) || width < 0) return RQ_ERR_ARG;
    if (layers > 1 && (layer_stride < c.pages * c.page_bytes || layer_stride % 16 != 0)) return RQ_ERR_ARG;
    if (keep > (int64_t)(new_table ? new_width : width) << c.page_shift || (new_table && new_width < 0)) return RQ_ERR_ARG;
    if (weights) {
        if (n < keep || n > (1 << 30) || w_layer_stride < 0 || w_seq_stride < 0 || w_head_stride < 0) return RQ_ERR_ARG;
        if (!rows_apart(n, layers, w_layer_stride, batch, w_seq_stride, c.kv_heads, w_head_stride)) return RQ_ERR_ARG;
    }
    // (a workgroup for every 64 rows, of which a grid holds fewer than 2^35)
    if ((double)layers * batch * c.kv_heads * (double)(keep / 64 + 2) >= (double)((int64_t)1 << 35)) return RQ_ERR_ARG;
    if (layers == 0 || batch == 0 || (keep == 0 && (!weights || n == 0))) return RQ_OK;
    if ((keep > 0 && (!index || !table)) || !aligned(index, 4) || !aligned(table, 4) || !aligned(new_table, 4) || !aligned(weights, 4)) return RQ_ERR_ARG;
    return rq::kv4_evict(c, rq::Kv4Evict{index, table, new_table, weights, w_layer_stride, w_seq_stride, w_head_stride, layers > 1 ? layer_stride : 0, layers,
                                         batch, (int)keep, width, new_width, (int)n}, static_cast<hipStream_t>(stream));
}

size_t rq_kv4_prefix_attention_workspace(const rq_kv4_t* cache, int64_t tokens, int heads, int groups, int batch, int decode, int window,
                                         int64_t max_prefix, int64_t max_len) {
    rq::Kv4 c;
    if (cache_of(cache, &c) != RQ_OK || shape_ok(c, tokens, heads, batch, window, max_len) != RQ_OK || tokens == 0 || batch == 0) return 0;
    if (groups < 1 || groups > (1 << 20) || max_prefix < 0 || max_prefix > (1 << 30) - max_len) return 0;
    const int cu = num_cu();
    if (cu <= 0) return 0;
    rq::Kv4Attention a{};
    a.tokens = (int)tokens;
    a.heads = heads;
    a.batch = batch;
    a.window = window_of(window, max_prefix + max_len);
    a.max_len = max_len;
    a.q_start = decode ? nullptr : &kRagged;
    return rq::kv4_prefix_workspace(c, a, rq::Kv4Prefix{nullptr, nullptr, nullptr, groups, 0, max_prefix}, cu);
}

int rq_kv4_prefix_attention_plan(const rq_kv4_t* cache, int dtype, int64_t tokens, int heads, int groups, int batch, int decode, int window,
                                 int64_t max_prefix, int64_t max_len, int compute_units, rq_kv4_prefix_plan_t* plan) {
    rq::Kv4 c;
    int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if ((rc = shape_ok(c, tokens, heads, batch, window, max_len)) != RQ_OK) return rc;
    if (!plan || (dtype != RQ_BF16 && dtype != RQ_F16) || compute_units < 0) return RQ_ERR_ARG;
    if (groups < 1 || groups > (1 << 20) || max_prefix < 0 || max_prefix > (1 << 30) - max_len) return RQ_ERR_ARG;
    if (tokens == 0 || batch == 0 || (decode && tokens != batch)) return RQ_ERR_ARG;
    const int cu = compute_units ? compute_units : num_cu();
    if (cu <= 0) return RQ_ERR_HIP;
    rq::Kv4Attention a{};
    a.dtype = dtype;
    a.tokens = (int)tokens;
    a.heads = heads;
    a.batch = batch;
    a.window = window_of(window, max_prefix + max_len);
    a.max_len = max_len;
    a.q_start = decode ? nullptr : &kRagged;
    *plan = rq::kv4_prefix_plan(c, a, rq::Kv4Prefix{nullptr, nullptr, nullptr, groups, 0, max_prefix}, cu);
    return RQ_OK;
}

int rq_kv4_prefix_attention(const rq_hadamard_t* h, const rq_kv4_t* cache, const void* Q, int dtype, int64_t tokens, int heads,
                            int64_t q_token_stride, int64_t q_head_stride, const int32_t* prefix_table, int groups, int prefix_width,
                            const int32_t* prefix_lens, const int32_t* group_start, const int32_t* table, int batch, int width, const int32_t* kv_lens,
                            const int32_t* q_start, float scale, int causal, int window, int64_t max_prefix, int64_t max_len, void* O,
                            int64_t o_token_stride, int64_t o_head_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    rq::Kv4 c;
    int rc = cache_of(cache, &c);
    if (rc != RQ_OK) return rc;
    if (!rotation_ok(h, c.head_dim) || (dtype != RQ_BF16 && dtype != RQ_F16)) return RQ_ERR_ARG;
    if ((rc = shape_ok(c, tokens, heads, batch, window, max_len)) != RQ_OK) return rc;
    if (width < 0 || prefix_width < 0 || (causal != 0 && causal != 1) || !(scale > 0.0f) || !std::isfinite(scale)) return RQ_ERR_ARG;
    if (groups < 0 || groups > (1 << 20) || max_prefix < 0 || max_prefix > (1 << 30) - max_len) return RQ_ERR_ARG;
    if (q_token_stride < 0 || q_head_stride < 0 || o_token_stride < 0 || o_head_stride < 0) return RQ_ERR_ARG;
    if ((tokens > 1 && o_token_stride < c.head_dim) || (heads > 1 && o_head_stride < c.head_dim)) return RQ_ERR_ARG;
    if (!q_start && tokens != batch) return RQ_ERR_ARG;                    // a token a sequence
    if (tokens == 0) return RQ_OK;
    if (batch == 0 || groups == 0 || !Q || !O || !kv_lens || !prefix_lens || !group_start) return RQ_ERR_ARG;
    if ((width > 0 && !table) || (prefix_width > 0 && !prefix_table) || (width + (int64_t)prefix_width > 0 && c.pages == 0)) return RQ_ERR_ARG;
    if (!aligned(Q, 2) || !aligned(O, 2) || !aligned(table, 4) || !aligned(kv_lens, 4) || !aligned(q_start, 4) || !aligned(lse, 4)) return RQ_ERR_ARG;
    if (!aligned(prefix_table, 4) || !aligned(prefix_lens, 4) || !aligned(group_start, 4)) return RQ_ERR_ARG;
    if (max_len > (int64_t)width << c.page_shift || max_prefix > (int64_t)prefix_width << c.page_shift) return RQ_ERR_ARG;
    const rq::Kv4Attention a{Q, O, lse, dtype, (int)tokens, heads, batch, width, q_token_stride, q_head_stride, o_token_stride, o_head_stride,
                             table, kv_lens, q_start, scale, causal != 0, h != nullptr, window_of(window, max_prefix + max_len), max_len};
    const rq::Kv4Prefix p{prefix_table, prefix_lens, group_start, groups, prefix_width, max_prefix};
    const int cu = num_cu();
    if (cu <= 0) return RQ_ERR_HIP;
    const size_t need = rq::kv4_prefix_workspace(c, a, p, cu);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return RQ_ERR_ARG;
    return rq::kv4_prefix_attention(c, a, p, cu, static_cast<float*>(workspace), static_cast<hipStream_t>(stream));
}

}  // extern "C"
