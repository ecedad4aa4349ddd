// C-ABI entry points of the paged KV cache: host-side validation, workspace carving, launches.
// Nothing here allocates, frees or synchronises; see include/sparse_prefill.h.
#include <math.h>

#include "overlap.hpp"
#include "paged.hpp"

using namespace spa;

namespace {

constexpr int kMostTokens = 1 << 30;      // longer windows and sinks cover everything, too

int check_paged(const spa_paged_params* p) {
    if (!p) return SPA_ERR_NULLPTR;
    if (p->batch < 1 || p->batch > kMaxRequests || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_tokens < 1) return SPA_ERR_BAD_SHAPE;
    if (p->n_q_heads % p->n_kv_heads) return SPA_ERR_BAD_SHAPE;
    if (p->head_dim != 64 && p->head_dim != 128) return SPA_ERR_BAD_SHAPE;
    if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128) return SPA_ERR_BAD_SHAPE;
    if (p->n_pages < 1 || (int64_t)p->n_pages * p->page_size > 0x7fffffffll) return SPA_ERR_BAD_SHAPE;
    if (p->max_pages < 1 || (int64_t)p->max_pages * p->page_size > kMostTokens) return SPA_ERR_BAD_SHAPE;
    if (p->n_tokens > (1 << 24) || (int64_t)p->n_tokens * p->n_q_heads > 0x7fffffffll || p->max_new_tokens < 0) return SPA_ERR_BAD_SHAPE;
    if (!(p->softmax_scale >= 0.0f) || isinf(p->softmax_scale)) return SPA_ERR_BAD_SHAPE;
    if (p->n_sink_tokens < 0 || p->window_tokens < 0 || !(p->softcap >= 0.0f) || p->softcap > 65536.0f) return SPA_ERR_BAD_PATTERN;
    return SPA_OK;
}

// least: what either stride must at least be; unit: elements of 16 bytes
int check_strided(const void* ptr, const int64_t s[2], int64_t least, int unit = 8) {
    if (!ptr) return SPA_ERR_NULLPTR;
    if (((uintptr_t)ptr) & 15u) return SPA_ERR_BAD_STRIDE;
    for (int a = 0; a < 2; ++a)
        if (s[a] < least || (s[a] & (unit - 1))) return SPA_ERR_BAD_STRIDE;
    return SPA_OK;
}
// pages of bf16 values, or with e of one-byte values and their exponents
int check_pages(const spa_paged_params* p, const void* k_pages, const void* vt_pages, const spa_paged_exps* e) {
    const int64_t page = (int64_t)p->page_size * p->head_dim;
    int rc;
    if ((rc = check_strided(k_pages, p->kp_stride, page, e ? 16 : 8)) || (rc = check_strided(vt_pages, p->vp_stride, page, e ? 16 : 8))) return rc;
    if (e && ((rc = check_strided(e->k, e->k_stride, p->page_size, 16)) || (rc = check_strided(e->v, e->v_stride, p->page_size, 16)))) return rc;
    return SPA_OK;
}
PagedExps paged_exps(const spa_paged_exps* e) {
    if (!e) return PagedExps{};
    return PagedExps{(uint8_t*)e->k, (uint8_t*)e->v, e->k_stride[0], e->k_stride[1], e->v_stride[0], e->v_stride[1]};
}

int check_table(const spa_paged_params* p) { return p->table_stride < p->max_pages ? SPA_ERR_BAD_STRIDE : SPA_OK; }

PagedDims paged_dims(const spa_paged_params* p) {
    PagedDims d;
    d.B = p->batch; d.Hq = p->n_q_heads; d.Hkv = p->n_kv_heads; d.G = p->n_q_heads / p->n_kv_heads; d.D = p->head_dim;
    d.P = p->page_size;
    d.log_p = d.P == 16 ? 4 : d.P == 32 ? 5 : d.P == 64 ? 6 : 7;
    d.n_pages = p->n_pages; d.C = p->max_pages; d.T = p->n_tokens; d.max_new = p->max_new_tokens;
    d.scale = p->softmax_scale == 0.0f ? 1.0f / sqrtf((float)d.D) : p->softmax_scale;
    d.cap = p->softcap;
    d.sink = p->n_sink_tokens < kMostTokens ? p->n_sink_tokens : kMostTokens;
    d.window = p->window_tokens < kMostTokens ? p->window_tokens : kMostTokens;
    d.table_stride = p->table_stride;
    d.q_t = p->q_stride[0]; d.q_h = p->q_stride[1]; d.o_t = p->o_stride[0]; d.o_h = p->o_stride[1];
    d.kp_p = p->kp_stride[0]; d.kp_h = p->kp_stride[1]; d.vp_p = p->vp_stride[0]; d.vp_h = p->vp_stride[1];
    return d;
}

// arrays of a call as rows of bytes
Rows words_of(const void* ptr, int64_t n) { return row_of(ptr, 4 * n); }
Rows table_rows(const spa_paged_params* p, const int32_t* table) { return rows_of(table, p->batch, 4 * (wide)p->table_stride, 1, 0, 4ll * p->max_pages); }
Rows token_rows(const spa_paged_params* p, const void* x, const int64_t s[2], int heads) { return rows_of(x, p->n_tokens, 2 * (wide)s[0], heads, 2 * (wide)s[1], 2ll * p->head_dim); }
Rows page_rows(const spa_paged_params* p, const void* x, const int64_t s[2], int bytes = 2) {
    return rows_of(x, p->n_pages, bytes * (wide)s[0], p->n_kv_heads, bytes * (wide)s[1], (int64_t)bytes * p->page_size * p->head_dim);
}
Rows exp_rows(const spa_paged_params* p, const void* x, const int64_t s[2]) { return rows_of(x, p->n_pages, s[0], p->n_kv_heads, s[1], p->page_size); }
Rows k_exp_rows(const spa_paged_params* p, const spa_paged_exps* e) { return e ? exp_rows(p, e->k, e->k_stride) : row_of(nullptr, 0); }
Rows v_exp_rows(const spa_paged_params* p, const spa_paged_exps* e) { return e ? exp_rows(p, e->v, e->v_stride) : row_of(nullptr, 0); }
// whether a written array lies on a read one, on another written one or on itself
template <int W, int R>
bool clash(const Rows (&written)[W], const Rows (&read)[R]) {
    for (int i = 0; i < W; ++i) {
        if (overlaps_itself(written[i])) return true;
        for (const Rows& r : read)
            if (overlap(written[i], r)) return true;
        for (int j = 0; j < i; ++j)
            if (overlap(written[i], written[j])) return true;
    }
    return false;
}

int launch_code(hipError_t e) { return e == hipSuccess ? SPA_OK : SPA_ERR_LAUNCH; }

// attention over quantised pages (exps) or of requests with shared prompts (shares)
int attend(const spa_paged_params* p, const void* q, const void* k_pages, const void* vt_pages, const spa_paged_exps* exps,
           const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens, const int32_t* shares, bool shared, const float* slopes_or_null, void* out,
           float* lse_or_null, void* ws, size_t ws_bytes, void* hip_stream) {
    if (!block_table || !q_starts || !kv_lens) return SPA_ERR_NULLPTR;
    int rc;
    if ((rc = check_table(p))) return rc;
    if ((rc = check_strided(q, p->q_stride, 0)) || (rc = check_strided(out, p->o_stride, p->head_dim)) || (rc = check_pages(p, k_pages, vt_pages, exps))) return rc;
    const PagedDims d = paged_dims(p);
    const PagedParts parts = shared ? paged_shared_parts(d, ws) : paged_parts(d, ws);
    if (parts.ws_bytes > 0 && !ws) return SPA_ERR_NULLPTR;
    if (((uintptr_t)ws) & 255u) return SPA_ERR_BAD_STRIDE;
    if (ws_bytes < parts.ws_bytes) return SPA_ERR_WORKSPACE_TOO_SMALL;
    const int bytes = exps ? 1 : 2;
    // several workgroups read a query whose output one of them writes
    const Rows read[] = {token_rows(p, q, p->q_stride, p->n_q_heads), page_rows(p, k_pages, p->kp_stride, bytes), page_rows(p, vt_pages, p->vp_stride, bytes),
                         k_exp_rows(p, exps), v_exp_rows(p, exps), table_rows(p, block_table), words_of(q_starts, p->batch + 1), words_of(kv_lens, p->batch),
                         words_of(shares, 3ll * p->batch), words_of(slopes_or_null, p->n_q_heads)};
    const Rows written[] = {token_rows(p, out, p->o_stride, p->n_q_heads), words_of(lse_or_null, (int64_t)p->n_tokens * p->n_q_heads),
                            row_of(ws, (int64_t)parts.ws_bytes)};
    if (clash(written, read) || k_pages == vt_pages || (exps && exps->k == exps->v)) return SPA_ERR_OVERLAP;
    if (shared)
        return launch_code(launch_paged_attn_shared(d, parts, q, k_pages, vt_pages, paged_exps(exps), block_table, q_starts, kv_lens, shares, slopes_or_null,
                                                    out, lse_or_null, (hipStream_t)hip_stream));
    return launch_code(launch_paged_attn_q8(d, parts, q, k_pages, vt_pages, paged_exps(exps), block_table, q_starts, kv_lens, slopes_or_null, out,
                                            lse_or_null, (hipStream_t)hip_stream));
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int spa_paged_workspace_bytes(const spa_paged_params* p, size_t* bytes) {
    const int rc = check_paged(p);
    if (rc) return rc;
    if (!bytes) return SPA_ERR_NULLPTR;
    *bytes = paged_parts(paged_dims(p), nullptr).ws_bytes;
    return SPA_OK;
}

int sparse_prefill_paged_plan(const spa_paged_params* p, const int32_t* ctx_lens, const int32_t* new_lens, const int32_t* free_pages,
                              int32_t n_free, const int32_t* free_range, int32_t* block_table, int32_t* q_starts, int32_t* kv_lens,
                              int32_t* slots, int32_t* positions_or_null, int32_t* taken, void* hip_stream) {
    int rc = check_paged(p);
    if (rc) return rc;
    if (!ctx_lens || !new_lens || !free_range || !block_table || !q_starts || !kv_lens || !slots || !taken) return SPA_ERR_NULLPTR;
    if (n_free < 0) return SPA_ERR_BAD_SHAPE;
    if (n_free > 0 && !free_pages) return SPA_ERR_NULLPTR;
    if ((rc = check_table(p))) return rc;
    const Rows read[] = {words_of(ctx_lens, p->batch), words_of(new_lens, p->batch), words_of(free_pages, n_free), words_of(free_range, 2)};
    const Rows written[] = {table_rows(p, block_table), words_of(q_starts, p->batch + 1), words_of(kv_lens, p->batch), words_of(slots, p->n_tokens),
                            words_of(positions_or_null, p->n_tokens), words_of(taken, 2)};
    if (clash(written, read)) return SPA_ERR_OVERLAP;
    return launch_code(launch_paged_plan(paged_dims(p), ctx_lens, new_lens, free_pages, n_free, free_range, block_table, q_starts, kv_lens,
                                         slots, positions_or_null, taken, (hipStream_t)hip_stream));
}

int sparse_prefill_paged_append(const spa_paged_params* p, const void* k, const void* v, const int32_t* slots, void* k_pages,
                                void* vt_pages, void* hip_stream) {
    int rc = check_paged(p);
    if (rc) return rc;
    if (!slots) return SPA_ERR_NULLPTR;
    const int64_t page = (int64_t)p->page_size * p->head_dim;
    if ((rc = check_strided(k, p->k_stride, 0)) || (rc = check_strided(v, p->v_stride, 0))) return rc;
    if ((rc = check_strided(k_pages, p->kp_stride, page)) || (rc = check_strided(vt_pages, p->vp_stride, page))) return rc;
    const Rows read[] = {token_rows(p, k, p->k_stride, p->n_kv_heads), token_rows(p, v, p->v_stride, p->n_kv_heads), words_of(slots, p->n_tokens)};
    const Rows written[] = {page_rows(p, k_pages, p->kp_stride), page_rows(p, vt_pages, p->vp_stride)};
    if (clash(written, read)) return SPA_ERR_OVERLAP;
    return launch_code(launch_paged_append(paged_dims(p), k, p->k_stride[0], p->k_stride[1], v, p->v_stride[0], p->v_stride[1], slots,
                                           k_pages, vt_pages, (hipStream_t)hip_stream));
}

int sparse_prefill_paged_attn(const spa_paged_params* p, const void* q, const void* k_pages, const void* vt_pages,
                              const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens, const float* slopes_or_null,
                              void* out, float* lse_or_null, void* ws, size_t ws_bytes, void* hip_stream) {
    int rc = check_paged(p);
    if (rc) return rc;
    if (!block_table || !q_starts || !kv_lens) return SPA_ERR_NULLPTR;
    if ((rc = check_table(p))) return rc;
    const int64_t page = (int64_t)p->page_size * p->head_dim;
    if ((rc = check_strided(q, p->q_stride, 0)) || (rc = check_strided(out, p->o_stride, p->head_dim))) return rc;
    if ((rc = check_strided(k_pages, p->kp_stride, page)) || (rc = check_strided(vt_pages, p->vp_stride, page))) return rc;
    const PagedDims d = paged_dims(p);
    const PagedParts parts = paged_parts(d, ws);
    if (parts.ws_bytes > 0 && !ws) return SPA_ERR_NULLPTR;
    if (((uintptr_t)ws) & 255u) return SPA_ERR_BAD_STRIDE;
    if (ws_bytes < parts.ws_bytes) return SPA_ERR_WORKSPACE_TOO_SMALL;
    // several workgroups read a query whose output one of them writes
    const Rows read[] = {token_rows(p, q, p->q_stride, p->n_q_heads), page_rows(p, k_pages, p->kp_stride), page_rows(p, vt_pages, p->vp_stride),
                         table_rows(p, block_table), words_of(q_starts, p->batch + 1), words_of(kv_lens, p->batch), words_of(slopes_or_null, p->n_q_heads)};
    const Rows written[] = {token_rows(p, out, p->o_stride, p->n_q_heads), words_of(lse_or_null, (int64_t)p->n_tokens * p->n_q_heads),
                            row_of(ws, (int64_t)parts.ws_bytes)};
    if (clash(written, read) || k_pages == vt_pages) return SPA_ERR_OVERLAP;
    return launch_code(launch_paged_attn(d, parts, q, k_pages, vt_pages, block_table, q_starts, kv_lens, slopes_or_null, out, lse_or_null,
                                         (hipStream_t)hip_stream));
}

int sparse_prefill_paged_append_quantised(const spa_paged_params* p, const void* k, const void* v, const int32_t* slots, void* k_pages,
                                   void* vt_pages, const spa_paged_exps* exps, void* hip_stream) {
    int rc = check_paged(p);
    if (rc) return rc;
    if (!slots || !exps) return SPA_ERR_NULLPTR;
    if ((rc = check_strided(k, p->k_stride, 0)) || (rc = check_strided(v, p->v_stride, 0)) || (rc = check_pages(p, k_pages, vt_pages, exps))) return rc;
    const Rows read[] = {token_rows(p, k, p->k_stride, p->n_kv_heads), token_rows(p, v, p->v_stride, p->n_kv_heads), words_of(slots, p->n_tokens)};
    const Rows written[] = {page_rows(p, k_pages, p->kp_stride, 1), page_rows(p, vt_pages, p->vp_stride, 1), k_exp_rows(p, exps), v_exp_rows(p, exps)};
    if (clash(written, read)) return SPA_ERR_OVERLAP;
    return launch_code(launch_paged_append_q8(paged_dims(p), k, p->k_stride[0], p->k_stride[1], v, p->v_stride[0], p->v_stride[1], slots, k_pages,
                                              vt_pages, paged_exps(exps), (hipStream_t)hip_stream));
}

int sparse_prefill_paged_attn_quantised(const spa_paged_params* p, const void* q, const void* k_pages, const void* vt_pages, const spa_paged_exps* exps,
                                 const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens, const float* slopes_or_null,
                                 void* out, float* lse_or_null, void* ws, size_t ws_bytes, void* hip_stream) {
    const int rc = check_paged(p);
    if (rc) return rc;
    if (!exps) return SPA_ERR_NULLPTR;
    return attend(p, q, k_pages, vt_pages, exps, block_table, q_starts, kv_lens, nullptr, false, slopes_or_null, out, lse_or_null, ws, ws_bytes, hip_stream);
}

int sparse_prefill_paged_read(const spa_paged_params* p, const void* k_pages, const void* vt_pages, const spa_paged_exps* exps_or_null,
                              const int32_t* block_table, const int32_t* starts, const int32_t* kv_lens, void* k, void* v, void* hip_stream) {
    int rc = check_paged(p);
    if (rc) return rc;
    if (!block_table || !starts || !kv_lens) return SPA_ERR_NULLPTR;
    if ((rc = check_table(p)) || (rc = check_pages(p, k_pages, vt_pages, exps_or_null))) return rc;
    if ((rc = check_strided(k, p->k_stride, p->head_dim)) || (rc = check_strided(v, p->v_stride, p->head_dim))) return rc;
    const int bytes = exps_or_null ? 1 : 2;
    const Rows read[] = {page_rows(p, k_pages, p->kp_stride, bytes), page_rows(p, vt_pages, p->vp_stride, bytes), k_exp_rows(p, exps_or_null),
                         v_exp_rows(p, exps_or_null), table_rows(p, block_table), words_of(starts, p->batch + 1), words_of(kv_lens, p->batch)};
    const Rows written[] = {token_rows(p, k, p->k_stride, p->n_kv_heads), token_rows(p, v, p->v_stride, p->n_kv_heads)};
    if (clash(written, read) || k_pages == vt_pages || (exps_or_null && exps_or_null->k == exps_or_null->v)) return SPA_ERR_OVERLAP;
    return launch_code(launch_paged_read(paged_dims(p), k_pages, vt_pages, paged_exps(exps_or_null), block_table, starts, kv_lens, k, p->k_stride[0],
                                         p->k_stride[1], v, p->v_stride[0], p->v_stride[1], (hipStream_t)hip_stream));
}

int sparse_prefill_paged_shares(const spa_paged_params* p, const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens,
                                int32_t min_tokens, int32_t* shares, void* hip_stream) {
    int rc = check_paged(p);
    if (rc) return rc;
    if (!block_table || !q_starts || !kv_lens || !shares) return SPA_ERR_NULLPTR;
    if (min_tokens < 0) return SPA_ERR_BAD_PATTERN;
    if ((rc = check_table(p))) return rc;
    const Rows read[] = {table_rows(p, block_table), words_of(q_starts, p->batch + 1), words_of(kv_lens, p->batch)};
    const Rows written[] = {words_of(shares, 3ll * p->batch)};
    if (clash(written, read)) return SPA_ERR_OVERLAP;
    return launch_code(launch_paged_shares(paged_dims(p), block_table, q_starts, kv_lens, min_tokens, shares, (hipStream_t)hip_stream));
}

int spa_paged_shared_workspace_bytes(const spa_paged_params* p, size_t* bytes) {
    const int rc = check_paged(p);
    if (rc) return rc;
    if (!bytes) return SPA_ERR_NULLPTR;
    *bytes = paged_shared_parts(paged_dims(p), nullptr).ws_bytes;
    return SPA_OK;
}

int sparse_prefill_paged_attn_shared(const spa_paged_params* p, const void* q, const void* k_pages, const void* vt_pages,
                                     const spa_paged_exps* exps_or_null, const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens,
                                     const int32_t* shares, const float* slopes_or_null, void* out, float* lse_or_null, void* ws, size_t ws_bytes,
                                     void* hip_stream) {
    const int rc = check_paged(p);
    if (rc) return rc;
    if (!shares) return SPA_ERR_NULLPTR;
    return attend(p, q, k_pages, vt_pages, exps_or_null, block_table, q_starts, kv_lens, shares, true, slopes_or_null, out, lse_or_null, ws, ws_bytes,
                  hip_stream);
}

}  // extern "C"
#pragma GCC visibility pop
