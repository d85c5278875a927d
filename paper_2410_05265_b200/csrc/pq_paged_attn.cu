// Attention over [full-precision prefix || paged 4-bit cache] for a ragged batch (pq_attn_kv4_paged), through a window (pq_attn_kv4_paged_window) and of drafted trees
// (pq_attn_kv4_paged_tree).
//
// Sequences with one new row (decode) and those with several (prompts, chunks) have a kernel each, with a form for windows; which sequences are whose is found on the
// device, from q_begin. A batch whose host bound says one row needs the first launch only. Drafted trees have a kernel of their own, whatever their rows.
#include "pq_paged_attn.cuh"

extern "C" size_t pq_attn_kv4_paged_workspace_bytes(const pq_ctx* ctx, const pq_kv4_paged* cache, int64_t n_rows, int32_t max_new) {
  if (!ctx || pq_check_paged(cache) != PQ_OK || n_rows <= 0 || max_new <= 0) return 0;
  const size_t one = pq_paged_decode_ws_bytes(ctx, cache), more = max_new > 1 ? pq_paged_prefill_ws_bytes(ctx) : 0;
  return one + more;  // the two kernels overlap
}

namespace {

// What the three entry points have in common; window 0: none, mask null: rows are consecutive tokens.
pq_status attention(pq_ctx* ctx, const pq_kv4_paged* c, const void* q, int64_t ldq, const int32_t* q_begin, int64_t n_rows, int32_t max_new, int32_t max_len,
                    int32_t window, int32_t n_sink, const uint32_t* mask, int32_t mask_words, void* out, float sm_scale, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx || n_rows < 0 || max_new < 0 || max_len < 0 || !(sm_scale > 0.0f) || !isfinite(sm_scale)) return PQ_ERR_INVALID_ARG;
  pq_status st = pq_check_paged(c);
  if (st != PQ_OK) return st;
  if (n_rows == 0 || c->pages.B == 0 || max_new == 0) return PQ_OK;
  if (!q || !out || !q_begin || ldq < static_cast<int64_t>(c->Hq) * 128) return PQ_ERR_INVALID_ARG;
  if (n_rows > 0x7fffffffll) return PQ_ERR_SHAPE;
  if (pq_misaligned16(q) || pq_misaligned16(out) || pq_misaligned16(ws) || ldq % 8 != 0) return PQ_ERR_ALIGN;
  if (!ws || ws_bytes < (mask ? pq_attn_kv4_paged_tree_workspace_bytes : pq_attn_kv4_paged_workspace_bytes)(ctx, c, n_rows, max_new)) return PQ_ERR_WORKSPACE;
  PagedAttnParams p{};
  p.q = static_cast<const __nv_bfloat16*>(q), p.ldq = ldq, p.out = static_cast<__nv_bfloat16*>(out), p.q_begin = q_begin;
  p.len = c->pages.len, p.table = c->pages.table;
  p.prefix_k = static_cast<const __half*>(c->prefix_k), p.prefix_v = static_cast<const __half*>(c->prefix_v);
  p.codes = c->codes, p.steps = c->steps, p.s_k = c->s_k, p.s_v = c->s_v, p.tickets = ctx->d_tickets, p.status = ctx->d_status;
  p.wait_clocks = ctx->wait_clocks;
  p.n_rows = static_cast<int32_t>(n_rows), p.scale2 = sm_scale * 1.4426950408889634f;
  p.B = c->pages.B, p.max_pages = c->pages.n_pages > 0 ? c->pages.max_pages : 0, p.page_log2 = pq_page_log2(c->pages.page), p.n_pages = c->pages.n_pages;
  p.Hq = c->Hq, p.Hkv = c->Hkv, p.G = c->Hq / c->Hkv, p.n_prefix = c->n_prefix, p.max_new = max_new;
  const int64_t capacity = static_cast<int64_t>(p.max_pages) << p.page_log2;
  const int64_t bound = max_len > 0 && max_len < capacity ? max_len : capacity;
  // a window that holds every cache is none; numbers past any cache's end stay clear of the end of 32 bits
  p.window = window >= capacity ? 0 : window, p.n_sink = p.window == 0 ? 0 : n_sink < capacity ? n_sink : static_cast<int32_t>(capacity);
  p.mask = mask, p.mask_words = mask_words;
  if (mask) return pq_paged_tree_launch(ctx, p, bound, ws, static_cast<cudaStream_t>(stream));
  // The kernel for several rows takes whole SMs and goes first; the one for single tokens, whose CTAs are small, starts beside it on the SMs that it leaves.
  if (max_new > 1) {
    st = pq_paged_prefill_launch(ctx, p, static_cast<uint8_t*>(ws) + pq_paged_decode_ws_bytes(ctx, c), static_cast<cudaStream_t>(stream));
    if (st != PQ_OK) return st;
  }
  return pq_paged_decode_launch(ctx, c, p, bound, ws, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" pq_status pq_attn_kv4_paged(pq_ctx* ctx, const pq_kv4_paged* c, const void* q, int64_t ldq, const int32_t* q_begin, int64_t n_rows,
                                       int32_t max_new, int32_t max_len, void* out, float sm_scale, void* ws, size_t ws_bytes, void* stream) {
  return attention(ctx, c, q, ldq, q_begin, n_rows, max_new, max_len, 0, 0, nullptr, 0, out, sm_scale, ws, ws_bytes, stream);
}

extern "C" pq_status pq_attn_kv4_paged_window(pq_ctx* ctx, const pq_kv4_paged* c, const void* q, int64_t ldq, const int32_t* q_begin, int64_t n_rows,
                                              int32_t max_new, int32_t max_len, int32_t window, int32_t n_sink, void* out, float sm_scale, void* ws,
                                              size_t ws_bytes, void* stream) {
  if (window < 1 || n_sink < 0) return PQ_ERR_INVALID_ARG;
  return attention(ctx, c, q, ldq, q_begin, n_rows, max_new, max_len, window, n_sink, nullptr, 0, out, sm_scale, ws, ws_bytes, stream);
}

extern "C" size_t pq_attn_kv4_paged_tree_workspace_bytes(const pq_ctx* ctx, const pq_kv4_paged* cache, int64_t n_rows, int32_t max_new) {
  if (!ctx || pq_check_paged(cache) != PQ_OK || n_rows <= 0 || max_new <= 0) return 0;
  return pq_paged_tree_ws_bytes(ctx);
}

extern "C" pq_status pq_attn_kv4_paged_tree(pq_ctx* ctx, const pq_kv4_paged* c, const void* q, int64_t ldq, const int32_t* q_begin, int64_t n_rows,
                                            int32_t max_new, int32_t max_len, const uint32_t* mask, int32_t mask_words, int32_t window, int32_t n_sink, void* out,
                                            float sm_scale, void* ws, size_t ws_bytes, void* stream) {
  if (window < 0 || n_sink < 0 || mask_words < 0) return PQ_ERR_INVALID_ARG;
  if (max_new > PQ_TREE_MAX_ROWS || max_new > 32ll * mask_words || (window > 0 && window < max_new)) return PQ_ERR_SHAPE;
  if (max_new > 0 && n_rows > 0 && !mask) return PQ_ERR_INVALID_ARG;
  return attention(ctx, c, q, ldq, q_begin, n_rows, max_new, max_len, window, n_sink, mask, mask_words, out, sm_scale, ws, ws_bytes, stream);
}
