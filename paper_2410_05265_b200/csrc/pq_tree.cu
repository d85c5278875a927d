// Trees of drafted tokens over the paged KV4 cache: ancestors and positions before the attention (pq_tree_plan), the accepted path behind it (pq_tree_accept),
// and the moves that put the accepted tokens behind one another (pq_kv4_paged_keep).
//
// All three are integer bookkeeping and copies of a few KB a sequence: latency decides. A CTA takes a sequence (of the moves a sequence and KV head), whose at most
// 128 drafts are a thread each.
#include "pq_paged.cuh"

namespace {

constexpr int TR_THREADS = PQ_TREE_MAX_ROWS;
constexpr int TR_WORDS = PQ_TREE_MAX_ROWS / 32;

struct TreeParams {
  const int32_t* q_begin;
  const int32_t* len;
  const int32_t* parent;
  const int32_t* draft;
  const int32_t* target;
  uint32_t* mask;
  int32_t* pos;
  int32_t* kept;
  int32_t* n_kept;
  int32_t* next;
  int32_t* status;
  int64_t capacity;
  int32_t B, n_rows, mask_words, pos0;
};

// Rows of sequence b; false, and none, where they are no rows of a tree.
__device__ __forceinline__ bool tree_rows(const TreeParams& p, int b, int most, int& r0, int& n) {
  r0 = pq::ld_dep(p.q_begin + b);
  const int64_t rows = static_cast<int64_t>(pq::ld_dep(p.q_begin + b + 1)) - r0;
  const bool ok = rows >= 0 && rows <= most && (rows == 0 || (r0 >= 0 && r0 + rows <= p.n_rows));
  n = ok ? static_cast<int>(rows) : 0;
  return ok;
}
// The rows behind the last sequence, dealt to the CTAs.
template <typename F>
__device__ __forceinline__ void padding_rows(const TreeParams& p, const F& f) {
  const int end = p.B > 0 ? pq::ld_dep(p.q_begin + p.B) : 0;
  for (int64_t r = max(end, 0) + static_cast<int64_t>(blockIdx.x) * TR_THREADS + threadIdx.x; r < p.n_rows; r += static_cast<int64_t>(gridDim.x) * TR_THREADS) f(r);
}

// Ancestors by doubling: after k rounds a row knows those of 2^k generations and who comes next.
__global__ void __launch_bounds__(TR_THREADS) tree_plan_kernel(const TreeParams p) {
  __shared__ uint4 bits[TR_THREADS];
  __shared__ int2 up[TR_THREADS];  // (the row 2^k generations up, or -1; generations counted so far)
  pq::pdl_wait();
  pq::pdl_trigger();
  const int t = threadIdx.x;
  padding_rows(p, [&](int64_t r) {
    for (int w = 0; w < p.mask_words; ++w) p.mask[r * p.mask_words + w] = 0;
    p.pos[r] = 0;
  });
  const int b = blockIdx.x;
  if (b >= p.B) return;
  int r0, n;
  bool ok = tree_rows(p, b, min(TR_THREADS, 32 * p.mask_words), r0, n);
  const int l = pq::ld_dep(p.len + b);
  const bool live = ok && l >= n && l <= p.capacity;  // the drafts are the last of the cached tokens
  int parent = -1;
  if (ok && t < n) {
    parent = pq::ld_dep(p.parent + r0 + t);
    if (parent < -1 || parent >= t) ok = false, parent = -1;
  }
  if (!ok || (n > 0 && !live)) pq::report(p.status, PQ_ERR_SHAPE);
  if (n == 0) return;
  uint4 m = make_uint4(t >> 5 == 0 ? 1u << (t & 31) : 0u, t >> 5 == 1 ? 1u << (t & 31) : 0u, t >> 5 == 2 ? 1u << (t & 31) : 0u, t >> 5 == 3 ? 1u << (t & 31) : 0u);
  int2 u = make_int2(parent, parent >= 0 ? 1 : 0);
  bits[t] = m, up[t] = u;
  for (int far = 1; far < n; far <<= 1) {
    __syncthreads();
    uint4 om = make_uint4(0, 0, 0, 0);
    int2 ou = make_int2(-1, 0);
    if (u.x >= 0) om = bits[u.x], ou = up[u.x];
    __syncthreads();
    m.x |= om.x, m.y |= om.y, m.z |= om.z, m.w |= om.w;
    u.x = ou.x, u.y += ou.y;
    bits[t] = m, up[t] = u;
  }
  if (t >= n) return;
  const uint32_t w4[TR_WORDS] = {m.x, m.y, m.z, m.w};
#pragma unroll
  for (int w = 0; w < TR_WORDS; ++w)
    if (w < p.mask_words) p.mask[static_cast<int64_t>(r0 + t) * p.mask_words + w] = live ? w4[w] : 0u;
  p.pos[r0 + t] = live ? p.pos0 + (l - n) + u.y : 0;
}

// Every draft that the model's choice after its parent equals offers itself to the parent, the lowest stays; one thread then follows the path from row 0.
__global__ void __launch_bounds__(TR_THREADS) tree_accept_kernel(const TreeParams p) {
  __shared__ int child[TR_THREADS], choice[TR_THREADS], path[TR_THREADS], count;
  pq::pdl_wait();
  pq::pdl_trigger();
  const int t = threadIdx.x;
  padding_rows(p, [&](int64_t r) { p.kept[r] = -1; });
  const int b = blockIdx.x;
  if (b >= p.B) return;
  int r0, n;
  bool ok = tree_rows(p, b, TR_THREADS, r0, n);
  int parent = -1, draft = 0;
  child[t] = TR_THREADS, path[t] = -1;
  if (ok && t < n) {
    parent = pq::ld_dep(p.parent + r0 + t), draft = pq::ld_dep(p.draft + r0 + t), choice[t] = pq::ld_dep(p.target + r0 + t);
    if (parent < -1 || parent >= t) ok = false, parent = -1;
  }
  if (!ok) pq::report(p.status, PQ_ERR_SHAPE);
  __syncthreads();
  if (parent >= 0 && choice[parent] == draft) atomicMin(&child[parent], t);
  __syncthreads();
  if (t == 0) {
    int k = 0;
    for (int r = 0; r < n; r = child[r]) path[k++] = r;  // (a child lies behind its parent: n steps at most)
    count = k;
  }
  __syncthreads();
  if (t < n) p.kept[r0 + t] = path[t];
  if (t == 0) p.n_kept[b] = count, p.next[b] = count > 0 ? choice[path[count - 1]] : -1;
}

// Token i of the kept ones goes from its place among the drafts, base + kept[i], to base + i. Places are read before any is written, so that the order of the moves and
// places that are both read and written do not matter: a thread holds its up to eight pieces of 16 bytes (128 tokens, keys and values) and two steps.
__global__ void __launch_bounds__(TR_THREADS) kv4_paged_keep_kernel(const TreeParams p, const int32_t* table, uint8_t* codes, float* steps, int32_t Hkv, int32_t max_pages,
                                                                    int32_t page_log2, int32_t n_pages) {
  pq::pdl_wait();
  const int b = blockIdx.x / Hkv, h = blockIdx.x % Hkv, t = threadIdx.x;
  int r0, n;
  const bool ok = tree_rows(p, b, TR_THREADS, r0, n);
  const int l = pq::ld_dep(p.len + b), k = pq::ld_dep(p.n_kept + b);
  const int64_t base = static_cast<int64_t>(l) - k;
  if (!ok || k < 0 || k > n || (n > 0 && (base < 0 || base + n > p.capacity))) {  // (the whole CTA alike)
    if (t == 0) pq::report(p.status, PQ_ERR_SHAPE);
    return;
  }
  bool lost = false;
  auto vector_of = [&](int64_t c) {  // index of the key vector at place c of this head, the value vector lies a page further on; -1 where the table holds no id
    const int id = pq::ld_dep(table + static_cast<int64_t>(b) * max_pages + (c >> page_log2));
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(n_pages)) {
      lost = true;
      return static_cast<int64_t>(-1);
    }
    return (((static_cast<int64_t>(id) * Hkv + h) * 2) << page_log2) + (c & ((1 << page_log2) - 1));
  };
  auto source_of = [&](int i) {  // row of token i, or -1 where it stays or there is none
    const int f = pq::ld_dep(p.kept + r0 + i);
    if (f < 0 || f >= n) lost = true;
    return f < 0 || f >= n || f == i ? -1 : f;
  };
  uint4 piece[8];
  int64_t to[8];
  float step[2];
  int64_t step_to[2] = {-1, -1};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int unit = e * TR_THREADS + t, i = unit >> 3, kv = (unit >> 2) & 1, c16 = unit & 3;
    to[e] = -1;
    if (i >= k) continue;
    const int f = source_of(i);
    if (f < 0) continue;
    const int64_t from = vector_of(base + f), dst = vector_of(base + i);
    if (from < 0 || dst < 0) continue;
    piece[e] = pq::ld_dep(reinterpret_cast<const uint4*>(codes + (from + (static_cast<int64_t>(kv) << page_log2)) * 64) + c16);
    to[e] = (dst + (static_cast<int64_t>(kv) << page_log2)) * 64 + c16 * 16;
  }
  if (steps) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int unit = e * TR_THREADS + t, i = unit >> 1, kv = unit & 1;
      if (i >= k) continue;
      const int f = source_of(i);
      if (f < 0) continue;
      const int64_t from = vector_of(base + f), dst = vector_of(base + i);
      if (from < 0 || dst < 0) continue;
      step[e] = pq::ld_dep(steps + from + (static_cast<int64_t>(kv) << page_log2));
      step_to[e] = dst + (static_cast<int64_t>(kv) << page_log2);
    }
  }
  if (lost) pq::report(p.status, PQ_ERR_SHAPE);
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (to[e] >= 0) *reinterpret_cast<uint4*>(codes + to[e]) = piece[e];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (step_to[e] >= 0) steps[step_to[e]] = step[e];
}

}  // namespace

extern "C" pq_status pq_tree_plan(pq_ctx* ctx, const pq_pages* pages, const int32_t* parent, const int32_t* q_begin, int64_t n_rows, int32_t pos0, uint32_t* mask,
                                  int32_t mask_words, int32_t* pos, void* stream) {
  if (!ctx || n_rows < 0 || pos0 < 0 || mask_words < 1) return PQ_ERR_INVALID_ARG;
  const pq_status st = pq_check_pages(pages);
  if (st != PQ_OK) return st;
  if (n_rows == 0) return PQ_OK;
  if (!q_begin || !parent || !mask || !pos) return PQ_ERR_INVALID_ARG;
  if (n_rows > 0x7fffffffll || mask_words > TR_WORDS) return PQ_ERR_SHAPE;
  if (static_cast<int64_t>(pages->max_pages) * pages->page + pos0 > 0x7fffffffll) return PQ_ERR_SHAPE;  // a position would not fit
  TreeParams p{};
  p.q_begin = q_begin, p.len = pages->len, p.parent = parent, p.mask = mask, p.pos = pos, p.status = ctx->d_status;
  p.capacity = static_cast<int64_t>(pages->max_pages) * pages->page;
  p.B = pages->B, p.n_rows = static_cast<int32_t>(n_rows), p.mask_words = mask_words, p.pos0 = pos0;
  return pq_launch_pdl(tree_plan_kernel, dim3(p.B > 0 ? p.B : 1), TR_THREADS, 0, static_cast<cudaStream_t>(stream), p);
}

extern "C" pq_status pq_tree_accept(pq_ctx* ctx, const int32_t* q_begin, int32_t B, const int32_t* parent, const int32_t* draft, const int32_t* target, int64_t n_rows,
                                    int32_t* kept, int32_t* n_kept, int32_t* next, void* stream) {
  if (!ctx || n_rows < 0 || B < 0) return PQ_ERR_INVALID_ARG;
  if (B > 0 && (!q_begin || !n_kept || !next)) return PQ_ERR_INVALID_ARG;
  if (n_rows > 0 && (!parent || !draft || !target || !kept)) return PQ_ERR_INVALID_ARG;
  if (n_rows > 0x7fffffffll || B > PQ_PAGED_MAX_SEQS) return PQ_ERR_SHAPE;
  if (B == 0 && n_rows == 0) return PQ_OK;
  TreeParams p{};
  p.q_begin = q_begin, p.parent = parent, p.draft = draft, p.target = target, p.kept = kept, p.n_kept = n_kept, p.next = next, p.status = ctx->d_status;
  p.B = B, p.n_rows = static_cast<int32_t>(n_rows);
  return pq_launch_pdl(tree_accept_kernel, dim3(B > 0 ? B : 1), TR_THREADS, 0, static_cast<cudaStream_t>(stream), p);
}

extern "C" pq_status pq_kv4_paged_keep(pq_ctx* ctx, const pq_kv4_paged* c, const int32_t* q_begin, const int32_t* kept, const int32_t* n_kept, int64_t n_rows,
                                       void* stream) {
  if (!ctx || n_rows < 0) return PQ_ERR_INVALID_ARG;
  const pq_status st = pq_check_paged(c);
  if (st != PQ_OK) return st;
  if (n_rows == 0 || c->pages.B == 0) return PQ_OK;
  if (!q_begin || !kept || !n_kept) return PQ_ERR_INVALID_ARG;
  if (n_rows > 0x7fffffffll) return PQ_ERR_SHAPE;
  TreeParams p{};
  p.q_begin = q_begin, p.len = c->pages.len, p.kept = const_cast<int32_t*>(kept), p.n_kept = const_cast<int32_t*>(n_kept), p.status = ctx->d_status;
  p.capacity = c->pages.n_pages > 0 ? static_cast<int64_t>(c->pages.max_pages) * c->pages.page : 0;
  p.B = c->pages.B, p.n_rows = static_cast<int32_t>(n_rows);
  return pq_launch_pdl(kv4_paged_keep_kernel, dim3(static_cast<unsigned>(p.B) * c->Hkv), TR_THREADS, 0, static_cast<cudaStream_t>(stream), p, c->pages.table, c->codes,
                       c->steps, c->Hkv, c->pages.max_pages, pq_page_log2(c->pages.page), c->pages.n_pages);
}
