// Attention over [full-precision prefix || paged 4-bit cache] for a ragged batch (pq_attn_kv4_paged).
//
// One CTA per (row, KV head): a thread scores one key of a chunk of 128 for all query heads of the group in fp32, then takes one head dim of
// the output over the chunk's keys; running maximum and sum per head.
#include "pq_paged_attn.cuh"

namespace {

constexpr int SA_THREADS = 128;

__device__ __forceinline__ float nibble(const uint8_t* row, int d) {
  const int b = row[d >> 1];
  return static_cast<float>((d & 1) ? static_cast<int8_t>(b) >> 4 : static_cast<int8_t>(b << 4) >> 4);
}

__global__ void __launch_bounds__(SA_THREADS) attn_simple_kernel(const PagedAttnParams p) {
  __shared__ float sq[PQ_PAGED_MAX_GROUP][128];
  __shared__ float sp[PQ_PAGED_MAX_GROUP][SA_THREADS];
  __shared__ float red[SA_THREADS / 32];
  __shared__ float s_m;
  pq::pdl_wait();
  const int64_t row = blockIdx.x;
  const int h = blockIdx.y, tid = threadIdx.x;
  int b = 0;
  while (b < p.B && p.q_begin[b + 1] <= row) ++b;
  if (b >= p.B || p.q_begin[b] > row) return;
  const int n = p.q_begin[b + 1] - p.q_begin[b];
  const int64_t capacity = static_cast<int64_t>(p.max_pages) << p.page_log2;
  int len = p.len[b];
  if (n == 1) return;  // the other kernel's
  if (n > p.max_new || len < 0 || len > capacity) {
    if (tid == 0) pq::report(p.status, PQ_ERR_SHAPE);
    if (n > p.max_new) return;
    len = len < 0 ? 0 : static_cast<int>(capacity);
  }
  const int seen = max(0, len - n + static_cast<int>(row - p.q_begin[b]) + 1);
  const int n_keys = p.n_prefix + seen;
  for (int i = tid; i < p.G * 128; i += SA_THREADS)
    sq[i >> 7][i & 127] = __bfloat162float(p.q[row * p.ldq + static_cast<int64_t>(h * p.G + (i >> 7)) * 128 + (i & 127)]);
  float m[PQ_PAGED_MAX_GROUP], den[PQ_PAGED_MAX_GROUP], o[PQ_PAGED_MAX_GROUP];
  for (int g = 0; g < PQ_PAGED_MAX_GROUP; ++g) m[g] = -INFINITY, den[g] = 0.0f, o[g] = 0.0f;
  auto vec_of = [&](int j, int which) -> int64_t {  // -1: no such page
    const int32_t id = p.table[static_cast<int64_t>(b) * p.max_pages + (j >> p.page_log2)];
    if (id < 0 || id >= p.n_pages) return -1;
    return (((static_cast<int64_t>(id) * p.Hkv + h) * 2 + which) << p.page_log2) + (j & ((1 << p.page_log2) - 1));
  };
  for (int j0 = 0; j0 < n_keys; j0 += SA_THREADS) {
    __syncthreads();
    const int j = j0 + tid;
    float x[PQ_PAGED_MAX_GROUP];
    for (int g = 0; g < PQ_PAGED_MAX_GROUP; ++g) x[g] = j < n_keys ? 0.0f : -INFINITY;
    if (j < p.n_prefix) {
      const __half* k = p.prefix_k + (static_cast<int64_t>(h) * p.n_prefix + j) * 128;
      for (int d = 0; d < 128; ++d)
        for (int g = 0; g < p.G; ++g) x[g] += sq[g][d] * __half2float(k[d]);
      for (int g = 0; g < p.G; ++g) x[g] *= p.scale2;
    } else if (j < n_keys) {
      const int64_t vec = vec_of(j - p.n_prefix, 0);
      if (vec >= 0) {
        for (int d = 0; d < 128; ++d)
          for (int g = 0; g < p.G; ++g) x[g] += sq[g][d] * nibble(p.codes + vec * 64, d);
        const float s = p.steps ? p.steps[vec] : p.s_k[h];
        for (int g = 0; g < p.G; ++g) x[g] *= s * p.scale2;
      } else {
        pq::report(p.status, PQ_ERR_SHAPE);
      }
    }
    for (int g = 0; g < p.G; ++g) {
      float mx = x[g];
      for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
      if ((tid & 31) == 0) red[tid >> 5] = mx;
      __syncthreads();
      if (tid == 0) s_m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
      __syncthreads();
      const float mn = fmaxf(m[g], s_m), alpha = exp2f(m[g] - mn);
      o[g] *= alpha, den[g] *= alpha, m[g] = mn;
      sp[g][tid] = exp2f(x[g] - mn);
    }
    __syncthreads();
    for (int i = 0; i < min(SA_THREADS, n_keys - j0); ++i) {
      const int jj = j0 + i;
      float v;
      if (jj < p.n_prefix) {
        v = __half2float(p.prefix_v[(static_cast<int64_t>(h) * p.n_prefix + jj) * 128 + tid]);
      } else {
        const int64_t vec = vec_of(jj - p.n_prefix, 1);
        v = vec < 0 ? 0.0f : nibble(p.codes + vec * 64, tid) * (p.steps ? p.steps[vec] : p.s_v[h]);
      }
      for (int g = 0; g < p.G; ++g) o[g] += sp[g][i] * v, den[g] += sp[g][i];
    }
  }
  for (int g = 0; g < p.G; ++g)
    p.out[(row * p.Hq + h * p.G + g) * 128 + tid] = __float2bfloat16(den[g] > 0.0f ? o[g] / den[g] : 0.0f);
}

}  // namespace

extern "C" size_t pq_attn_kv4_paged_workspace_bytes(const pq_ctx* ctx, const pq_kv4_paged* cache, int64_t n_rows, int32_t max_new) {
  if (!ctx || pq_check_paged(cache) != PQ_OK || n_rows <= 0 || max_new <= 0) return 0;
  return pq_paged_decode_ws_bytes(ctx, cache);
}

extern "C" pq_status pq_attn_kv4_paged(pq_ctx* ctx, const pq_kv4_paged* c, const void* q, int64_t ldq, const int32_t* q_begin, int64_t n_rows,
                                       int32_t max_new, int32_t max_len, void* out, float sm_scale, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx || n_rows < 0 || max_new < 0 || max_len < 0 || !(sm_scale > 0.0f) || !isfinite(sm_scale)) return PQ_ERR_INVALID_ARG;
  pq_status st = pq_check_paged(c);
  if (st != PQ_OK) return st;
  if (n_rows == 0 || c->pages.B == 0 || max_new == 0) return PQ_OK;
  if (!q || !out || !q_begin || ldq < static_cast<int64_t>(c->Hq) * 128) return PQ_ERR_INVALID_ARG;
  if (n_rows > 0x7fffffffll) return PQ_ERR_SHAPE;
  if (pq_misaligned16(q) || pq_misaligned16(out) || pq_misaligned16(ws) || ldq % 8 != 0) return PQ_ERR_ALIGN;
  if (!ws || ws_bytes < pq_attn_kv4_paged_workspace_bytes(ctx, c, n_rows, max_new)) return PQ_ERR_WORKSPACE;
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
  st = pq_paged_decode_launch(ctx, c, p, bound, ws, static_cast<cudaStream_t>(stream));
  if (st != PQ_OK || max_new == 1) return st;
  return pq_launch_pdl(attn_simple_kernel, dim3(static_cast<unsigned>(n_rows), c->Hkv), SA_THREADS, 0, static_cast<cudaStream_t>(stream), p);
}
