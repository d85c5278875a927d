// Block tables, slots and positions of a step of the paged KV4 cache, built on the device from the request lengths, and the return of the
// pages of ended requests.
//
// Both are integer bookkeeping over at most a few thousand sequences and a few hundred thousand rows: 12 bytes a row, so latency decides. One
// launch each, one cluster: every CTA forms the prefix sums over the sequences for itself (a few loads, cheaper than handing them round),
// gives the same verdict on the step as the others, and writes its share of the rows and of the pages; the lengths and the count of free
// pages, which every CTA reads, are written behind the cluster's barrier, so that they may be advanced in place. No atomics, no counter
// that outlives the launch; the order of the pages is that of the definition whatever the shape of the launch.
#include <atomic>

#include "pq_paged.cuh"

namespace {

constexpr int PG_THREADS = 512;
constexpr int PG_CLUSTER = 8;           // CTAs of a large step
constexpr int64_t PG_ONE_CTA = 4096;    // rows (or pages that may go back) that one CTA takes alone

struct PlanParams {
  int32_t* table;
  const int32_t* len;
  int32_t* free_list;
  const int32_t* n_free;
  const int32_t* n_new;  // plan: new tokens; release: flags; keep: how many stay
  int32_t* n_kept;       // keep: the same array, -1 everywhere after a refusal
  int32_t* q_begin;
  int64_t* slot;
  int32_t* pos;
  int32_t* len_out;
  int32_t* n_free_out;
  int32_t* status;
  int64_t n_rows;
  int32_t B, max_pages, page_log2, n_pages, pos0;
};

__device__ __forceinline__ int pages_of(int tokens, int page_log2) { return static_cast<int>((static_cast<int64_t>(tokens) + (1 << page_log2) - 1) >> page_log2); }

// Shared memory: rows[B + 1], pages[B + 1], len[B].
__global__ void __launch_bounds__(PG_THREADS) page_plan_kernel(const PlanParams p) {
  extern __shared__ __align__(16) int32_t pg_smem[];
  __shared__ int64_t part[PG_THREADS / 32];
  __shared__ int bad;
  int32_t *rows = pg_smem, *pages = rows + p.B + 1, *len = pages + p.B + 1;
  pq::pdl_wait();
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  const int32_t n_free = pq::ld_dep(p.n_free);
  const int64_t capacity = static_cast<int64_t>(p.max_pages) << p.page_log2;
  for (int b = threadIdx.x; b < p.B; b += PG_THREADS) {
    const int32_t l = pq::ld_dep(p.len + b), n = pq::ld_dep(p.n_new + b);
    const bool ok = l >= 0 && n >= 0 && static_cast<int64_t>(l) + n <= capacity;
    if (!ok) bad = 1;
    len[b] = l;
    rows[b] = ok ? n : 0;
    pages[b] = ok ? pages_of(l + n, p.page_log2) - pages_of(l, p.page_log2) : 0;
  }
  __syncthreads();
  const int64_t total = pq::block_scan<PG_THREADS>(rows, p.B, part), need = pq::block_scan<PG_THREADS>(pages, p.B, part);
  const bool refused = bad || total > p.n_rows || n_free < 0 || n_free > p.n_pages || need > n_free;
  const int n_ctas = gridDim.x, tid = blockIdx.x * PG_THREADS + threadIdx.x, n_threads = n_ctas * PG_THREADS;
  auto page_id = [&](int64_t k) {  // the k-th page of the step; -1 where the list holds no id
    const int32_t id = pq::ld_dep(p.free_list + (n_free - 1 - k));
    return id >= 0 && id < p.n_pages ? id : -1;
  };
  bool lost = false;  // an id that is none was met
  if (!refused) {
    for (int64_t k = tid; k < need; k += n_threads) {
      const int b = pq::find_segment(pages, p.B, static_cast<int32_t>(k));
      const int32_t id = page_id(k);
      lost |= id < 0;
      p.table[static_cast<int64_t>(b) * p.max_pages + pages_of(len[b], p.page_log2) + (k - pages[b])] = id;
    }
  }
  // four rows to a thread and step: one search, 16-byte stores
  const int64_t n_live = refused ? 0 : total;
  for (int64_t r0 = 4 * static_cast<int64_t>(tid); r0 < p.n_rows; r0 += 4 * static_cast<int64_t>(n_threads)) {
    int64_t slot[4];
    int32_t pos[4];
    int b = r0 < n_live ? pq::find_segment(rows, p.B, static_cast<int32_t>(r0)) : 0;
    int32_t last_page = -1, last_id = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t r = r0 + i;
      slot[i] = -1, pos[i] = 0;
      if (r < n_live) {
        if (r >= rows[b + 1]) {
          b = pq::find_segment(rows, p.B, static_cast<int32_t>(r));
          last_page = -1;
        }
        const int32_t c = len[b] + static_cast<int32_t>(r - rows[b]), pg = c >> p.page_log2, old = pages_of(len[b], p.page_log2);
        if (pg != last_page) {
          if (pg < old) {
            last_id = pq::ld_dep(p.table + static_cast<int64_t>(b) * p.max_pages + pg);
            if (last_id < 0 || last_id >= p.n_pages) last_id = -1;
          } else {
            last_id = page_id(pages[b] + (pg - old));
          }
          last_page = pg;
          lost |= last_id < 0;
        }
        if (last_id >= 0) slot[i] = (static_cast<int64_t>(last_id) << p.page_log2) + (c & ((1 << p.page_log2) - 1));
        pos[i] = p.pos0 + c;
      }
    }
    if (r0 + 4 <= p.n_rows) {
      *reinterpret_cast<longlong2*>(p.slot + r0) = make_longlong2(slot[0], slot[1]);
      *reinterpret_cast<longlong2*>(p.slot + r0 + 2) = make_longlong2(slot[2], slot[3]);
      *reinterpret_cast<int4*>(p.pos + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
      for (int i = 0; i < p.n_rows - r0; ++i) p.slot[r0 + i] = slot[i], p.pos[r0 + i] = pos[i];
    }
  }
  if (lost || (refused && tid == 0)) pq::report(p.status, PQ_ERR_SHAPE);
  for (int b = tid; b <= p.B; b += n_threads) p.q_begin[b] = refused ? 0 : rows[b];
  // every CTA has read the lengths and the count: they may be written, in place too
  if (n_ctas > 1)
    pq::cluster_sync();
  else
    __syncthreads();
  for (int b = tid; b < p.B; b += n_threads) p.len_out[b] = refused ? len[b] : len[b] + (rows[b + 1] - rows[b]);
  if (tid == 0) *p.n_free_out = refused ? n_free : n_free - static_cast<int32_t>(need);
}

// Shared memory: pages[B + 1], len[B].
__global__ void __launch_bounds__(PG_THREADS) page_release_kernel(const PlanParams p) {
  extern __shared__ __align__(16) int32_t pg_smem[];
  __shared__ int64_t part[PG_THREADS / 32];
  __shared__ int bad, no_id;
  int32_t *pages = pg_smem, *len = pages + p.B + 1;
  pq::pdl_wait();
  if (threadIdx.x == 0) bad = no_id = 0;
  __syncthreads();
  const int32_t n_free = pq::ld_dep(p.n_free);
  const int64_t capacity = static_cast<int64_t>(p.max_pages) << p.page_log2;
  for (int b = threadIdx.x; b < p.B; b += PG_THREADS) {
    const int32_t l = pq::ld_dep(p.len + b);
    const bool done = pq::ld_dep(p.n_new + b) != 0;
    const bool ok = l >= 0 && l <= capacity;
    if (done && !ok) bad = 1;
    len[b] = l;
    pages[b] = done && ok ? pages_of(l, p.page_log2) : 0;
  }
  __syncthreads();
  const int64_t total = pq::block_scan<PG_THREADS>(pages, p.B, part);
  bool refused = bad || n_free < 0 || n_free + total > p.n_pages;
  const int n_ctas = gridDim.x, tid = blockIdx.x * PG_THREADS + threadIdx.x, n_threads = n_ctas * PG_THREADS;
  auto page_id = [&](int64_t k) {  // the k-th page that goes back
    const int b = pq::find_segment(pages, p.B, static_cast<int32_t>(k));
    return pq::ld_dep(p.table + static_cast<int64_t>(b) * p.max_pages + (k - pages[b]));
  };
  // Are all of them ids? Every thread looks at its own (the first stays in a register), the CTAs tell one another.
  int32_t first = 0;
  if (!refused) {
    bool none = false;
    for (int64_t k = tid; k < total; k += n_threads) {
      const int32_t id = page_id(k);
      if (k == tid) first = id;
      none |= id < 0 || id >= p.n_pages;
    }
    if (none) no_id = 1;
    if (n_ctas > 1) {
      pq::cluster_sync();
      refused = __syncthreads_or(threadIdx.x < n_ctas && pq::ld_cluster(&no_id, threadIdx.x));
    } else {
      __syncthreads();
      refused = no_id;
    }
  }
  if (!refused) {
    for (int64_t k = tid; k < total; k += n_threads) p.free_list[n_free + k] = k == tid ? first : page_id(k);
  } else if (tid == 0) {
    pq::report(p.status, PQ_ERR_SHAPE);
  }
  if (n_ctas > 1)
    pq::cluster_sync();
  else
    __syncthreads();
  for (int b = tid; b < p.B; b += n_threads) p.len_out[b] = !refused && pq::ld_dep(p.n_new + b) != 0 ? 0 : len[b];
  if (tid == 0) *p.n_free_out = refused ? n_free : n_free + static_cast<int32_t>(total);
}

// The last tokens of a sequence leave: of the rows q_begin[b] .. q_begin[b + 1] - 1, which are the last of the cached ones, the first n_kept[b] stay. Shared memory:
// pages[B + 1], len[B] (after). The moves that follow in every layer's cache see the lengths and the counts alone, and a refusal for one sequence, for the list or for an id
// leaves the lengths of all as they were: the counts are then set to -1, which no move follows.
__global__ void __launch_bounds__(PG_THREADS) page_keep_kernel(const PlanParams p) {
  extern __shared__ __align__(16) int32_t pg_smem[];
  __shared__ int64_t part[PG_THREADS / 32];
  __shared__ int bad, no_id;
  int32_t *pages = pg_smem, *len = pages + p.B + 1;
  pq::pdl_wait();
  if (threadIdx.x == 0) bad = no_id = 0;
  __syncthreads();
  const int32_t n_free = pq::ld_dep(p.n_free);
  const int64_t capacity = static_cast<int64_t>(p.max_pages) << p.page_log2;
  for (int b = threadIdx.x; b < p.B; b += PG_THREADS) {
    const int64_t l = pq::ld_dep(p.len + b), k = pq::ld_dep(p.n_new + b), n = static_cast<int64_t>(pq::ld_dep(p.q_begin + b + 1)) - pq::ld_dep(p.q_begin + b);
    const bool ok = l >= 0 && l <= capacity && k >= 0 && k <= n && n <= l;
    if (!ok) bad = 1;
    len[b] = ok ? static_cast<int32_t>(l - n + k) : 0;
    pages[b] = ok ? pages_of(static_cast<int32_t>(l), p.page_log2) - pages_of(len[b], p.page_log2) : 0;
  }
  __syncthreads();
  const int64_t total = pq::block_scan<PG_THREADS>(pages, p.B, part);
  bool refused = bad || n_free < 0 || n_free + total > p.n_pages;
  const int n_ctas = gridDim.x, tid = blockIdx.x * PG_THREADS + threadIdx.x, n_threads = n_ctas * PG_THREADS;
  auto page_id = [&](int64_t k) {  // the k-th page that goes back
    const int b = pq::find_segment(pages, p.B, static_cast<int32_t>(k));
    return pq::ld_dep(p.table + static_cast<int64_t>(b) * p.max_pages + pages_of(len[b], p.page_log2) + (k - pages[b]));
  };
  int32_t first = 0;
  if (!refused) {  // are all of them ids
    bool none = false;
    for (int64_t k = tid; k < total; k += n_threads) {
      const int32_t id = page_id(k);
      if (k == tid) first = id;
      none |= id < 0 || id >= p.n_pages;
    }
    if (none) no_id = 1;
    if (n_ctas > 1) {
      pq::cluster_sync();
      refused = __syncthreads_or(threadIdx.x < n_ctas && pq::ld_cluster(&no_id, threadIdx.x));
    } else {
      __syncthreads();
      refused = no_id;
    }
  }
  if (!refused) {
    for (int64_t k = tid; k < total; k += n_threads) p.free_list[n_free + k] = k == tid ? first : page_id(k);
  } else if (tid == 0) {
    pq::report(p.status, PQ_ERR_SHAPE);
  }
  if (n_ctas > 1) pq::cluster_sync();  // every CTA has read the lengths and the counts
  __syncthreads();
  for (int b = tid; b < p.B; b += n_threads) {
    p.len_out[b] = refused ? pq::ld_dep(p.len + b) : len[b];
    if (refused) p.n_kept[b] = -1;
  }
  if (tid == 0) *p.n_free_out = refused ? n_free : n_free + static_cast<int32_t>(total);
}

// Bytes of dynamic shared memory of `arrays` arrays over the sequences, some of them one longer.
constexpr size_t pg_smem_bytes(int64_t B, int arrays, int longer) { return (static_cast<size_t>(arrays) * B + longer) * sizeof(int32_t); }

// The kernel's limit on shared memory belongs to the device, not to the call or the context: it is set once, to the most that any call takes, so that the calls of
// another host thread never find it lower.
pq_status launch(const pq_ctx* ctx, void (*kern)(const PlanParams), std::atomic<bool> (&limit_set)[64], const PlanParams& p, int64_t items, int arrays, int longer,
                 cudaStream_t st) {
  if (ctx->device < 0 || ctx->device >= 64) return PQ_ERR_UNSUPPORTED;
  const size_t smem = pg_smem_bytes(p.B, arrays, longer);
  if (!limit_set[ctx->device].load(std::memory_order_relaxed)) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(pg_smem_bytes(PQ_PAGED_MAX_SEQS, arrays, longer))) != cudaSuccess) {
      cudaGetLastError();
      return PQ_ERR_CUDA;
    }
    limit_set[ctx->device].store(true, std::memory_order_relaxed);
  }
  const int ctas = items > PG_ONE_CTA ? PG_CLUSTER : 1;
  return pq_launch_cluster_pdl(kern, dim3(ctas), PG_THREADS, smem, ctas, st, p);
}

PlanParams base_params(pq_ctx* ctx, const pq_pages* c) {
  PlanParams p{};
  p.table = c->table, p.len = c->len, p.free_list = c->free_list, p.n_free = c->n_free;
  p.status = ctx->d_status;
  p.B = c->B, p.max_pages = c->max_pages, p.page_log2 = pq_page_log2(c->page), p.n_pages = c->n_pages;
  return p;
}

}  // namespace

extern "C" pq_status pq_page_plan(pq_ctx* ctx, const pq_pages* pages, const int32_t* n_new, int32_t pos0, int64_t n_rows, int32_t* q_begin,
                                  int64_t* slot, int32_t* pos, int32_t* len_out, int32_t* n_free_out, void* stream) {
  if (!ctx || !q_begin || !n_free_out || n_rows < 0 || pos0 < 0 || (n_rows > 0 && (!slot || !pos))) return PQ_ERR_INVALID_ARG;
  const pq_status st = pq_check_pages(pages);
  if (st != PQ_OK) return st;
  if (pages->B > 0 && (!n_new || !len_out)) return PQ_ERR_INVALID_ARG;
  if (n_rows > 0x7fffffffll) return PQ_ERR_SHAPE;
  if (static_cast<int64_t>(pages->max_pages) * pages->page + pos0 > 0x7fffffffll) return PQ_ERR_SHAPE;  // a position would not fit
  if (pq_misaligned16(slot) || pq_misaligned16(pos)) return PQ_ERR_ALIGN;
  PlanParams p = base_params(ctx, pages);
  p.n_new = n_new, p.pos0 = pos0, p.n_rows = n_rows, p.q_begin = q_begin, p.slot = slot, p.pos = pos, p.len_out = len_out, p.n_free_out = n_free_out;
  static std::atomic<bool> limit_set[64] = {};
  return launch(ctx, page_plan_kernel, limit_set, p, n_rows, 3, 2, static_cast<cudaStream_t>(stream));
}

extern "C" pq_status pq_page_release(pq_ctx* ctx, const pq_pages* pages, const int32_t* done, int32_t* len_out, int32_t* n_free_out, void* stream) {
  if (!ctx || !n_free_out) return PQ_ERR_INVALID_ARG;
  const pq_status st = pq_check_pages(pages);
  if (st != PQ_OK) return st;
  if (pages->B > 0 && (!done || !len_out)) return PQ_ERR_INVALID_ARG;
  PlanParams p = base_params(ctx, pages);
  p.n_new = done, p.len_out = len_out, p.n_free_out = n_free_out;
  static std::atomic<bool> limit_set[64] = {};
  return launch(ctx, page_release_kernel, limit_set, p, pages->n_pages, 2, 1, static_cast<cudaStream_t>(stream));
}

extern "C" pq_status pq_page_keep(pq_ctx* ctx, const pq_pages* pages, const int32_t* q_begin, int32_t* n_kept, int32_t* len_out, int32_t* n_free_out, void* stream) {
  if (!ctx || !n_free_out) return PQ_ERR_INVALID_ARG;
  const pq_status st = pq_check_pages(pages);
  if (st != PQ_OK) return st;
  if (pages->B > 0 && (!q_begin || !n_kept || !len_out)) return PQ_ERR_INVALID_ARG;
  PlanParams p = base_params(ctx, pages);
  p.q_begin = const_cast<int32_t*>(q_begin), p.n_new = p.n_kept = n_kept, p.len_out = len_out, p.n_free_out = n_free_out;
  static std::atomic<bool> limit_set[64] = {};
  return launch(ctx, page_keep_kernel, limit_set, p, pages->B, 2, 1, static_cast<cudaStream_t>(stream));
}
