// What the kernels of the paged KV4 cache share: checks of the descriptors, the cluster launch, prefix sums over a CTA.
#pragma once

#include "pq_common.cuh"

#define PQ_PAGED_MAX_SEQS 8192
#define PQ_PAGED_MAX_PREFIX 64
#define PQ_PAGED_MAX_GROUP 8  // query heads per KV head

static inline bool pq_misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

static inline int pq_page_log2(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

static inline pq_status pq_check_pages(const pq_pages* c) {
  if (!c || !c->n_free || c->B < 0 || c->max_pages < 0 || c->n_pages < 0) return PQ_ERR_INVALID_ARG;
  if ((c->B > 0 && (!c->len || (c->max_pages > 0 && !c->table))) || (c->n_pages > 0 && !c->free_list)) return PQ_ERR_INVALID_ARG;  // (an empty array has no address)
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return PQ_ERR_SHAPE;
  if (c->B > PQ_PAGED_MAX_SEQS || static_cast<int64_t>(c->max_pages) * c->page > (1ll << 30)) return PQ_ERR_SHAPE;  // (a key's number and a step beyond it fit 32 bits)
  return PQ_OK;
}

static inline pq_status pq_check_paged(const pq_kv4_paged* c) {
  if (!c) return PQ_ERR_INVALID_ARG;
  const pq_status st = pq_check_pages(&c->pages);
  if (st != PQ_OK) return st;
  if ((!c->codes && c->pages.n_pages > 0) || (!c->steps && (!c->s_k || !c->s_v))) return PQ_ERR_INVALID_ARG;
  if (c->Hq <= 0 || c->Hkv <= 0 || c->n_prefix < 0 || (c->n_prefix > 0 && (!c->prefix_k || !c->prefix_v))) return PQ_ERR_INVALID_ARG;
  if (c->D != 128 || c->Hq % c->Hkv != 0 || c->Hq / c->Hkv > PQ_PAGED_MAX_GROUP || c->n_prefix > PQ_PAGED_MAX_PREFIX || c->Hkv > 4096)
    return PQ_ERR_SHAPE;
  if (pq_misaligned16(c->codes) || pq_misaligned16(c->steps) ||
      (c->n_prefix > 0 && (pq_misaligned16(c->prefix_k) || pq_misaligned16(c->prefix_v))))
    return PQ_ERR_ALIGN;
  return PQ_OK;
}

// Launch as clusters of `cluster` CTAs along x, behind the kernel before it without a launch gap: the kernel executes pq::pdl_wait()
// before it reads or writes anything.
template <typename... P, typename... A>
static inline pq_status pq_launch_cluster_pdl(void (*kern)(P...), dim3 grid, int block, size_t smem, int cluster, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...) != cudaSuccess) {
    cudaGetLastError();
    return PQ_ERR_CUDA;
  }
  return pq_launch_status();
}

namespace pq {

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The counterpart of a shared variable in CTA `rank` of the cluster.
__device__ __forceinline__ int ld_cluster(const int* p, int rank) {
  uint32_t a;
  int v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ int64_t ld_dep(const int64_t* p) {
  int64_t v;
  asm volatile("ld.global.b64 %0, [%1];" : "=l"(v) : "l"(p));
  return v;
}

// First b in [0, n) with begin[b + 1] > x (begin[0 .. n] ascending, begin[n] > x): the sequence that holds element x.
__device__ __forceinline__ int find_segment(const int32_t* begin, int n, int32_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (begin[mid + 1] > x)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

// In place: v[0 .. n] becomes the exclusive prefix sums of v[0 .. n - 1] (v[n] the total), by all THREADS threads; returns the total in 64
// bits. `part`: THREADS / 32 values of shared memory. Every thread takes a contiguous stretch, a warp scan joins the stretches.
template <int THREADS>
__device__ int64_t block_scan(int32_t* v, int n, int64_t* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = (n + THREADS - 1) / THREADS;
  const int lo = min(n, static_cast<int>(threadIdx.x) * per), hi = min(n, lo + per);
  int64_t sum = 0;
  for (int i = lo; i < hi; ++i) sum += v[i];
  int64_t inc = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= d) inc += o;
  }
  if (lane == 31) part[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    int64_t w = lane < THREADS / 32 ? part[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w += o;
    }
    if (lane < THREADS / 32) part[lane] = w;
  }
  __syncthreads();
  int64_t at = inc - sum + (warp > 0 ? part[warp - 1] : 0);
  const int64_t total = part[THREADS / 32 - 1];
  for (int i = lo; i < hi; ++i) {
    const int32_t x = v[i];
    v[i] = static_cast<int32_t>(at);
    at += x;
  }
  if (threadIdx.x == 0) v[n] = static_cast<int32_t>(total);
  __syncthreads();
  return total;
}

}  // namespace pq
