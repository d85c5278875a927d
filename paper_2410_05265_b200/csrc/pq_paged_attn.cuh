// Parameters and small device helpers of the kernels of paged attention: for single tokens (pq_paged_decode.cu), for sequences of several rows
// (pq_paged_prefill.cu), both with a form for windows, and for drafted trees (pq_paged_tree.cu).
#pragma once

#include <math.h>

#include "pq_paged.cuh"

struct PagedAttnParams {
  const __nv_bfloat16* q;
  int64_t ldq;
  __nv_bfloat16* out;
  const int32_t* q_begin;
  const int32_t* len;
  const int32_t* table;
  const __half* prefix_k;
  const __half* prefix_v;
  const uint8_t* codes;
  const float* steps;  // null: the static steps
  const float* s_k;
  const float* s_v;
  float* ws_o;   // partial outputs in value units: [2 * workers] x rows x 128
  float* ws_ml;  // their reference exponents (log2 units) and denominators
  uint32_t* tickets;
  int32_t* status;
  long long wait_clocks;
  float scale2;  // sm_scale log2(e)
  int32_t n_rows, B, max_pages, page_log2, n_pages, Hq, Hkv, G, n_prefix, max_new;
  int32_t csize;    // decode: CTAs of a worker (one cluster)
  int32_t workers;  // 0: one worker per (sequence, KV head)
  int32_t window;       // 0: none; else the cached keys at the places c - window + 1 .. c of a token at place c, and those before n_sink
  int32_t n_sink;
  const uint32_t* mask;  // null, or [n_rows][mask_words]: the drafts of its sequence that a row sees
  int32_t mask_words;
};

// One mbarrier try_wait may suspend its thread for thousands of clocks (three of them on a barrier that nothing completes take 15700), in which an ordinary wait ends. A
// limit below that is kept by forms of the kernels that poll instead (POLL): with them a test makes waits run out. As a choice inside the kernels it
// took 2 to 4 % of them.
#define PQ_SUSPENDED_CLOCKS 16384

// Tickets 0 .. 15 belong to the appends, those from PQ_N_TICKETS / 2 on to the one-launch decode step. The decode attention of the contiguous cache counts from 16 on,
// too: every call leaves its tickets at zero, and calls of a context are in stream order.
#define PQ_PAGED_TICKET0 16
#define PQ_PAGED_MAX_WORKERS 4096

size_t pq_paged_decode_ws_bytes(const pq_ctx* ctx, const pq_kv4_paged* c);
size_t pq_paged_prefill_ws_bytes(const pq_ctx* ctx);
pq_status pq_paged_prefill_launch(pq_ctx* ctx, PagedAttnParams p, void* ws, cudaStream_t st);
size_t pq_paged_tree_ws_bytes(const pq_ctx* ctx);
pq_status pq_paged_tree_launch(pq_ctx* ctx, PagedAttnParams p, int64_t max_len, void* ws, cudaStream_t st);
pq_status pq_paged_decode_launch(pq_ctx* ctx, const pq_kv4_paged* c, PagedAttnParams p, int64_t max_len, void* ws, cudaStream_t st);

namespace pq {

__device__ __forceinline__ float lg2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Own steps: the exponent of a weight carries log2 of the value's step, w = 2^(s + log2 step - m), and the denominator is the sum of w / step. Steps may lie 2^120
// apart, and a key whose weight is 2^-120 of the largest still belongs in the denominator. So w is formed PQ_UP octaves up (2^(15 + 60) at most), where fp32
// reaches down to 2^-186 of the reference, 1 / step is kept PQ_UP octaves down (no product leaves fp32), and what goes to the products is
// w 2^-PQ_UP. What is lost of the denominator lies 2^-50 below the rest of it.
constexpr float PQ_UP = 60.0f, PQ_DOWN = 0x1p-60f;
// x 2^d for d <= 0, the denominator moved to another reference: in two factors, since references may then lie further apart than fp32 reaches.
__device__ __forceinline__ float at_reference(float x, float d) {
  return x * ex2_approx(fmaxf(d, -120.0f)) * ex2_approx(fminf(d + 120.0f, 0.0f));
}
// (a & M) ^ C in one LOP3; the constants are immediates
template <uint32_t M, uint32_t C>
__device__ __forceinline__ uint32_t and_xor(uint32_t a) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(d) : "r"(a), "n"(M), "n"(C));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// 1-D bulk copy global -> shared, completion counted in bytes on an mbarrier.
__device__ __forceinline__ void bulk_load(uint32_t dst_smem, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst_smem), "l"(src), "r"(bytes),
               "r"(smem_u32(bar))
               : "memory");
}
// Is the phase over? Does not suspend.
__device__ __forceinline__ bool mbar_test_wait(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// One look at a wait, and a bounded wait.
template <bool POLL>
__device__ __forceinline__ bool mbar_look(uint64_t* bar, uint32_t parity) {
  return POLL ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity);
}
template <bool POLL>
__device__ __forceinline__ bool mbar_look_for(uint64_t* bar, uint32_t parity, long long limit) {
  if (!POLL) return mbar_wait_for(bar, parity, limit);
  const long long t0 = clock64();
  while (!mbar_test_wait(bar, parity))
    if (clock64() - t0 > limit) return false;
  return true;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}

}  // namespace pq
