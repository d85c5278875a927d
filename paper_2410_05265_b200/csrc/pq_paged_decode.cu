// Attention of single tokens (decode) over [full-precision prefix || paged 4-bit cache]: the sequences of a ragged batch that have one row.
//
// Bound by HBM in principle (128 bytes, with own steps 136, per key and KV head; the query heads of a group share them), in practice by the ALU close behind: a
// block of 32 keys costs about 580 warp instructions, a logic instruction for every two codes among them (45 - 54 % of that pipe, 43 - 51 % of the issue
// slots). A long cache streams at 0.72 of the measured copy rate and a call costs 20 - 26 us besides (prefix sums 2, first blocks 3.5, a stretch's
// pieces merged 2 - 6 each, the joined pairs 2, CTAs of an SM that end one after another). 48 ragged sequences to 6000 tokens, 32 heads on 8: 64 us
// (own steps), 56 (static); 5 ragged to 50000, 64 heads: 60; one of 1021: 6.7.
// Tried: rings of three and four blocks, five CTAs to an SM (no difference), multiplications for the shifts (slower), clusters of 1, 2 and 4 where 8 are
// taken (2 % either way), longer stretches for the CTAs that an SM favours (2 - 5 % faster with eight heads to a group of four, 3 % slower with more).
//
// A worker is one CTA or a cluster of CTAs, four warps each. Work is counted in rounds of 128 keys of a (sequence, KV head) pair.
//   one worker per pair (workers == 0): short caches, one wave of CTAs; the cluster merges on chip, the result is final.
//   a fixed number of workers: every worker takes an equal stretch of the rounds of all pairs laid end to end (a prefix sum over the lengths, which
//     every CTA forms for itself), whatever the lengths are. A pair inside one stretch is final; a pair that several stretches share
//     leaves partials in the workspace, and the last worker to finish merges them in the order of the workers, so that results do
//     not depend on who came last.
// Warps work alone: warp w of the worker takes every 4 * csize-th block of 32 keys, brings it into its own ring of staging slots
// by bulk copies (16 rows of keys or values each, page by page; the ids of the pages of the next block are loaded one block ahead), and no
// CTA barrier stands in the key loop. The ring runs on across the pairs of a stretch.
//   scores   S^T[key, head] with the fp16 MMA, keys on the 16-row side. code + 8 is taken as the fp16 number whose bits it is (a subnormal, (code + 8) 2^-24;
//            the odd nibbles four bits up, with q / 16): one LOP3 for two codes, and 8 sum(q) is taken off each score. The offset is of
//            the codes' own size, so that fp32 sums lose by it what sums of values of 8 steps lose. The query is scaled by a power of two per head, so that every bf16
//            query fits fp16.
//   softmax  in log2 units against a reference exponent per head that moves only when a score exceeds it by more than DP_HEADROOM
//   output   O^T = V^T P^T with the fp16 MMA, head dims on the 16-row side, codes + 8 as above; one more MMA over codes of zero gives what the offset adds
//            and, for static steps, the denominator, both from the same rounded P. Own steps: the exponent of a weight takes log2 of the value's step with it, w = 2^(s + log2 step - m), so
//            that fp16 holds the largest of what enters the sum whatever the steps are; the denominator is the sum of w / step in fp32 (PQ_UP).
#include <atomic>

#include "pq_paged_attn.cuh"

namespace {

constexpr int DP_WARPS = 4;
constexpr int DP_THREADS = DP_WARPS * 32;
constexpr int DP_ROUND = 128;  // keys of a unit of work
constexpr int DP_BLOCK = 32;   // keys of a warp's step
constexpr int DP_ROWS = 8;     // query heads per KV head the MMA tile carries
constexpr int DP_SO_STRIDE = 136;
constexpr float DP_HEADROOM = 15.0f;  // log2 units: weights stay below 2^16, inside fp16
constexpr int DP_SLOTS = 2;           // staged blocks per warp

// Bytes of a staging slot: 32 rows of keys, 32 rows of values, with own steps 32 + 32 floats.
__host__ __device__ constexpr int slot_bytes(bool dyn) { return DP_BLOCK * 128 + (dyn ? DP_BLOCK * 8 : 0); }
// Dynamic shared memory: staging, the warps' partial outputs, prefix scores, and (equal stretches) rounds and lengths of the sequences.
constexpr size_t dynamic_smem(bool dyn, int G, int n_prefix, int seqs) {
  return DP_WARPS * DP_SLOTS * slot_bytes(dyn) + static_cast<size_t>(DP_WARPS) * G * DP_SO_STRIDE * 4 + static_cast<size_t>(G) * n_prefix * 4 +
         (seqs > 0 ? (3 * static_cast<size_t>(seqs) + 1) * 4 : 0);
}
constexpr size_t smem_kb(size_t bytes) { return (bytes + 1023) / 1024; }
constexpr size_t DP_MAX_KB = smem_kb(dynamic_smem(true, DP_ROWS, PQ_PAGED_MAX_PREFIX, PQ_PAGED_MAX_SEQS));

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two codes of a word as (code + 8) 2^-24 (nibbles 0 and 4) and (code + 8) 2^-20 (nibbles 1 and 5), fp16 subnormals: their bits are the numbers.
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) { return pq::and_xor<0x000F000Fu, 0x00080008u>(w); }
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) { return pq::and_xor<0x00F000F0u, 0x00800080u>(w); }
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t map_cta(uint32_t smem_addr, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ float2 ld_cluster_f2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ void store_out(__nv_bfloat16* dst, const float4& a, float inv) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(a.x * inv, a.y * inv), hi = __floats2bfloat162_rn(a.z * inv, a.w * inv);
  uint2 v;
  v.x = *reinterpret_cast<const uint32_t*>(&lo), v.y = *reinterpret_cast<const uint32_t*>(&hi);
  *reinterpret_cast<uint2*>(dst) = v;
}

// The rows r0 .. r1 - 1 of a sequence: is it this kernel's, and is it one that has to be reported (the rule of the kernel for several rows).
__device__ __forceinline__ bool one_row(const PagedAttnParams& p, int r0, int r1) { return r0 >= 0 && r0 < p.n_rows && r1 == r0 + 1; }
__device__ __forceinline__ bool odd_rows(const PagedAttnParams& p, int r0, int r1, bool bad_len) {
  const int64_t n = static_cast<int64_t>(r1) - r0;
  return n > p.max_new || n < 0 || (n > 0 && (r0 < 0 || r1 > p.n_rows || bad_len));
}

// WIDE: clusters of sixteen, for a few long sequences (their merge in the other kernel would cost it registers).
template <bool DYN, bool WIDE, bool POLL>
__global__ void __launch_bounds__(DP_THREADS, 4) paged_decode_kernel(const PagedAttnParams p) {
  constexpr int SLOT = slot_bytes(DYN);
  extern __shared__ __align__(128) uint8_t dp_smem[];
  float* sm_o = reinterpret_cast<float*>(dp_smem + DP_WARPS * DP_SLOTS * SLOT);  // [warp][head][DP_SO_STRIDE]; dim 16a + 2b + c at 16b + 2a + c
  float* cl_o = sm_o;  // [head] rows of the first warp, once they have been read: this CTA's partial of a cluster, dims in order
  float* sm_pre = sm_o + DP_WARPS * p.G * DP_SO_STRIDE;                     // [head][n_prefix]
  int32_t* scan = reinterpret_cast<int32_t*>(sm_pre + p.G * p.n_prefix);    // [B + 1] rounds before a sequence (workers > 0)
  int32_t* lens = scan + p.B + 1;                                           // [B]
  int32_t* rows = lens + p.B;                                               // [B] the row of a sequence that has exactly one
  __shared__ __align__(8) uint64_t full[DP_WARPS][DP_SLOTS];
  __shared__ float sm_ml[DP_WARPS][DP_ROWS][2];
  __shared__ float2 cl_ml[DP_ROWS];
  __shared__ uint4 sm_q[DP_ROWS][17];  // the queries as MMA operand; a padded row keeps the eight heads of a load apart
  __shared__ float2 sm_f[DP_ROWS];
  __shared__ int64_t part[DP_WARPS];
  __shared__ float4 sm_step[DYN ? DP_WARPS : 1][DYN ? DP_BLOCK : 1];
  __shared__ int sm_last[2];
  __shared__ int4 sm_shared[2];  // (row, KV head, first and last worker)

  const int csize = p.csize, worker = blockIdx.x / csize, rank = blockIdx.x % csize;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int G = p.G, page_log2 = p.page_log2;
  // Behind the kernel for several rows (max_new > 1) there is no wait here: that kernel lets this one start behind its own wait for what came before, and the
  // two have nothing in common but what both read. So that it ends no earlier than the other, its last CTA waits when it is done (one is enough, and
  // the others give their SMs free). What a wait would do for the SM's L1 the fence does: loads behind it see what was written before the launch.
  const bool beside = p.max_new > 1;
  if (beside) {
    __threadfence();
  } else {
    pq::pdl_wait();
    pq::pdl_trigger();
  }
  auto leave = [&]() {
    if (beside && blockIdx.x == gridDim.x - 1) pq::pdl_wait();
  };
  if (lane == 0) {
    for (int s = 0; s < DP_SLOTS; ++s) pq::mbar_init(&full[warp][s], 1);
    pq::mbar_fence_init();
  }
  const int64_t capacity = static_cast<int64_t>(p.max_pages) << page_log2;
  auto clip_len = [&](int l) { return l < 0 ? 0 : l > capacity ? static_cast<int>(capacity) : l; };

  // ---- this worker's stretch of units [u0, u1)
  int u0 = 0, u1 = 0, b_direct = 0, h_direct = 0, len_direct = 0, row_direct = 0, n_workers = 1, U = 0;
  const bool direct = p.workers == 0;
  if (direct) {
    b_direct = worker / p.Hkv, h_direct = worker % p.Hkv;
    const int l = pq::ld_dep(p.len + b_direct);
    len_direct = clip_len(l);
    const int r0 = pq::ld_dep(p.q_begin + b_direct), r1 = pq::ld_dep(p.q_begin + b_direct + 1);
    if (threadIdx.x == 0 && odd_rows(p, r0, r1, l != len_direct)) pq::report(p.status, PQ_ERR_SHAPE);
    if (!one_row(p, r0, r1)) return leave();  // the whole cluster alike
    row_direct = r0;
    u1 = max(1, (len_direct + DP_ROUND - 1) / DP_ROUND);
    __syncwarp();
  } else {
    bool odd = false;
    for (int b = threadIdx.x; b < p.B; b += DP_THREADS) {
      const int l = pq::ld_dep(p.len + b), lc = clip_len(l);
      const int r0 = pq::ld_dep(p.q_begin + b), r1 = pq::ld_dep(p.q_begin + b + 1);
      odd |= odd_rows(p, r0, r1, l != lc);
      lens[b] = lc, rows[b] = r0;
      scan[b] = one_row(p, r0, r1) ? max(1, (lc + DP_ROUND - 1) / DP_ROUND) : 0;
    }
    __syncthreads();
    const int64_t total = pq::block_scan<DP_THREADS>(scan, p.B, part) * p.Hkv;
    if (total > 0x7fffffffll) odd = true;  // (more keys than the chip's memory holds)
    if (odd && blockIdx.x == 0) pq::report(p.status, PQ_ERR_SHAPE);
    if (total > 0x7fffffffll || total == 0) return leave();
    U = static_cast<int>(total);
    n_workers = min(p.workers, max(1, U / csize));  // at least a round to a CTA
    if (worker >= n_workers) return leave();
    u0 = static_cast<int>(static_cast<int64_t>(U) * worker / n_workers);
    u1 = static_cast<int>(static_cast<int64_t>(U) * (worker + 1) / n_workers);
  }
  struct Piece {
    int b, h, r0, r1, rounds, len;  // rounds r0 .. r1 - 1 of the `rounds` of the pair
  };
  auto first_piece = [&]() {
    Piece x;
    if (direct) {
      x.b = b_direct, x.h = h_direct, x.r0 = 0, x.r1 = x.rounds = u1, x.len = len_direct;
      return x;
    }
    x.b = pq::find_segment(scan, p.B, u0 / p.Hkv);
    const int before = scan[x.b];
    x.rounds = scan[x.b + 1] - before;
    const int rel = u0 - before * p.Hkv;
    x.h = rel / x.rounds;
    x.r0 = rel - x.h * x.rounds;
    x.r1 = min(x.rounds, x.r0 + (u1 - u0));
    x.len = lens[x.b];
    return x;
  };
  auto advance = [&](Piece& x, int u) {  // to the piece that begins at unit u < u1
    if (++x.h == p.Hkv) {
      x.h = 0;
      do ++x.b;
      while (scan[x.b + 1] == scan[x.b]);
      x.rounds = scan[x.b + 1] - scan[x.b];
      x.len = lens[x.b];
    }
    x.r0 = 0, x.r1 = min(x.rounds, u1 - u);
  };

  // ---- staging: the cursor of what is requested runs ahead of the computation, across the pieces of the stretch
  const int first_key = (rank * DP_WARPS + warp) * DP_BLOCK, stride = csize * DP_WARPS * DP_BLOCK;
  Piece is_piece = first_piece();
  int is_u = u0, is_key = 0, is_end = 0, is_id = -1;
  bool is_ok = false, timed_out = false;
  const uint8_t* const stage = dp_smem + warp * DP_SLOTS * SLOT;
  const uint32_t stage0 = pq::smem_u32(stage);
  // lanes 0 .. 3 copy rows (group of 16 keys = bit 1, keys or values = bit 0), lanes 4 .. 7 the steps of the same
  const int cp_group = (lane >> 1) & 1, cp_kv = lane & 1, page_mask = (1 << page_log2) - 1;
  const bool cp_steps = DYN && (lane & 4), cp_lane = lane < (DYN ? 8 : 4);
  const int cp_unit = cp_steps ? 4 : 64;  // bytes of a row
  const uint32_t cp_bytes = cp_steps ? 64 : 1024;
  const uint32_t cp_dst = stage0 + (cp_steps ? DP_BLOCK * 128 + cp_kv * (DP_BLOCK * 4) + cp_group * 64 : cp_kv * (DP_BLOCK * 64) + cp_group * 1024);
  const uint8_t* const cp_base = cp_steps ? reinterpret_cast<const uint8_t*>(p.steps) : p.codes;
  const int64_t page_bytes = static_cast<int64_t>(p.Hkv * 2 * cp_unit) << page_log2;
  const uint8_t* is_src = cp_base;  // the head's rows inside a page
  const int32_t* is_row = p.table;
  // The page of this lane's group of the cursor's block. An id that is none is reported and page 0 read in its place.
  auto fetch_id = [&]() {
    const int k = is_key + 16 * cp_group;
    is_id = cp_lane && k < is_end ? pq::ld_dep(is_row + (k >> page_log2)) : -1;
  };
  auto next_piece = [&]() {
    is_ok = false;
    while (is_u < u1) {
      if (is_u != u0) advance(is_piece, is_u);
      const Piece& x = is_piece;
      is_u += x.r1 - x.r0;
      is_key = x.r0 * DP_ROUND + first_key, is_end = min(x.len, x.r1 * DP_ROUND);
      if (is_key < is_end) {
        is_ok = true;
        is_row = p.table + static_cast<int64_t>(x.b) * p.max_pages;
        is_src = cp_base + ((static_cast<int64_t>(2 * x.h + cp_kv) * cp_unit) << page_log2);
        fetch_id();
        break;
      }
    }
  };
  int n_issued = 0, n_done = 0;
  auto issue = [&]() {  // the cursor's block into the next slot; the whole warp
    if (!is_ok) return;
    const int s = n_issued % DP_SLOTS, k = is_key + 16 * cp_group;
    uint64_t* bar = &full[warp][s];
    const bool both = is_key + 16 < is_end;
    if (lane == 0) pq::mbar_arrive_expect_tx(bar, (both ? 2u : 1u) * (2 * 1024 + (DYN ? 2 * 64 : 0)));
    if (cp_lane && k < is_end) {
      if (static_cast<uint32_t>(is_id) >= static_cast<uint32_t>(p.n_pages)) {
        pq::report(p.status, PQ_ERR_SHAPE);
        is_id = 0;
      }
      pq::bulk_load(cp_dst + s * SLOT, is_src + is_id * page_bytes + (k & page_mask) * cp_unit, cp_bytes, bar);
    }
    ++n_issued;
    is_key += stride;
    if (is_key < is_end)
      fetch_id();
    else
      next_piece();
  };
  // What a piece needs first, requested while the piece before it is merged: 8 dims of a query head (sixteen threads to a head) and the steps.
  Piece x = first_piece();
  int row = 0;
  uint4 q_raw;
  float s_k_h, s_v_h;
  auto request = [&]() {
    row = direct ? row_direct : rows[x.b];
    const int head = threadIdx.x >> 4;
    const __nv_bfloat16* q0 = p.q + row * p.ldq + static_cast<int64_t>(x.h) * G * 128;
    q_raw = head < G ? pq::ld_dep(reinterpret_cast<const uint4*>(q0 + head * 128) + (threadIdx.x & 15)) : make_uint4(0, 0, 0, 0);
    s_k_h = DYN ? 1.0f : pq::ld_dep(p.s_k + x.h), s_v_h = DYN ? 1.0f : pq::ld_dep(p.s_v + x.h);
  };
  request();
  next_piece();
  for (int s = 0; s < DP_SLOTS; ++s) issue();
  int n_shared = 0;  // pairs this worker shares with others: its first and its last
  for (int u = u0; u < u1;) {
    const int kend = min(x.len, x.r1 * DP_ROUND);
    const bool whole = x.r0 == 0 && x.r1 == x.rounds;
    const bool has_prefix = x.r0 == 0 && rank == csize - 1 && p.n_prefix > 0;  // the CTA with the fewest blocks of the pair's first stretch
    const __nv_bfloat16* q0 = p.q + row * p.ldq + static_cast<int64_t>(x.h) * G * 128;
    const float value_unit = s_v_h;
    __syncthreads();  // what the warps read of the piece before, they have read
    // ---- prefix keys in fp32: eight lanes per (head, key) pair, 16 dims each
    if (has_prefix) {
      const int n_pairs = G * p.n_prefix, sub = threadIdx.x & 7;
      for (int pair0 = 0; pair0 < n_pairs; pair0 += DP_THREADS / 8) {
        const int pair = pair0 + (threadIdx.x >> 3);
        const bool ok = pair < n_pairs;
        const int r = ok ? pair / p.n_prefix : 0, j = ok ? pair % p.n_prefix : 0;
        const uint4* qr = reinterpret_cast<const uint4*>(q0 + r * 128 + 16 * sub);
        const uint4* kr = reinterpret_cast<const uint4*>(p.prefix_k + (static_cast<int64_t>(x.h) * p.n_prefix + j) * 128 + 16 * sub);
        const uint4 qv[2] = {pq::ld_dep(qr), pq::ld_dep(qr + 1)}, kv[2] = {pq::ld_dep(kr), pq::ld_dep(kr + 1)};
        float acc = 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t qw[4] = {qv[i].x, qv[i].y, qv[i].z, qv[i].w}, kw[4] = {kv[i].x, kv[i].y, kv[i].z, kv[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 kf = __half22float2(*reinterpret_cast<const __half2*>(&kw[e]));
            acc = fmaf(__uint_as_float(qw[e] << 16), kf.x, acc);
            acc = fmaf(__uint_as_float(qw[e] & 0xFFFF0000u), kf.y, acc);
          }
        }
        acc += __shfl_xor_sync(0xffffffffu, acc, 1);
        acc += __shfl_xor_sync(0xffffffffu, acc, 2);
        acc += __shfl_xor_sync(0xffffffffu, acc, 4);
        if (ok && sub == 0) sm_pre[r * p.n_prefix + j] = acc * p.scale2;
      }
    }
    // ---- the query as B operand, made once per CTA: sixteen threads to a head, eight dims each. A 32-bit word of a packed key row holds the codes of dims
    // 8W..8W+7; nibble i of its low half is dim 8W+i, nibble i of its high half dim 8W+4+i. Fragment j of a lane holds (q[D], q[D+4]) in its
    // first and (q[D+1], q[D+5]) / 16 in its second register with D = 32t + 8(j>>1) + 2(j&1), of head g: the k rows 2t, 2t+1 and 2t+8,
    // 2t+9 of score MMA j.
    {
      const int head = threadIdx.x >> 4, part8 = threadIdx.x & 15;
      const uint32_t ww[4] = {q_raw.x, q_raw.y, q_raw.z, q_raw.w};
      uint32_t top = 0;  // largest magnitude of the head as bits
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, max(ww[e] & 0x7FFF0000u, (ww[e] << 16) & 0x7FFF0000u));
#pragma unroll
      for (int m = 1; m < 16; m <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
      // a power of two that brings the largest value to [2^8, 2^9); the scale and its inverse are normal numbers
      int ex = static_cast<int>(top >> 23);
      ex = ex < 10 ? 10 : ex > 254 ? 254 : ex;  // (a head of zeros, subnormals, infinities or NaN)
      const float up = __uint_as_float(static_cast<uint32_t>(127 + 8 + 127 - ex) << 23), down = 1.0f / up;
      float f[8], sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = __uint_as_float((e & 1) ? (ww[e >> 1] & 0xFFFF0000u) : (ww[e >> 1] << 16)) * up;
      uint32_t frag[4];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {  // score MMA j = 2 (dims / 8) + jj uses nibbles 2jj and 2jj + 1
        frag[2 * jj] = pq::pack_f16(f[2 * jj], f[2 * jj + 4]);
        frag[2 * jj + 1] = pq::pack_f16(f[2 * jj + 1] * 0.0625f, f[2 * jj + 5] * 0.0625f);
        // the offset is that of the values the MMA multiplies with
        const float2 e0 = __half22float2(*reinterpret_cast<const __half2*>(&frag[2 * jj])), e1 = __half22float2(*reinterpret_cast<const __half2*>(&frag[2 * jj + 1]));
        sum += (e0.x + e0.y) + 16.0f * (e1.x + e1.y);
      }
#pragma unroll
      for (int m = 1; m < 16; m <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
      const float unit = down * s_k_h * p.scale2;
      sm_q[head][part8] = make_uint4(frag[0], frag[1], frag[2], frag[3]);
      if (part8 == 0) sm_f[head] = make_float2(unit * 16777216.0f, -8.0f * sum * unit);
    }
    __syncthreads();
    uint32_t qb[8][2];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint4 v = sm_q[g][4 * t + w];
      qb[2 * w][0] = v.x, qb[2 * w][1] = v.y, qb[2 * w + 1][0] = v.z, qb[2 * w + 1][1] = v.w;
    }
    // a raw score r of heads 2t, 2t + 1 is r f + n in log2 units (DYN: times the key's step)
    const float2 fn0 = sm_f[2 * t], fn1 = sm_f[2 * t + 1];
    const float f_lo = fn0.x, f_hi = fn1.x, n_lo = fn0.y, n_hi = fn1.y;
    // Reference exponents of heads 2t and 2t + 1 (the same in all lanes of equal t). A head that does not exist keeps a huge one: its
    // weights are zero and it never asks for a move.
    float m0 = 2 * t < G ? -INFINITY : 1e30f, m1 = 2 * t + 1 < G ? -INFINITY : 1e30f;
    float z0 = m0 == -INFINITY ? 0.0f : m0, z1 = m1 == -INFINITY ? 0.0f : m1;  // what is subtracted (-inf less -inf would be no number)
    // Tile m, times 2^24: o[m][0], o[m][1] = dim 16g+2m of heads 2t, 2t+1, o[m][2], o[m][3] = 16 x dim 16g+2m+1, each with 8 sum(weight) too much:
    // that is `zero`, summed by the same instructions in the same order over codes of zero, so that the two carry the same bias of
    // the accumulation. It also is the denominator (static steps).
    float o[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    float den0 = 0.0f, den1 = 0.0f;  // DYN: this lane's shares of the denominators of heads 2t, 2t+1

    const uint32_t k_off = g * 64 + 16 * t;      // key g (and g + 8): 32 codes at dims 32t..32t+31
    const uint32_t v_off = (2 * t) * 64 + 8 * g;  // keys 2t, 2t+1, 2t+8, 2t+9: 16 codes at dims 16g..16g+15
    for (int key0 = x.r0 * DP_ROUND + first_key; key0 < kend; key0 += stride) {
      const int s = n_done % DP_SLOTS;
      bool late = !__all_sync(0xffffffffu, pq::mbar_look<POLL>(&full[warp][s], (n_done / DP_SLOTS) & 1));
      if (late) late = timed_out || n_done >= n_issued || __any_sync(0xffffffffu, !pq::mbar_look_for<POLL>(&full[warp][s], (n_done / DP_SLOTS) & 1, p.wait_clocks));
      if (late) {
        timed_out = true;  // nothing more is requested; the pieces run out without work
        is_ok = false;
        break;
      }
      const uint8_t* const slot = stage + s * SLOT;
      float rs[2][2];  // DYN: 2^-PQ_UP / step of the values of keys g, g + 8
      float c[2][4];  // scores: [0], [1] = key g x heads 2t, 2t+1; [2], [3] = key g + 8 x the same heads
      if (DYN) {
        // lane j turns the steps of key j into what all lanes need, once: (step of the key, log2 and reciprocal of the step of the value); a key past the
        // end has the score -inf
        const float* st = reinterpret_cast<const float*>(slot + DP_BLOCK * 128) + lane;
        const float k_step = st[0], v_step = st[DP_BLOCK];
        const bool dead = key0 + lane >= kend;
        sm_step[warp][lane] = dead ? make_float4(0.0f, -INFINITY, 0.0f, 0.0f) : make_float4(k_step, pq::lg2_approx(v_step), pq::rcp_approx(v_step) * pq::PQ_DOWN, 0.0f);
        __syncwarp();
      }
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const uint8_t* kb = slot + v * 1024 + k_off;
        const uint4 kc0 = *reinterpret_cast<const uint4*>(kb), kc1 = *reinterpret_cast<const uint4*>(kb + 8 * 64);
        float ca[4] = {0.0f, 0.0f, 0.0f, 0.0f}, cb[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const uint32_t wl[4] = {kc0.x, kc0.y, kc0.z, kc0.w}, wh[4] = {kc1.x, kc1.y, kc1.z, kc1.w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t wl8 = wl[w] >> 8, wh8 = wh[w] >> 8;
          mma_f16(ca, codes_lo(wl[w]), codes_lo(wh[w]), codes_hi(wl[w]), codes_hi(wh[w]), qb[2 * w][0], qb[2 * w][1]);
          mma_f16(cb, codes_lo(wl8), codes_lo(wh8), codes_hi(wl8), codes_hi(wh8), qb[2 * w + 1][0], qb[2 * w + 1][1]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) c[v][i] = fmaf(ca[i] + cb[i], i & 1 ? f_hi : f_lo, i & 1 ? n_hi : n_lo);
        if (DYN) {
          const float4 a = sm_step[warp][16 * v + g], b = sm_step[warp][16 * v + 8 + g];
          c[v][0] = fmaf(c[v][0], a.x, a.y), c[v][1] = fmaf(c[v][1], a.x, a.y);
          c[v][2] = fmaf(c[v][2], b.x, b.y), c[v][3] = fmaf(c[v][3], b.x, b.y);
          rs[v][0] = a.z, rs[v][1] = b.z;
        }
      }
      if (!DYN && key0 + DP_BLOCK > kend) {  // the last block of a sequence
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          if (key0 + 16 * v + g >= kend) c[v][0] = c[v][1] = -INFINITY;
          if (key0 + 16 * v + 8 + g >= kend) c[v][2] = c[v][3] = -INFINITY;
        }
      }
      // maxima of heads 2t, 2t+1 over this lane's keys; a reference moves only when one exceeds it by more than the headroom (the first
      // block of a warp always takes this path)
      float x0 = max3(c[0][0], c[0][2], fmaxf(c[1][0], c[1][2])), x1 = max3(c[0][1], c[0][3], fmaxf(c[1][1], c[1][3]));
      if (__any_sync(0xffffffffu, x0 > m0 + DP_HEADROOM || x1 > m1 + DP_HEADROOM)) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, d));
          x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, d));
        }
        const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
        const float d_lo = n0 == -INFINITY ? 0.0f : m0 - n0, d_hi = n1 == -INFINITY ? 0.0f : m1 - n1;
        const float a_lo = pq::ex2_approx(d_lo), a_hi = pq::ex2_approx(d_hi);
        m0 = n0, m1 = n1;
        zero[0] *= a_lo, zero[1] *= a_hi, zero[2] *= a_lo, zero[3] *= a_hi;
        if (DYN) den0 = pq::at_reference(den0, d_lo), den1 = pq::at_reference(den1, d_hi);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i][0] *= a_lo, o[i][1] *= a_hi, o[i][2] *= a_lo, o[i][3] *= a_hi;
        z0 = m0 == -INFINITY ? 0.0f : m0, z1 = m1 == -INFINITY ? 0.0f : m1;
      }
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const uint8_t* vb = slot + DP_BLOCK * 64 + v * 1024 + v_off;
        const uint2 vc0 = *reinterpret_cast<const uint2*>(vb), vc1 = *reinterpret_cast<const uint2*>(vb + 64);
        const uint2 vc2 = *reinterpret_cast<const uint2*>(vb + 8 * 64), vc3 = *reinterpret_cast<const uint2*>(vb + 9 * 64);
        const float zu0 = DYN ? z0 - pq::PQ_UP : z0, zu1 = DYN ? z1 - pq::PQ_UP : z1, down = DYN ? pq::PQ_DOWN : 1.0f;
        const float w0 = pq::ex2_approx(c[v][0] - zu0), w1 = pq::ex2_approx(c[v][1] - zu1);
        const float w2 = pq::ex2_approx(c[v][2] - zu0), w3 = pq::ex2_approx(c[v][3] - zu1);
        // weights in fp16, transposed from (key, head pair) to the (key pair, head) layout of an MMA B operand
        const uint32_t pb0 = movmatrix_trans(pq::pack_f16(w0 * down, w1 * down)), pb1 = movmatrix_trans(pq::pack_f16(w2 * down, w3 * down));
        if (DYN) {
          den0 = fmaf(w0, rs[v][0], den0), den1 = fmaf(w1, rs[v][0], den1);
          den0 = fmaf(w2, rs[v][1], den0), den1 = fmaf(w3, rs[v][1], den1);
        }
        mma_f16(zero, codes_lo(0u), codes_hi(0u), codes_lo(0u), codes_hi(0u), pb0, pb1);
        // ---- O^T += V^T P^T. A merged word pairs the same four dims of two neighbouring keys; nibbles 1 and 3 (16 x) are the rows g + 8 of the tile.
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const uint32_t sel = (q4 & 1) ? 0x7632u : 0x5410u;
          const uint32_t ya = __byte_perm(q4 < 2 ? vc0.x : vc0.y, q4 < 2 ? vc1.x : vc1.y, sel);
          const uint32_t yb = __byte_perm(q4 < 2 ? vc2.x : vc2.y, q4 < 2 ? vc3.x : vc3.y, sel);
          const uint32_t ya8 = ya >> 8, yb8 = yb >> 8;
          mma_f16(o[2 * q4], codes_lo(ya), codes_hi(ya), codes_lo(yb), codes_hi(yb), pb0, pb1);
          mma_f16(o[2 * q4 + 1], codes_lo(ya8), codes_hi(ya8), codes_lo(yb8), codes_hi(yb8), pb0, pb1);
        }
      }
      ++n_done;
      __syncwarp();
      issue();
    }

    // ---- merge the warps of this CTA and the prefix into one partial, in value units. The next piece's first loads and the first prefix values are
    // requested ahead of the barrier.
    const Piece done = x;
    const int done_row = row, next_u = u + (x.r1 - x.r0);
    if (next_u < u1) {
      advance(x, next_u);
      request();
    }
    uint2 pv[4];
    const uint2* const pv_row = reinterpret_cast<const uint2*>(p.prefix_v + static_cast<int64_t>(done.h) * p.n_prefix * 128) + lane;
#pragma unroll
    for (int j = 0; j < 4; ++j) pv[j] = has_prefix && j < p.n_prefix ? pq::ld_dep(pv_row + j * 32) : make_uint2(0u, 0u);
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int head = 2 * t + hh;
      if (head < G) {
#pragma unroll
        for (int m = 0; m < 8; ++m)
          *reinterpret_cast<float2*>(sm_o + (warp * G + head) * DP_SO_STRIDE + 16 * m + 2 * g) = make_float2((o[m][hh] - zero[hh]) * 16777216.0f, (o[m][2 + hh] - zero[2 + hh]) * 1048576.0f);
      }
    }
    if (DYN) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        den0 += __shfl_xor_sync(0xffffffffu, den0, d);
        den1 += __shfl_xor_sync(0xffffffffu, den1, d);
      }
    } else {
      den0 = zero[0] * 2097152.0f, den1 = zero[1] * 2097152.0f;  // 2^24 / 8
    }
    if (g == 0) {
      if (2 * t < G) sm_ml[warp][2 * t][0] = m0, sm_ml[warp][2 * t][1] = den0;
      if (2 * t + 1 < G) sm_ml[warp][2 * t + 1][0] = m1, sm_ml[warp][2 * t + 1][1] = den1;
    }
    __syncthreads();
    // partial of this worker: slot 2w when the pair began with an earlier worker, 2w + 1 when it begins here and goes on
    const int64_t ws_slot = (2 * static_cast<int64_t>(worker) + (done.r0 == 0 ? 1 : 0)) * G;
    __nv_bfloat16* dst = p.out + (static_cast<int64_t>(done_row) * p.Hq + static_cast<int64_t>(done.h) * G) * 128;
    {
      // warp w takes the heads w, w + 4; a lane the head dims 4 lane .. 4 lane + 3
      const int n_pre = has_prefix ? p.n_prefix : 0;
      const int qpos = 16 * ((2 * lane) & 7) + 2 * (lane >> 2);  // dims 4 lane, +1 here, dims 4 lane + 2, +3 sixteen floats on
      for (int r = warp; r < G; r += DP_WARPS) {
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < DP_WARPS; ++w) m = fmaxf(m, sm_ml[w][r][0]);
        for (int j = 0; j < n_pre; ++j) m = fmaxf(m, sm_pre[r * p.n_prefix + j]);
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float l = 0.0f;
#pragma unroll
        for (int w = 0; w < DP_WARPS; ++w) {
          const float mw = sm_ml[w][r][0];
          const float e = mw == -INFINITY ? 0.0f : pq::ex2_approx(mw - m);
          const float* src = sm_o + (w * G + r) * DP_SO_STRIDE + qpos;
          const float2 lo = *reinterpret_cast<const float2*>(src), hi = *reinterpret_cast<const float2*>(src + 16);
          acc.x = fmaf(lo.x, e, acc.x), acc.y = fmaf(lo.y, e, acc.y), acc.z = fmaf(hi.x, e, acc.z), acc.w = fmaf(hi.y, e, acc.w);
          l = DYN ? l + pq::at_reference(sm_ml[w][r][1], mw == -INFINITY ? mw : mw - m) : fmaf(sm_ml[w][r][1], e, l);
        }
        acc.x *= value_unit, acc.y *= value_unit, acc.z *= value_unit, acc.w *= value_unit;
        auto add_prefix = [&](int j, const uint2& v) {
          const float e = pq::ex2_approx(sm_pre[r * p.n_prefix + j] - m);
          const float2 v01 = __half22float2(*reinterpret_cast<const __half2*>(&v.x)), v23 = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
          acc.x = fmaf(e, v01.x, acc.x), acc.y = fmaf(e, v01.y, acc.y), acc.z = fmaf(e, v23.x, acc.z), acc.w = fmaf(e, v23.y, acc.w);
          l += e;
        };
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < n_pre) add_prefix(j, pv[j]);
        for (int j = 4; j < n_pre; ++j) add_prefix(j, pq::ld_dep(pv_row + j * 32));
        if (csize > 1) {
          __syncwarp();  // the rows of this head are this warp's alone: all lanes have read them
          *reinterpret_cast<float4*>(cl_o + r * DP_SO_STRIDE + 4 * lane) = acc;
          if (lane == 0) cl_ml[r] = make_float2(m, l);
        } else if (whole) {
          store_out(dst + r * 128 + 4 * lane, acc, l > 0.0f ? 1.0f / l : 0.0f);
        } else {
          *reinterpret_cast<float4*>(p.ws_o + (ws_slot + r) * 128 + 4 * lane) = acc;
          if (lane == 0) *reinterpret_cast<float2*>(p.ws_ml + (ws_slot + r) * 2) = make_float2(m, l);
        }
      }
    }
    if (csize > 1) {
      // the threads of the cluster take the (head, four dims) items in turn and read the CTAs' partials through distributed shared memory
      pq::cluster_sync();
      for (int item = rank * DP_THREADS + threadIdx.x; item < G * 32; item += csize * DP_THREADS) {
        const int r = item >> 5, c4 = item & 31;
        const uint32_t o_addr = pq::smem_u32(cl_o + r * DP_SO_STRIDE + 4 * c4), ml_addr = pq::smem_u32(cl_ml + r);
        float m = -INFINITY, l = 0.0f;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        auto eight = [&](int sp0) {
          float4 v[8];
          float2 ml[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f), ml[k] = make_float2(-INFINITY, 0.0f);
            if (sp0 + k < csize) v[k] = ld_cluster_f4(map_cta(o_addr, sp0 + k)), ml[k] = ld_cluster_f2(map_cta(ml_addr, sp0 + k));
          }
          float mn = m;
#pragma unroll
          for (int k = 0; k < 8; ++k) mn = fmaxf(mn, ml[k].x);
          const float keep = m == -INFINITY ? 0.0f : pq::ex2_approx(m - mn);
          l = DYN ? pq::at_reference(l, m == -INFINITY ? m : m - mn) : l * keep;
          acc.x *= keep, acc.y *= keep, acc.z *= keep, acc.w *= keep, m = mn;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float w = ml[k].x == -INFINITY ? 0.0f : pq::ex2_approx(ml[k].x - m);
            acc.x = fmaf(v[k].x, w, acc.x), acc.y = fmaf(v[k].y, w, acc.y), acc.z = fmaf(v[k].z, w, acc.z), acc.w = fmaf(v[k].w, w, acc.w);
            l = DYN ? l + pq::at_reference(ml[k].y, ml[k].x == -INFINITY ? ml[k].x : ml[k].x - m) : fmaf(ml[k].y, w, l);
          }
        };
        eight(0);
        if (WIDE) eight(8);
        if (whole) {
          store_out(dst + r * 128 + 4 * c4, acc, l > 0.0f ? 1.0f / l : 0.0f);
        } else {
          *reinterpret_cast<float4*>(p.ws_o + (ws_slot + r) * 128 + 4 * c4) = acc;
          if (c4 == 0) *reinterpret_cast<float2*>(p.ws_ml + (ws_slot + r) * 2) = make_float2(m, l);
          __threadfence();
        }
      }
      pq::cluster_sync();  // the partials in shared memory have been read, those in the workspace written
    }
    if (!whole) {  // the pair's units are shared by several workers
      const int pair0 = u - done.r0;
      auto worker_of = [&](int unit) { return static_cast<int>(((static_cast<int64_t>(unit) + 1) * n_workers - 1) / U); };
      if (threadIdx.x == 0) sm_shared[n_shared & 1] = make_int4(done_row, done.h, worker_of(pair0), worker_of(pair0 + done.rounds - 1));
      ++n_shared;
    }
    u = next_u;
  }
  // ---- the last of the workers w0 .. w1 of a shared pair to come here merges their partials, in that order. The tickets of both pairs are
  // drawn together at the end: one trip, and the fence in front of it has little left to wait for.
  if (n_shared > 0 && rank == 0) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x < n_shared) {
      const int w0 = sm_shared[threadIdx.x].z, w1 = sm_shared[threadIdx.x].w;
      sm_last[threadIdx.x] = atomicAdd(p.tickets + PQ_PAGED_TICKET0 + w0, 1u) == static_cast<uint32_t>(w1 - w0);
    }
    __syncthreads();
    __threadfence();
    for (int i = 0; i < n_shared; ++i) {
      if (!sm_last[i]) continue;
      const int w0 = sm_shared[i].z, w1 = sm_shared[i].w;
      __nv_bfloat16* dst = p.out + (static_cast<int64_t>(sm_shared[i].x) * p.Hq + static_cast<int64_t>(sm_shared[i].y) * G) * 128;
      for (int r = warp; r < G; r += DP_WARPS) {
        float m = -INFINITY, l = 0.0f;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int base = w0; base <= w1; base += 32) {  // a lane per partial for the weights, then the partials in turn
          const int n = min(32, w1 - base + 1);
          const int64_t mine = 2 * static_cast<int64_t>(base + lane) + (base + lane == w0 ? 1 : 0);
          const float2 ml = lane < n ? __ldcg(reinterpret_cast<const float2*>(p.ws_ml) + mine * G + r) : make_float2(-INFINITY, 0.0f);
          float4 ahead[8];  // the first partials are on their way while the weights are formed
          auto load = [&](int k) {
            const int64_t slot = 2 * static_cast<int64_t>(base + k) + (base + k == w0 ? 1 : 0);
            return __ldcg(reinterpret_cast<const float4*>(p.ws_o) + (slot * G + r) * 32 + lane);
          };
#pragma unroll
          for (int k = 0; k < 8; ++k) ahead[k] = k < n ? load(k) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          float mc = ml.x;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) mc = fmaxf(mc, __shfl_xor_sync(0xffffffffu, mc, d));
          const float mn = fmaxf(m, mc), keep = m == -INFINITY ? 0.0f : pq::ex2_approx(m - mn);
          const float w = ml.x == -INFINITY ? 0.0f : pq::ex2_approx(ml.x - mn);
          float lw = DYN ? pq::at_reference(ml.y, ml.x == -INFINITY ? ml.x : ml.x - mn) : ml.y * w;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) lw += __shfl_xor_sync(0xffffffffu, lw, d);
          l = (DYN ? pq::at_reference(l, m == -INFINITY ? m : m - mn) : l * keep) + lw;
          m = mn;
          acc.x *= keep, acc.y *= keep, acc.z *= keep, acc.w *= keep;
          auto add = [&](const float4& v, int k) {
            const float wk = __shfl_sync(0xffffffffu, w, k);
            acc.x = fmaf(v.x, wk, acc.x), acc.y = fmaf(v.y, wk, acc.y), acc.z = fmaf(v.z, wk, acc.z), acc.w = fmaf(v.w, wk, acc.w);
          };
#pragma unroll
          for (int k = 0; k < 8; ++k) add(ahead[k], k);  // (those past n are zeros)
#pragma unroll 4
          for (int k = 8; k < n; ++k) add(load(k), k);
        }
        store_out(dst + r * 128 + 4 * lane, acc, l > 0.0f ? 1.0f / l : 0.0f);
      }
      if (threadIdx.x == 0) p.tickets[PQ_PAGED_TICKET0 + w0] = 0;
    }
  }
  // every copy that was started has landed before the shared memory is given back (after a wait that ran out some are still on their way)
  if (lane == 0) {
    for (int n = n_done; n < n_issued; ++n) pq::mbar_wait(&full[warp][n % DP_SLOTS], (n / DP_SLOTS) & 1);
    if (timed_out) pq::report(p.status, PQ_ERR_TIMEOUT);
  }
  __syncwarp();
  leave();
}

constexpr int DP_CTAS_PER_SM = 4;

void (*kernel_of(bool dyn, int csize, bool poll))(const PagedAttnParams) {
  if (poll) return dyn ? paged_decode_kernel<true, true, true> : paged_decode_kernel<false, true, true>;  // (any cluster size)
  if (csize > 8) return dyn ? paged_decode_kernel<true, true, false> : paged_decode_kernel<false, true, false>;
  return dyn ? paged_decode_kernel<true, false, false> : paged_decode_kernel<false, false, false>;
}

int most_ctas(const pq_ctx* ctx) { return DP_CTAS_PER_SM * ctx->sm_count; }

// Clusters of csize CTAs that are resident at once: fewer than the CTAs alone would be, since a cluster stays inside a group of SMs. Asked once per
// device, kernel, cluster size and size of the shared memory in whole KB: the answer, and with it how the work is split, follows from the call alone.
int resident_workers(const pq_ctx* ctx, bool dyn, int csize, size_t smem) {
  static std::atomic<uint16_t> known[64][2][5][DP_MAX_KB + 1] = {};  // one more than the answer
  const int ci = csize == 16 ? 4 : csize == 8 ? 3 : csize == 4 ? 2 : csize == 2 ? 1 : 0;
  std::atomic<uint16_t>& slot = known[ctx->device][dyn][ci][smem_kb(smem)];
  int n = slot.load(std::memory_order_relaxed);
  if (n > 0) return n - 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(most_ctas(ctx) / csize * csize);
  cfg.blockDim = dim3(DP_THREADS);
  cfg.dynamicSmemBytes = smem_kb(smem) * 1024;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = csize, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, kernel_of(dyn, csize, false), &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();
    n = csize > 8 ? 0 : ctx->sm_count / csize;  // (clusters of more than eight need not fit at all)
  }
  if (n > most_ctas(ctx) / csize) n = most_ctas(ctx) / csize;
  slot.store(static_cast<uint16_t>(n + 1), std::memory_order_relaxed);
  return n;
}

}  // namespace

size_t pq_paged_decode_ws_bytes(const pq_ctx* ctx, const pq_kv4_paged* c) {
  return static_cast<size_t>(2) * most_ctas(ctx) * (c->Hq / c->Hkv) * (128 + 2) * sizeof(float);
}

pq_status pq_paged_decode_launch(pq_ctx* ctx, const pq_kv4_paged* c, PagedAttnParams p, int64_t max_len, void* ws, cudaStream_t st) {
  const bool dyn = p.steps != nullptr, poll = p.wait_clocks < PQ_SUSPENDED_CLOCKS;
  // the largest there is, once per device and kernel
  static std::atomic<bool> attr_set[64][2] = {};
  if (ctx->device < 0 || ctx->device >= 64) return PQ_ERR_UNSUPPORTED;
  if (!attr_set[ctx->device][dyn].load(std::memory_order_relaxed)) {
    const int most = static_cast<int>(DP_MAX_KB * 1024);
    for (auto* const kern : {kernel_of(dyn, 1, false), kernel_of(dyn, 16, false), kernel_of(dyn, 16, true)}) {
      if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess ||
          (kern != kernel_of(dyn, 1, false) && cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)) {
        cudaGetLastError();
        return PQ_ERR_CUDA;
      }
    }
    attr_set[ctx->device][dyn].store(true, std::memory_order_relaxed);
  }
  const int64_t pairs = static_cast<int64_t>(p.B) * p.Hkv, most = most_ctas(ctx);
  const int64_t rounds = (max_len + DP_ROUND - 1) / DP_ROUND;
  // Few pairs share the chip: a cluster of CTAs to a pair or stretch keeps the partials that meet in the workspace few.
  int64_t csize = most / pairs;
  csize = csize >= 8 ? 8 : csize >= 4 ? 4 : csize >= 2 ? 2 : 1;
  // One worker per pair or equal stretches, by an estimate for sequences of max_len tokens: a round of a CTA takes 0.75 us and 0.45 us for every CTA on its
  // SM, the call 6 us besides; equal stretches fill the SMs (2.1 us a round) but cost 20 us (prefix sums, a second piece, the merge through the
  // workspace). us, one worker per pair / equal stretches, 8 KV heads: 1 sequence x 6000 tokens 12.3 / 21.2, x 12000 19.0 / 25.2, x 20000 27.6 / 27.5,
  // x 60000 75 / 37; 4 x 12000 23.7 / 34.1, x 20000 34.6 / 40.8, x 35000 53.6 / 53.0, x 60000 86 / 75; 16 x 8000 44.8 / 54.0; 30 x 3000 35.6 / 44.6;
  // 60 x 3000 61.5 / 64.8; 5 ragged to 50000 69 / 58, 48 ragged to 6000 70 / 56.
  const size_t smem_one = dynamic_smem(dyn, p.G, p.n_prefix, 0);
  int64_t one = csize;
  while (one > 1 && one > rounds) one >>= 1;
  // us with clusters of 8 / 16, 1 sequence of 2100 tokens (17 rounds) 8.3 / 8.9, 4000 10.7 / 9.7, 6000 12.3 / 11.1, 12000 18.9 / 15.0, 20000 27.1 / 20.0.
  if (one == 8 && rounds >= 24 && pairs * 16 <= ctx->sm_count && pairs <= resident_workers(ctx, dyn, 16, smem_one)) one = 16;
  bool direct = pairs <= resident_workers(ctx, dyn, static_cast<int>(one), smem_one);
  if (direct) {
    const double sms = ctx->sm_count, per_sm = pairs * one > ctx->sm_count ? pairs * one / sms : 1.0;
    const double t_one = static_cast<double>((rounds + one - 1) / one) * (0.75 + 0.45 * per_sm) + 6.0;
    const double t_equal = 20.0 + 2.1 * static_cast<double>(pairs * rounds) / (DP_CTAS_PER_SM * sms);
    direct = t_one <= t_equal;
  }
  if (direct) csize = one;
  const size_t smem = dynamic_smem(dyn, p.G, p.n_prefix, direct ? 0 : p.B);
  p.csize = static_cast<int32_t>(csize);
  p.workers = direct ? 0 : resident_workers(ctx, dyn, p.csize, smem);
  if (p.workers > PQ_PAGED_MAX_WORKERS) p.workers = PQ_PAGED_MAX_WORKERS;
  p.ws_o = static_cast<float*>(ws);
  p.ws_ml = p.ws_o + static_cast<size_t>(2) * p.workers * p.G * 128;
  const int64_t grid = (direct ? pairs : p.workers) * csize;
  return pq_launch_cluster_pdl(kernel_of(dyn, p.csize, poll), dim3(static_cast<unsigned>(grid)), DP_THREADS, smem, p.csize, st, p);
}
