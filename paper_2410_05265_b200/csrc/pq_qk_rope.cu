// Norm of every query and key head and rotary embedding with positions of one to three axes in one pass (pq_qk_norm_rope), the same with the
// quantize-on-write into the paged KV4 cache (pq_qk_norm_rope_kv4_paged_append), and the read-back of cached vectors (pq_kv4_paged_read).
//
// Bound by HBM: a head is read once and written once (256 bytes each way, 64 bytes as codes). Sixteen lanes take a head, a warp two heads of a
// kind; a lane holds dims 4l .. 4l+3 and 64+4l .. 64+4l+3, so both halves of a rotary pair and the index bits 0, 1 and 6 of the
// Hadamard transform are inside the lane, its bits 2 to 5 four shuffles away. Angles are reduced in 64 bits as fractions of a turn (a position
// of 10^5 leaves an fp32 angle three digits).
// The key heads of the append are computed in 64 bits up to the quotient that is rounded to a code: with fp32 about one code in a million depends
// on the order of a sum, so that a prompt cached in chunks would differ from the same prompt cached at once. They are a small share of
// the heads.
#include <math.h>

#include <type_traits>

#include "pq_paged.cuh"

namespace {

constexpr int QR_THREADS = 128;
constexpr int QR_WARPS = QR_THREADS / 32;
constexpr int QR_AHEAD = 4;  // units (two heads each) a warp requests together

struct QkParams {
  const __nv_bfloat16* x;
  int64_t ld;
  const __nv_bfloat16* gq;
  const __nv_bfloat16* gk;
  const int32_t* pos;
  int64_t ld_pos;
  __nv_bfloat16* y;  // append: the query heads only
  int64_t ldy;
  int64_t N;
  float eps;
  int32_t Hq, Hk, rotate;
  int32_t end0, end1;  // frequencies below end0 follow axis 0, below end1 axis 1, the others axis 2
  // append
  const int64_t* slot;
  uint8_t* codes;
  float* steps;
  const float* s_k;
  const float* s_v;
  int32_t* status;
  int64_t n_slots;
  int32_t page_log2;
  double turns[64];  // theta^(-2i/128) / (2 pi)
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void unpack8(const uint2& a, const uint2& b, float (&f)[8]) {
  f[0] = bf16_lo(a.x), f[1] = bf16_hi(a.x), f[2] = bf16_lo(a.y), f[3] = bf16_hi(a.y);
  f[4] = bf16_lo(b.x), f[5] = bf16_hi(b.x), f[6] = bf16_lo(b.y), f[7] = bf16_hi(b.y);
}

template <typename T>
__device__ __forceinline__ T half_warp_sum(T v) {
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
template <typename T>
__device__ __forceinline__ T half_warp_max(T v) {
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) {
    const T o = __shfl_xor_sync(0xffffffffu, v, m);
    v = o > v ? o : v;
  }
  return v;
}

__device__ __forceinline__ float inv_sqrt(float x) { return 1.0f / sqrtf(x); }
__device__ __forceinline__ double inv_sqrt(double x) { return 1.0 / sqrt(x); }

// norm, gain, rotary position and, on demand, the Hadamard transform of one head, in T
template <typename T>
__device__ __forceinline__ void transform(T (&f)[8], bool norm, T eps, const float (&g)[8], const T* cs, const T* sn, int l, bool rotate) {
  if (norm) {
    T ss = T(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma(f[e], f[e], ss);
    const T r = inv_sqrt(half_warp_sum(ss) * T(0.0078125) + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = f[e] * r * T(g[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const T c = cs[4 * l + e], s = sn[4 * l + e], a = f[e], b = f[4 + e];
    f[e] = fma(a, c, -(b * s));
    f[4 + e] = fma(b, c, a * s);
  }
  if (rotate) {
#pragma unroll
    for (int m = 1; m < 8; m <<= 1) {  // index bits 0, 1 and 6
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e & m) continue;
        const T a = f[e], b = f[e | m];
        f[e] = a + b, f[e | m] = a - b;
      }
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) {  // index bits 2 to 5: the upper partner holds the difference
      const T sg = l & m ? T(-1) : T(1);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = fma(f[e], sg, __shfl_xor_sync(0xffffffffu, f[e], m));
    }
    const T norm128 = T(0.08838834764831844055);  // 1 / sqrt(128)
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= norm128;
  }
}

__device__ __forceinline__ uint32_t clamp_code(float q) { return static_cast<uint32_t>(max(-8, min(7, __float2int_rn(q)))) & 0xFu; }

template <bool APPEND>
__global__ void __launch_bounds__(QR_THREADS) qk_norm_rope_kernel(const QkParams p) {
  __shared__ float cs[64], sn[64];
  __shared__ double csk[APPEND ? 64 : 1], snk[APPEND ? 64 : 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
  const int uq = (p.Hq + 1) >> 1, uk = (p.Hk + 1) >> 1;
  const int n_units = uq + (APPEND ? 2 : 1) * uk;  // keys, then (append) values, then queries: the longest first
  pq::pdl_wait();
  if (!APPEND) pq::pdl_trigger();  // a writer of cache rows does not (see pq_launch_pdl)
  const bool norm = p.gq != nullptr;
  float gq[8], gk[8];
  {
    uint2 a = make_uint2(0u, 0u), b = a, c = a, d = a;
    if (norm) {
      a = pq::ld_dep(reinterpret_cast<const uint2*>(p.gq) + l), b = pq::ld_dep(reinterpret_cast<const uint2*>(p.gq) + 16 + l);
      c = pq::ld_dep(reinterpret_cast<const uint2*>(p.gk) + l), d = pq::ld_dep(reinterpret_cast<const uint2*>(p.gk) + 16 + l);
    }
    unpack8(a, b, gq);
    unpack8(c, d, gk);
  }
  for (int64_t t = blockIdx.x; t < p.N; t += gridDim.x) {
    int64_t slot = 0;
    if (APPEND) {
      slot = pq::ld_dep(p.slot + t);
      if (slot < 0) continue;
      if (slot >= p.n_slots) {
        if (threadIdx.x == 0) pq::report(p.status, PQ_ERR_SHAPE);
        continue;
      }
    }
    __syncthreads();  // the angles of the token before have been used
    if (threadIdx.x < 64) {
      const int i = threadIdx.x;
      const int axis = i < p.end0 ? 0 : i < p.end1 ? 1 : 2;
      const double turn = static_cast<double>(pq::ld_dep(p.pos + axis * p.ld_pos + t)) * p.turns[i];
      const double frac = turn - rint(turn);  // in [-1/2, 1/2], exact
      if (APPEND) {
        double s, c;
        sincospi(2.0 * frac, &s, &c);
        csk[APPEND ? i : 0] = c, snk[APPEND ? i : 0] = s;
        cs[i] = static_cast<float>(c), sn[i] = static_cast<float>(s);
      } else {
        float s, c;
        sincospif(static_cast<float>(2.0 * frac), &s, &c);
        cs[i] = c, sn[i] = s;
      }
    }
    __syncthreads();
    const uint8_t* xr = reinterpret_cast<const uint8_t*>(p.x + t * p.ld);
    for (int first = warp; first < n_units; first += QR_AHEAD * QR_WARPS) {
      uint2 wa[QR_AHEAD], wb[QR_AHEAD];
      int head[QR_AHEAD];
#pragma unroll
      for (int a = 0; a < QR_AHEAD; ++a) {
        const int u = first + a * QR_WARPS;
        if (u >= n_units) break;
        // kind 0: keys, 1: values, 2: queries; the second half of an odd last pair repeats its head and stores nothing
        const int kind = u < uk ? 0 : (APPEND && u < 2 * uk) ? 1 : 2;
        const int in_kind = 2 * (kind == 0 ? u : kind == 1 ? u - uk : u - (APPEND ? 2 : 1) * uk) + half;
        const int count = kind == 2 ? p.Hq : p.Hk;
        const int h = min(in_kind, count - 1);
        head[a] = in_kind < count ? h : -1 - h;
        const int col = kind == 2 ? h : kind == 0 ? p.Hq + h : p.Hq + p.Hk + h;
        const uint2* src = reinterpret_cast<const uint2*>(xr + static_cast<int64_t>(col) * 256);
        wa[a] = pq::ld_dep(src + l), wb[a] = pq::ld_dep(src + 16 + l);
      }
#pragma unroll
      for (int a = 0; a < QR_AHEAD; ++a) {
        const int u = first + a * QR_WARPS;
        if (u >= n_units) break;
        const int kind = u < uk ? 0 : (APPEND && u < 2 * uk) ? 1 : 2;
        const bool mine = head[a] >= 0;
        const int h = mine ? head[a] : -1 - head[a];
        float f[8];
        unpack8(wa[a], wb[a], f);
        if (!APPEND || kind == 2) {
          const bool is_q = kind == 2;
          float g[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = is_q ? gq[e] : gk[e];
          transform<float>(f, norm, p.eps, g, cs, sn, l, p.rotate != 0);
          if (mine) {
            uint2* dst = reinterpret_cast<uint2*>(p.y + t * p.ldy + static_cast<int64_t>(is_q ? h : p.Hq + h) * 128);
            dst[l] = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
            dst[16 + l] = make_uint2(pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
          }
          continue;
        }
        uint32_t code[8];
        float s;
        if (kind == 0) {
          double y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = static_cast<double>(f[e]);
          transform<double>(y, norm, static_cast<double>(p.eps), gk, csk, snk, l, p.rotate != 0);
          if (p.steps) {
            double mx = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmax(mx, fabs(y[e]));
            mx = half_warp_max(mx);
            s = mx < 0x1p-57 ? 1.0f : __double2float_rn(mx / 7.0);
          } else {
            s = pq::ld_dep(p.s_k + h);
          }
          // (1 / s in 64 bits leaves the quotient exact to 2^-52: rounded to fp32 it is the exact quotient's fp32 value, ties of representable ones included)
          const double inv = 1.0 / static_cast<double>(s);
#pragma unroll
          for (int e = 0; e < 8; ++e) code[e] = clamp_code(__double2float_rn(y[e] * inv));
        } else {
          if (p.steps) {
            float mx = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf(f[e]));
            mx = half_warp_max(mx);
            s = mx < 0x1p-57f ? 1.0f : __fdiv_rn(mx, 7.0f);
          } else {
            s = pq::ld_dep(p.s_v + h);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) code[e] = clamp_code(__fdiv_rn(f[e], s));
        }
        if (mine) {
          const int64_t row = ((slot >> p.page_log2) * p.Hk + h) * 2 + kind;  // (page, head, keys or values)
          const int64_t vec = (row << p.page_log2) + (slot & ((1 << p.page_log2) - 1));
          uint16_t* dst = reinterpret_cast<uint16_t*>(p.codes + vec * 64);
          dst[l] = static_cast<uint16_t>(code[0] | code[1] << 4 | code[2] << 8 | code[3] << 12);
          dst[16 + l] = static_cast<uint16_t>(code[4] | code[5] << 4 | code[6] << 8 | code[7] << 12);
          if (p.steps && l == 0) p.steps[vec] = s;
        }
      }
    }
  }
}

// Eight codes of a cached vector to a thread: 4 bytes in, 16 bytes out.
constexpr int RD_THREADS = 256;
__global__ void __launch_bounds__(RD_THREADS)
    kv4_paged_read_kernel(const uint8_t* codes, const float* steps, const float* s_k, const float* s_v, const int64_t* slots, int64_t N, int Hkv,
                          int page_log2, int64_t n_slots, __nv_bfloat16* out, int32_t* status) {
  pq::pdl_wait();
  pq::pdl_trigger();
  const int64_t n_units = N * Hkv * 32;  // (row, keys or values, head, group of eight dims)
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * RD_THREADS + threadIdx.x; u < n_units; u += static_cast<int64_t>(gridDim.x) * RD_THREADS) {
    const int part = static_cast<int>(u & 15);
    const int64_t vec_out = u >> 4;
    const int h = static_cast<int>(vec_out % Hkv), which = static_cast<int>((vec_out / Hkv) & 1);
    const int64_t slot = pq::ld_dep(slots + vec_out / (2 * Hkv));
    if (slot < 0) continue;
    if (slot >= n_slots) {
      pq::report(status, PQ_ERR_SHAPE);
      continue;
    }
    const int64_t vec = ((((slot >> page_log2) * Hkv + h) * 2 + which) << page_log2) + (slot & ((1 << page_log2) - 1));
    const uint32_t w = pq::ld_dep(reinterpret_cast<const uint32_t*>(codes + vec * 64) + part);
    const float s = steps ? pq::ld_dep(steps + vec) : pq::ld_dep((which ? s_v : s_k) + h);
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int lo = static_cast<int>(w << (28 - 8 * i)) >> 28, hi = static_cast<int>(w << (24 - 8 * i)) >> 28;
      o[i] = pack_bf16(static_cast<float>(lo) * s, static_cast<float>(hi) * s);
    }
    *reinterpret_cast<uint4*>(out + vec_out * 128 + part * 8) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// Checks what both entry points take and fills the parameters that follow from it.
pq_status rope_params(QkParams& p, const void* x, int64_t N, int32_t Hq, int32_t Hk, int64_t n_cols, int64_t ld, const void* gq, const void* gk,
                      float eps, const int32_t* pos, int32_t n_axes, int64_t ld_pos, const int32_t* sections, double theta, int32_t rotate, void* y,
                      int64_t ldy, int64_t y_cols) {
  if (!x || !y || !pos || Hq < 0 || Hk < 0 || Hq + static_cast<int64_t>(Hk) <= 0 || (gq != nullptr) != (gk != nullptr)) return PQ_ERR_INVALID_ARG;
  if (!(theta > 0.0) || !isfinite(theta) || !(eps >= 0.0f)) return PQ_ERR_INVALID_ARG;
  if (n_axes < 1 || n_axes > 3 || (n_axes > 1 && (!sections || ld_pos < N))) return PQ_ERR_INVALID_ARG;
  if (ld < n_cols || ldy < y_cols || (y == x && ldy != ld)) return PQ_ERR_INVALID_ARG;
  if (Hq > 65536 || Hk > 65536) return PQ_ERR_SHAPE;
  int32_t sec[3] = {64, 0, 0};
  if (sections) {
    int64_t sum = 0;
    for (int a = 0; a < 3; ++a) {
      sec[a] = a < n_axes ? sections[a] : 0;
      if (sec[a] < 0) return PQ_ERR_INVALID_ARG;
      sum += sec[a];
    }
    if (sum != 64) return PQ_ERR_SHAPE;
  }
  if (pq_misaligned16(x) || pq_misaligned16(y) || pq_misaligned16(gq) || pq_misaligned16(gk) || ld % 8 != 0 || ldy % 8 != 0) return PQ_ERR_ALIGN;
  p.x = static_cast<const __nv_bfloat16*>(x), p.ld = ld;
  p.gq = static_cast<const __nv_bfloat16*>(gq), p.gk = static_cast<const __nv_bfloat16*>(gk);
  p.pos = pos, p.ld_pos = ld_pos;
  p.y = static_cast<__nv_bfloat16*>(y), p.ldy = ldy;
  p.N = N, p.eps = eps, p.Hq = Hq, p.Hk = Hk, p.rotate = rotate;
  p.end0 = sec[0], p.end1 = sec[0] + sec[1];
  for (int i = 0; i < 64; ++i) p.turns[i] = pow(theta, -2.0 * i / 128.0) / 6.283185307179586476925286766559;
  return PQ_OK;
}

}  // namespace

extern "C" pq_status pq_qk_norm_rope(pq_ctx* ctx, const void* x, int64_t N, int32_t Hq, int32_t Hk, int32_t D, int64_t ld, const void* gq,
                                     const void* gk, float eps, const int32_t* pos, int32_t n_axes, int64_t ld_pos, const int32_t* sections,
                                     double theta, int32_t rotate, void* y, int64_t ldy, void* stream) {
  if (!ctx || N < 0) return PQ_ERR_INVALID_ARG;
  if (D != 128) return PQ_ERR_SHAPE;
  if (N == 0) return PQ_OK;
  QkParams p{};
  const int64_t cols = (static_cast<int64_t>(Hq) + Hk) * 128;
  const pq_status st = rope_params(p, x, N, Hq, Hk, cols, ld, gq, gk, eps, pos, n_axes, ld_pos, sections, theta, rotate, y, ldy, cols);
  if (st != PQ_OK) return st;
  const int64_t grid = N < 16LL * ctx->sm_count ? N : 16LL * ctx->sm_count;
  return pq_launch_pdl(qk_norm_rope_kernel<false>, dim3(static_cast<unsigned>(grid)), QR_THREADS, 0, static_cast<cudaStream_t>(stream), p);
}

extern "C" pq_status pq_qk_norm_rope_kv4_paged_append(pq_ctx* ctx, const pq_kv4_paged* c, const void* qkv, int64_t N, int64_t ld, const void* gq,
                                                      const void* gk, float eps, const int32_t* pos, int32_t n_axes, int64_t ld_pos,
                                                      const int32_t* sections, double theta, int32_t rotate, const int64_t* slot, void* q_out,
                                                      int64_t ldq, void* stream) {
  if (!ctx || N < 0) return PQ_ERR_INVALID_ARG;
  const pq_status cs = pq_check_paged(c);
  if (cs != PQ_OK) return cs;
  if (N == 0) return PQ_OK;
  if (!slot) return PQ_ERR_INVALID_ARG;
  QkParams p{};
  const pq_status st = rope_params(p, qkv, N, c->Hq, c->Hkv, (c->Hq + 2ll * c->Hkv) * 128, ld, gq, gk, eps, pos, n_axes, ld_pos, sections, theta, rotate,
                                   q_out, ldq, static_cast<int64_t>(c->Hq) * 128);
  if (st != PQ_OK) return st;
  p.slot = slot, p.codes = c->codes, p.steps = c->steps, p.s_k = c->s_k, p.s_v = c->s_v, p.status = ctx->d_status;
  p.page_log2 = pq_page_log2(c->pages.page);
  p.n_slots = static_cast<int64_t>(c->pages.n_pages) << p.page_log2;
  const int64_t grid = N < 16LL * ctx->sm_count ? N : 16LL * ctx->sm_count;
  return pq_launch_pdl(qk_norm_rope_kernel<true>, dim3(static_cast<unsigned>(grid)), QR_THREADS, 0, static_cast<cudaStream_t>(stream), p);
}

extern "C" pq_status pq_kv4_paged_read(pq_ctx* ctx, const pq_kv4_paged* c, const int64_t* slot, int64_t N, void* out, void* stream) {
  if (!ctx || N < 0) return PQ_ERR_INVALID_ARG;
  const pq_status cs = pq_check_paged(c);
  if (cs != PQ_OK) return cs;
  if (N == 0) return PQ_OK;
  if (!slot || !out) return PQ_ERR_INVALID_ARG;
  if (pq_misaligned16(out)) return PQ_ERR_ALIGN;
  const int page_log2 = pq_page_log2(c->pages.page);
  int64_t grid = (N * c->Hkv * 32 + RD_THREADS - 1) / RD_THREADS;
  if (grid > 8LL * ctx->sm_count) grid = 8LL * ctx->sm_count;
  return pq_launch_pdl(kv4_paged_read_kernel, dim3(static_cast<unsigned>(grid)), RD_THREADS, 0, static_cast<cudaStream_t>(stream), c->codes, c->steps, c->s_k,
                       c->s_v, slot, N, c->Hkv, page_log2, static_cast<int64_t>(c->pages.n_pages) << page_log2, static_cast<__nv_bfloat16*>(out),
                       ctx->d_status);
}
