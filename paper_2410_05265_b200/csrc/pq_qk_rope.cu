// Norm of every query and key head and rotary embedding with positions of one to three axes in one pass (pq_qk_norm_rope), the same with the
// quantize-on-write into the paged KV4 cache (pq_qk_norm_rope_kv4_paged_append), and the read-back of cached vectors (pq_kv4_paged_read).
//
// Bound by HBM: a head is read once and written once (256 bytes each way, 64 bytes as codes). L lanes take a head, a warp 32 / L heads of a block of tokens; a
// lane holds C = 64 / L dims of each half, t C .. t C + C - 1 and 64 + t C ..: both halves of a rotary pair and the lower stages of the Hadamard
// transform are inside the lane, log2 L stages are shuffles, and the fp32 arithmetic runs on packed pairs. L = 4 for many tokens (with L = 16 the
// kernel is bound by instruction issue: 4099 x 72 heads with R3 48.5 us, against 35.4 = 0.65 of the measured copy rate; L = 8 with a token's factors kept in
// registers and a warp's heads in a row, which takes half the load off the shared-memory pipe, 40.3, with two heads requested ahead 43.0), L = 16 for few, where
// the chain of one head is the time. Angles are reduced in 64 bits as fractions of a turn (a position of 10^5 leaves an fp32 angle three digits).
// The append of 6001 tokens x 80 heads with R3 and own steps takes 73 us.
// The key heads of the append are computed in 64 bits up to the quotient that is rounded to a code: with fp32 about one code in a million depends
// on the order of a sum, so that a prompt cached in chunks would differ from the same prompt cached at once. They are a small share of
// the heads.
#include <math.h>

#include "pq_paged.cuh"

namespace {

constexpr int QR_THREADS = 128;
constexpr int QR_WARPS = QR_THREADS / 32;
constexpr int QR_TOKENS = 4;  // most tokens of a CTA
static_assert(QR_TOKENS == 4, "the search for a head's token");
constexpr int QR_ROW = 80;    // 64 angles, every sixteen followed by four words: four lanes that read sixteen each meet in no bank

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
  int32_t tokens;    // of a CTA
  double turns[64];  // theta^(-2i/128) / (2 pi)
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ int angle_at(int i) { return i + ((i >> 4) << 2); }
__device__ __forceinline__ float2 unpack_bf16(uint32_t w) { return make_float2(bf16_lo(w), bf16_hi(w)); }

// The elements of a lane: C dims of the lower half as pairs in a, of the upper half in b.
template <int C>
struct Lane {
  float2 a[C / 2], b[C / 2];
};

__device__ __forceinline__ void butterfly(float2& x, float2& y) {
  const float2 u = x;
  x = __fadd2_rn(u, y), y = __ffma2_rn(y, make_float2(-1.0f, -1.0f), u);
}

// norm, gain, rotary position and, on demand, the Hadamard transform of one head. `f4`: this lane's stretch of the token's factors, four rows of QR_ROW: with the
// gains ga, gb of the two halves, cos ga, -sin gb, cos gb, sin ga. The factor of the norm is common to the head: it is returned and applied to
// what leaves.
template <int C>
__device__ __forceinline__ float transform(Lane<C>& f, bool norm, float eps, const float* f4, int t, bool rotate) {
  constexpr int P = C / 2, L = 64 / C;
  float r = rotate ? 0.08838834764831845f : 1.0f;  // 1 / sqrt(128) of the transform
  if (norm) {
    float2 s0 = make_float2(0.0f, 0.0f), s1 = s0;
#pragma unroll
    for (int j = 0; j < P; ++j) s0 = __ffma2_rn(f.a[j], f.a[j], s0), s1 = __ffma2_rn(f.b[j], f.b[j], s1);
    float ss = (s0.x + s0.y) + (s1.x + s1.y);
#pragma unroll
    for (int m = 1; m < L; m <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
    r = r / sqrtf(ss * 0.0078125f + eps);
  }
#pragma unroll
  for (int j = 0; j < P; j += 2) {
    const float4 ca = *reinterpret_cast<const float4*>(f4 + 2 * j), sb = *reinterpret_cast<const float4*>(f4 + QR_ROW + 2 * j);
    const float4 cb = *reinterpret_cast<const float4*>(f4 + 2 * QR_ROW + 2 * j), sa = *reinterpret_cast<const float4*>(f4 + 3 * QR_ROW + 2 * j);
    const float2 a0 = f.a[j], b0 = f.b[j], a1 = f.a[j + 1], b1 = f.b[j + 1];
    f.a[j] = __ffma2_rn(b0, make_float2(sb.x, sb.y), __fmul2_rn(a0, make_float2(ca.x, ca.y)));
    f.b[j] = __ffma2_rn(b0, make_float2(cb.x, cb.y), __fmul2_rn(a0, make_float2(sa.x, sa.y)));
    f.a[j + 1] = __ffma2_rn(b1, make_float2(sb.z, sb.w), __fmul2_rn(a1, make_float2(ca.z, ca.w)));
    f.b[j + 1] = __ffma2_rn(b1, make_float2(cb.z, cb.w), __fmul2_rn(a1, make_float2(sa.z, sa.w)));
  }
  if (rotate) {
#pragma unroll
    for (int j = 0; j < P; ++j) {  // index bit 6, then bit 0
      butterfly(f.a[j], f.b[j]);
      f.a[j] = make_float2(f.a[j].x + f.a[j].y, f.a[j].x - f.a[j].y);
      f.b[j] = make_float2(f.b[j].x + f.b[j].y, f.b[j].x - f.b[j].y);
    }
#pragma unroll
    for (int m = 1; m < P; m <<= 1)  // the other bits inside the lane
#pragma unroll
      for (int j = 0; j < P; ++j)
        if (!(j & m)) butterfly(f.a[j], f.a[j | m]), butterfly(f.b[j], f.b[j | m]);
#pragma unroll
    for (int m = 1; m < L; m <<= 1) {  // across lanes: the upper partner holds the difference
      const float2 sg = t & m ? make_float2(-1.0f, -1.0f) : make_float2(1.0f, 1.0f);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const float2 oa = make_float2(__shfl_xor_sync(0xffffffffu, f.a[j].x, m), __shfl_xor_sync(0xffffffffu, f.a[j].y, m));
        const float2 ob = make_float2(__shfl_xor_sync(0xffffffffu, f.b[j].x, m), __shfl_xor_sync(0xffffffffu, f.b[j].y, m));
        f.a[j] = __ffma2_rn(f.a[j], sg, oa), f.b[j] = __ffma2_rn(f.b[j], sg, ob);
      }
    }
  }
  return r;
}

// The same in 64 bits: y[0 .. C-1] of the lower half, y[C .. 2C-1] of the upper.
template <int C>
__device__ __forceinline__ void transform64(double (&y)[2 * C], bool norm, double eps, const float* gain_a, const float* gain_b, const double* cs,
                                            const double* sn, int t, bool rotate) {
  constexpr int L = 64 / C;
  const double turn = rotate ? 0.08838834764831844055 : 1.0;
  double r = turn;
  if (norm) {
    double s0 = 0.0, s1 = 0.0;
#pragma unroll
    for (int e = 0; e < C; ++e) s0 = fma(y[e], y[e], s0), s1 = fma(y[C + e], y[C + e], s1);
    double ss = s0 + s1;
#pragma unroll
    for (int m = 1; m < L; m <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
    r = turn / sqrt(ss * 0.0078125 + eps);
  }
#pragma unroll
  for (int e = 0; e < C; ++e) {
    double a = y[e] * r, b = y[C + e] * r;
    if (norm) a *= static_cast<double>(gain_a[e]), b *= static_cast<double>(gain_b[e]);
    const double c = cs[e], s = sn[e];
    y[e] = fma(a, c, -(b * s));
    y[C + e] = fma(b, c, a * s);
  }
  if (rotate) {
#pragma unroll
    for (int m = 1; m < 2 * C; m <<= 1)  // the bits inside the lane
#pragma unroll
      for (int e = 0; e < 2 * C; ++e)
        if (!(e & m)) {
          const double u = y[e], v = y[e | m];
          y[e] = u + v, y[e | m] = u - v;
        }
#pragma unroll
    for (int m = 1; m < L; m <<= 1) {
      const double sg = t & m ? -1.0 : 1.0;
#pragma unroll
      for (int e = 0; e < 2 * C; ++e) y[e] = fma(y[e], sg, __shfl_xor_sync(0xffffffffu, y[e], m));
    }
  }
}

__device__ __forceinline__ uint32_t clamp_code(float q) { return static_cast<uint32_t>(max(-8, min(7, __float2int_rn(q)))) & 0xFu; }

template <bool APPEND, int L>
__global__ void __launch_bounds__(QR_THREADS, APPEND ? 4 : 5) qk_norm_rope_kernel(const QkParams p) {
  constexpr int C = 64 / L, P = C / 2, W = C / 4, PER_WARP = 32 / L;  // dims of a half, pairs, 8-byte words, heads of a unit
  __shared__ __align__(16) float factors[QR_TOKENS][APPEND ? 1 : 2][4][QR_ROW];  // of the queries and (what is not appended) of the keys
  __shared__ __align__(16) double csk[APPEND ? QR_TOKENS : 1][APPEND ? QR_ROW : 1], snk[APPEND ? QR_TOKENS : 1][APPEND ? QR_ROW : 1];
  __shared__ __align__(16) float gains[2][2 * QR_ROW];  // queries, keys; dims 0 .. 63 and 64 .. 127 padded as the angles are
  __shared__ int64_t slots[QR_TOKENS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & (L - 1), group = lane / L;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * p.tokens;
  const int n_tok = static_cast<int>(min(static_cast<int64_t>(p.tokens), p.N - t0));
  // Heads of the block, token by token, PER_WARP to a unit: the append's keys (the longest), its values, and what goes out as bf16.
  const int n_k = APPEND ? n_tok * p.Hk : 0, n_out = n_tok * (APPEND ? p.Hq : p.Hq + p.Hk);
  const int uk = (n_k + PER_WARP - 1) / PER_WARP, n_units = 2 * uk + (n_out + PER_WARP - 1) / PER_WARP;
  struct Unit {
    int kind, tok, h;  // kind 0 keys, 1 values, 2 out as bf16: the same for the warp
    bool live;
    uint2 w[2 * W];
  };
  pq::pdl_wait();
  if (!APPEND) pq::pdl_trigger();  // a writer of cache rows does not (see pq_launch_pdl)
  if (APPEND && threadIdx.x < n_tok) {
    int64_t s = pq::ld_dep(p.slot + t0 + threadIdx.x);
    if (s >= p.n_slots) {
      pq::report(p.status, PQ_ERR_SHAPE);
      s = -1;
    }
    slots[threadIdx.x] = s;
  }
  if (APPEND) __syncthreads();
  auto request = [&](int u, Unit& x) {
    x.kind = u < uk ? 0 : u < 2 * uk ? 1 : 2;
    const int per = x.kind == 2 ? (APPEND ? p.Hq : p.Hq + p.Hk) : p.Hk;
    const int v = PER_WARP * (x.kind == 0 ? u : x.kind == 1 ? u - uk : u - 2 * uk) + group;
    const bool in = v < (x.kind == 2 ? n_out : n_k);
    x.tok = in ? (v >= per) + (v >= 2 * per) + (v >= 3 * per) : 0;  // of at most QR_TOKENS
    x.h = in ? v - x.tok * per : 0;
    x.live = in && (!APPEND || slots[x.tok] >= 0);
    const int head = x.kind == 0 ? p.Hq + x.h : x.kind == 1 ? p.Hq + p.Hk + x.h : x.h;
    const __nv_bfloat16* src = p.x + (t0 + x.tok) * p.ld + static_cast<int64_t>(head) * 128 + t * C;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (W >= 2) {
#pragma unroll
        for (int j = 0; j < W; j += 2) {
          const uint4 v4 = x.live ? pq::ld_dep(reinterpret_cast<const uint4*>(src + 64 * i) + j / 2) : make_uint4(0, 0, 0, 0);
          x.w[i * W + j] = make_uint2(v4.x, v4.y), x.w[i * W + (W > 1 ? j + 1 : j)] = make_uint2(v4.z, v4.w);
        }
      } else {
        x.w[i] = x.live ? pq::ld_dep(reinterpret_cast<const uint2*>(src + 64 * i)) : make_uint2(0, 0);
      }
    }
  };
  Unit next;
  if (warp < n_units) request(warp, next);  // on its way while the angles are formed
  const bool norm = p.gq != nullptr;
  if (norm) {  // a pair of gains to a thread
    const int which = threadIdx.x >> 6, i = threadIdx.x & 63;
    const uint32_t w = pq::ld_dep(reinterpret_cast<const uint32_t*>(which ? p.gk : p.gq) + i);
    float* dst = gains[which] + (i >= 32 ? QR_ROW : 0) + angle_at((2 * i) & 63);
    dst[0] = bf16_lo(w), dst[1] = bf16_hi(w);
  }
  __syncthreads();
  auto put = [&](int tok, int i, float c, float s) {
    const int at = angle_at(i);
#pragma unroll
    for (int which = 0; which < (APPEND ? 1 : 2); ++which) {
      const float ga = norm ? gains[which][at] : 1.0f, gb = norm ? gains[which][QR_ROW + at] : 1.0f;
      float(*f)[QR_ROW] = factors[tok][which];
      f[0][at] = c * ga, f[1][at] = -s * gb, f[2][at] = c * gb, f[3][at] = s * ga;
    }
  };
  for (int k = threadIdx.x; k < n_tok * 64; k += QR_THREADS) {
    const int i = k & 63, tok = k >> 6;
    const int axis = i < p.end0 ? 0 : i < p.end1 ? 1 : 2;
    const double turn = static_cast<double>(pq::ld_dep(p.pos + axis * p.ld_pos + t0 + tok)) * p.turns[i];
    const double frac = turn - rint(turn);  // in [-1/2, 1/2], exact
    if (APPEND) {
      double s, c;
      sincospi(2.0 * frac, &s, &c);
      csk[APPEND ? tok : 0][APPEND ? angle_at(i) : 0] = c, snk[APPEND ? tok : 0][APPEND ? angle_at(i) : 0] = s;
      put(tok, i, static_cast<float>(c), static_cast<float>(s));
    } else {
      float s, c;
      sincospif(static_cast<float>(2.0 * frac), &s, &c);
      put(tok, i, c, s);
    }
  }
  __syncthreads();
  const int col = angle_at(t * C);  // of this lane's stretch in a padded row

  for (int u = warp; u < n_units; u += QR_WARPS) {
    const Unit x = next;
    if (u + QR_WARPS < n_units) request(u + QR_WARPS, next);
    const int64_t row = t0 + x.tok;
    Lane<C> f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      f.a[2 * i] = unpack_bf16(x.w[i].x), f.a[2 * i + 1] = unpack_bf16(x.w[i].y);
      f.b[2 * i] = unpack_bf16(x.w[W + i].x), f.b[2 * i + 1] = unpack_bf16(x.w[W + i].y);
    }
    if (!APPEND || x.kind == 2) {
      const float r = transform<C>(f, norm, p.eps, factors[x.tok][!APPEND && x.h >= p.Hq ? 1 : 0][0] + col, t, p.rotate != 0);
      const float2 r2 = make_float2(r, r);
#pragma unroll
      for (int j = 0; j < P; ++j) f.a[j] = __fmul2_rn(f.a[j], r2), f.b[j] = __fmul2_rn(f.b[j], r2);
      if (x.live) {
        __nv_bfloat16* dst = p.y + row * p.ldy + static_cast<int64_t>(x.h) * 128 + t * C;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2* o = i ? f.b : f.a;
          if (W >= 2) {
#pragma unroll
            for (int j = 0; j < P; j += 4)
              reinterpret_cast<uint4*>(dst + 64 * i)[j / 4] = make_uint4(pack_bf16(o[j].x, o[j].y), pack_bf16(o[j + 1].x, o[j + 1].y),
                                                                         pack_bf16(o[(j + 2) % P].x, o[(j + 2) % P].y), pack_bf16(o[(j + 3) % P].x, o[(j + 3) % P].y));
          } else {
            *reinterpret_cast<uint2*>(dst + 64 * i) = make_uint2(pack_bf16(o[0].x, o[0].y), pack_bf16(o[1].x, o[1].y));
          }
        }
      }
      continue;
    }
    uint32_t codes[2][(C + 7) / 8] = {};  // eight to a word
    float s;
    if (x.kind == 0) {
      double y[2 * C];
#pragma unroll
      for (int j = 0; j < P; ++j) {
        y[2 * j] = static_cast<double>(f.a[j].x), y[2 * j + 1] = static_cast<double>(f.a[j].y);
        y[C + 2 * j] = static_cast<double>(f.b[j].x), y[C + 2 * j + 1] = static_cast<double>(f.b[j].y);
      }
      transform64<C>(y, norm, static_cast<double>(p.eps), gains[1] + col, gains[1] + QR_ROW + col, csk[APPEND ? x.tok : 0] + (APPEND ? col : 0),
                     snk[APPEND ? x.tok : 0] + (APPEND ? col : 0), t, p.rotate != 0);
      if (p.steps) {
        double mx = 0.0;
#pragma unroll
        for (int e = 0; e < 2 * C; ++e) mx = fmax(mx, fabs(y[e]));
#pragma unroll
        for (int m = 1; m < L; m <<= 1) mx = fmax(mx, __shfl_xor_sync(0xffffffffu, mx, m));
        s = mx < 0x1p-57 ? 1.0f : __double2float_rn(mx / 7.0);
      } else {
        s = pq::ld_dep(p.s_k + x.h);
      }
      // (1 / s in 64 bits leaves the quotient exact to 2^-52: rounded to fp32 it is the exact quotient's fp32 value, ties of representable ones included)
      const double inv = 1.0 / static_cast<double>(s);
#pragma unroll
      for (int e = 0; e < 2 * C; ++e) codes[e / C][(e % C) >> 3] |= clamp_code(__double2float_rn(y[e] * inv)) << (4 * (e & 7 & (C - 1)));
    } else {
      if (p.steps) {
        float mx = 0.0f;
#pragma unroll
        for (int j = 0; j < P; ++j) mx = fmaxf(fmaxf(mx, fmaxf(fabsf(f.a[j].x), fabsf(f.a[j].y))), fmaxf(fabsf(f.b[j].x), fabsf(f.b[j].y)));
#pragma unroll
        for (int m = 1; m < L; m <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, m));
        s = mx < 0x1p-57f ? 1.0f : __fdiv_rn(mx, 7.0f);
      } else {
        s = pq::ld_dep(p.s_v + x.h);
      }
#pragma unroll
      for (int e = 0; e < 2 * C; ++e) {
        const float2 pair = e < C ? f.a[(e % C) >> 1] : f.b[(e % C) >> 1];
        codes[e / C][(e % C) >> 3] |= clamp_code(__fdiv_rn(e & 1 ? pair.y : pair.x, s)) << (4 * (e & 7 & (C - 1)));
      }
    }
    if (x.live) {
      const int64_t slot = slots[x.tok];
      const int64_t vec = ((((slot >> p.page_log2) * p.Hk + x.h) * 2 + x.kind) << p.page_log2) + (slot & ((1 << p.page_log2) - 1));  // (page, head, keys or values)
      uint8_t* dst = p.codes + vec * 64 + t * P;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (C >= 16)
          *reinterpret_cast<uint2*>(dst + 32 * i) = make_uint2(codes[i][0], codes[i][(C + 7) / 8 - 1]);
        else
          *reinterpret_cast<uint16_t*>(dst + 32 * i) = static_cast<uint16_t>(codes[i][0]);
      }
      if (p.steps && t == 0) p.steps[vec] = s;
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
  if (ld < n_cols || ldy < y_cols || (y == x && ldy != ld && N > 1)) return PQ_ERR_INVALID_ARG;  // (of a single row the distance says nothing)
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
  // the frequencies of the last theta of this thread: 64 powers cost as much as the launch
  static thread_local double of_theta = 0.0, turns[64];
  if (theta != of_theta) {
    for (int i = 0; i < 64; ++i) turns[i] = pow(theta, -2.0 * i / 128.0) / 6.283185307179586476925286766559;
    of_theta = theta;
  }
  for (int i = 0; i < 64; ++i) p.turns[i] = turns[i];
  return PQ_OK;
}

// A CTA takes one token while the tokens do not fill the SMs four times over, then more, up to QR_TOKENS.
pq_status launch(void (*many)(const QkParams), void (*few)(const QkParams), pq_ctx* ctx, QkParams& p, cudaStream_t st) {
  const int64_t per = p.N / (4LL * ctx->sm_count);
  p.tokens = static_cast<int32_t>(per < 1 ? 1 : per > QR_TOKENS ? QR_TOKENS : per);
  const int64_t grid = (p.N + p.tokens - 1) / p.tokens;
  if (grid > 0x7fffffffll) return PQ_ERR_SHAPE;
  return pq_launch_pdl(p.N <= 2LL * ctx->sm_count ? few : many, dim3(static_cast<unsigned>(grid)), QR_THREADS, 0, st, p);
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
  return launch(qk_norm_rope_kernel<false, 4>, qk_norm_rope_kernel<false, 16>, ctx, p, static_cast<cudaStream_t>(stream));
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
  return launch(qk_norm_rope_kernel<true, 4>, qk_norm_rope_kernel<true, 16>, ctx, p, static_cast<cudaStream_t>(stream));
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
