// Causal attention of sequences with several rows (prompts, chunks of prompts) over [full-precision prefix || paged 4-bit cache].
//
// Both products run on tcgen05.mma kind::f16 with fp32 accumulators in tensor memory. An item is (sequence, KV head, 2 x floor(128/G) consecutive tokens):
// the G query heads of the KV head fill two 128-row tiles, so that a key tile is expanded once for all of them. An item walks its key tiles (the
// prefix, up to 64 full-precision keys, is a first tile of its own; then 128 cached keys each).
// Work is counted in key tiles and a few more for every item. One CTA per SM takes an equal stretch of the units of all items laid end to end (prefix sums over
// the sequences; inside a sequence the number of tiles before an item is a sum of floors with a closed form), whatever the lengths are: a chunk of a
// long prompt and short prompts fill the chip alike. An item inside one stretch is final; a long item that several stretches share leaves
// partials in the workspace, and the last CTA to finish merges them in the order of the CTAs (short items are not cut).
//   loader warp      bulk copies of the packed K and V rows (and steps) of a key tile, page by page, into a landing ring
//   expansion warps  codes -> K as bf16 integers, V as fp16 integers, both exact, written as [key][dim] tiles in the 128-byte-swizzled layout that serves as
//                    the K-major B operand of S = Q K^T and as the MN-major B operand of O = P V. With own steps they also prepare, per
//                    key, (step of the key x scale, log2 and reciprocal of the step of the value).
//   MMA warp         S_i = Q_i K^T (bf16: every query is exact, whatever its magnitude; prefix keys, fp16, as two bf16 terms), O_i += P_i V with P as the
//                    tensor-memory A operand (fp16)
//   softmax warps    eight per row tile, four for each half of the key columns. A thread has two columns of every eight of four rows (the fragment layout of
//                    tcgen05.ld 16x256b), so that what is read per key serves four rows. The exponent of a weight takes log2 of the value's
//                    step with it, w = 2^(s + log2 step - m): O is in value units, fp16 holds the largest of what enters the sum whatever
//                    the steps are, the denominator is the sum of w / step in fp32 (PQ_UP). Weights are formed in one pass against the
//                    reference m so far; it moves, and the pass is repeated, only when an exponent exceeds it by more than 15 (and at an item's second
//                    tile where that lies far below, PP_LOW).
// Roundings to fewer bits: w to fp16 (2^-11; below 2^-14 in steps of 2^-24 of the reference's weight), the result to bf16. The denominator is the sum of the weights before
// their rounding.
// Inside every group of eight head dims the expansion leaves the order 0,4,1,5,2,6,3,7; Q and the prefix rows are stored in the same order and the output
// columns are put back when they are written. Every wait is bounded.
//
// Bound by the exponentials and the hand-overs between softmax and tensor core: a key tile of an item takes about 4300 clocks, of which the two products need
// 2048 on the tensor core and the 32768 exponentials 2048 on the four special-function units; both row tiles' exponentials overlap (2100), then follow the
// vote on the reference and the store of the weights (700) and the wait for the products (1500). An item costs 10000 clocks more (queries, first
// scores, prefix, output). Measured: 2048 rows x 64 heads behind 21952 keys 1500 us, 0.62 of the measured bf16 rate (1651 TFLOP/s) on the products of visible pairs (own
// steps 1815), 4096 rows x 64 heads 360 (453), 2048 rows 132 (154), 4 ragged prompts up to 2000 x 32 heads 162 (192), 515 rows 26 (29).
// Tried and slower: a thread per row (own steps 2011 us: the constants of 64 keys per thread), half tiles of 64 keys with the scores of two in flight,
// row tiles that form their weights in turn (1631; 1573 with half of the pass shared), queries of later items brought in by the expansion warps (the same),
// eight expansion warps (their 48 registers spill).
#include <atomic>
#include <type_traits>

#include "pq_paged_attn.cuh"

namespace {

constexpr int PP_ROWS = 128;          // query rows per tile (MMA M)
constexpr int PP_KEYS = 128;          // keys per tile
constexpr int PP_PREFIX = 64;         // most key rows of the prefix tile
constexpr int PP_HALF = 128 * 128;    // bytes of one half tile: 128 rows x 64 two-byte values (128 bytes, swizzled)
constexpr int PP_TILE = 2 * PP_HALF;  // a [128][128] tile: dims 0..63, then dims 64..127
constexpr int PP_LAND = PP_KEYS * 64 + 2 * PP_KEYS * 4;  // packed rows of K or V, behind those of V the steps of both
constexpr int PP_LANDS = 3;           // landing slots: K and V rows of a tile take one each, in turn
constexpr int PP_STAGES = 2;
constexpr int PP_SOFTMAX_WARPS = 16;  // per row tile two sets of four warps, a set takes half of the key columns
constexpr int PP_EXPAND_WARPS = 4;
constexpr int PP_WARP_EXPAND0 = PP_SOFTMAX_WARPS, PP_WARP_MMA = PP_WARP_EXPAND0 + PP_EXPAND_WARPS, PP_WARP_LOAD = PP_WARP_MMA + 1;
constexpr int PP_THREADS = 768;  // the warps behind the loader only give their registers
constexpr int PP_TMEM_COLS = 512;     // S0 | S1 | O0 | O1, 128 columns each; each half of P_i lies over the first half of its columns of S_i
constexpr int PP_ITEM_UNITS = 4;    // units of work that an item costs besides its key tiles (queries, prefix, output: 9 us; a tile 2.4)
constexpr int PP_SHORT = 8;         // an item of so many key tiles or fewer is not shared between workers
constexpr float PP_LAZY = 15.0f;      // log2 units an exponent may exceed the reference before it is moved: weights stay inside fp16
// A prefixed key may draw nearly all of the weight while its value is small: what the other weights keep of their bits is then what the output keeps. So where the
// largest exponent of an item's second tile lies more than PP_LOW below the reference, the reference goes down to it, by PP_FAR_.. at most (the sums, in fp32, grow by
// that: of a prefix, whose values are fp16, to 2^102; of cached keys, whose denominators may be 2^60 already, to 2^107). Tried instead: the reference 8 or 10 below the largest exponent always, which moves again and again (4 ragged prompts 191 -> 226 and 242 us).
constexpr float PP_LOW = 10.0f, PP_FAR_PREFIX = 80.0f, PP_FAR_CACHED = 40.0f;
// Registers: 768 threads at 80; the softmax warpgroups take 96, the others leave 48 (512 x 96 + 256 x 48 = 768 x 80).
constexpr int PP_REGS_SOFTMAX = 96, PP_REGS_OTHERS = 48;
constexpr int PP_HALF_KEYS = PP_KEYS / 2;  // key columns of a softmax thread
constexpr int PP_TICKET0 = PQ_PAGED_TICKET0 + PQ_PAGED_MAX_WORKERS;
constexpr int PP_PARTIAL = 256 * 128;  // floats of an item's partial output: [dims / 4][row][4]

struct PpStart {  // where a worker's stretch begins
  int b, h, rt, j0, u0, u1, U, workers;  // (u1 comes by itself)
};
struct PpShared {  // an item that several workers share
  int w0, w1, b, h, rt, row0, n;
};
struct PpBarriers {
  uint64_t land_full[PP_LANDS], land_empty[PP_LANDS];
  uint64_t k_full[PP_STAGES], k_empty[PP_STAGES], v_full[PP_STAGES], v_empty[PP_STAGES];
  uint64_t s_full[2], p_full[2], o_final[2];
  uint64_t q_ready[2], drain;
  int64_t part[PP_THREADS / 32];
  uint32_t tmem_base;
  volatile int abort_flag;
  int merge[2];
  PpStart start;
  PpShared shared[2];
  uint32_t pair_out[2][4];   // [row tile][rows / 32]: a warp of these rows has given up
  float row[2][2][PP_ROWS];  // [row tile][set]: what the two threads of a row tell each other
};
struct PpSteps {  // of pairs of keys: (key step x scale, of both, log2 of the value step, of both) and (2^-PQ_UP / value step, of both)
  float4 key[PP_KEYS / 2];
  float2 inv[PP_KEYS / 2];
};
constexpr size_t PP_SMEM_BYTES = 1024 /*alignment slack*/ + 2 * PP_TILE /*Q*/ + PP_STAGES * 2 * PP_TILE /*K, V*/ + PP_LANDS * PP_LAND +
                                 PP_STAGES * sizeof(PpSteps) + sizeof(PpBarriers);
static_assert(PP_SMEM_BYTES <= 227 * 1024, "shared memory budget");
static_assert((PQ_PAGED_MAX_SEQS + 1) * 4 <= PP_STAGES * 2 * PP_TILE, "the prefix sums lie in the K and V buffers before the pipeline starts");

__device__ __forceinline__ float max3f(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t hfma2_u32(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t bsub2_u32(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Eight codes of one packed word (nibble i = head dim i of the group) as exact fp16 integers in the order (0,4) (1,5) (2,6) (3,7): nibbles 0 and 4 under the
// exponent of 1024 read 1032 + code, nibbles 1 and 5 stay four bits up and read 1152 + 16 * code; one fused multiply-add each removes the offset
// (and the factor 16).
__device__ __forceinline__ uint4 expand8_f16(uint32_t w) {
  const uint32_t w8 = w >> 8;
  const uint32_t ONE = 0x3C003C00u, SIXTEENTH = 0x2C002C00u;  // half2(1, 1), half2(1/16, 1/16)
  const uint32_t M1032 = 0xE408E408u, M72 = 0xD480D480u;      // half2(-1032, -1032), half2(-72, -72)
  uint4 o;
  o.x = hfma2_u32(pq::and_xor<0x000F000Fu, 0x64086408u>(w), ONE, M1032);
  o.y = hfma2_u32(pq::and_xor<0x00F000F0u, 0x64806480u>(w), SIXTEENTH, M72);
  o.z = hfma2_u32(pq::and_xor<0x000F000Fu, 0x64086408u>(w8), ONE, M1032);
  o.w = hfma2_u32(pq::and_xor<0x00F000F0u, 0x64806480u>(w8), SIXTEENTH, M72);
  return o;
}
// The same as exact bf16 integers: under the exponent of 128 (bf16 has seven fraction bits) a nibble reads 136 + code.
__device__ __forceinline__ uint4 expand8_bf16(uint32_t w) {
  const uint32_t OFF = 0x43084308u;  // bf16x2(136, 136)
  return make_uint4(bsub2_u32(pq::and_xor<0x000F000Fu, 0x43084308u>(w), OFF), bsub2_u32(pq::and_xor<0x000F000Fu, 0x43084308u>(w >> 4), OFF),
                    bsub2_u32(pq::and_xor<0x000F000Fu, 0x43084308u>(w >> 8), OFF), bsub2_u32(pq::and_xor<0x000F000Fu, 0x43084308u>(w >> 12), OFF));
}
// Eight two-byte values (d0 .. d7 in four words) in the same order (0,4) (1,5) (2,6) (3,7).
__device__ __forceinline__ uint4 permute8(const uint4& v) {
  return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}
// Two fp16 values as two bf16 terms whose sum they are (8 + 8 of at most 11 significand bits): the first or the second.
__device__ __forceinline__ uint32_t bf16_term(uint32_t h2, bool second) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h2));
  __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
  if (second) {
    const float2 hi = __bfloat1622float2(b);
    b = __floats2bfloat162_rn(f.x - hi.x, f.y - hi.y);
  }
  return *reinterpret_cast<const uint32_t*>(&b);
}
// Byte offset of 16-byte chunk c16 (eight dims; 0..15) of row r inside a [rows][128] tile of two-byte values.
__device__ __forceinline__ uint32_t tile_off(int r, int c16) {
  return static_cast<uint32_t>((c16 >> 3) * PP_HALF + r * 128 + (((c16 & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ void sts128(uint32_t a, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// ---- tcgen05 forms used here (cta_group::1, kind::f16) ----------------------------------------------------
// Instruction descriptor: A and B both fp16 or both bf16 -> fp32, A K-major (or in tensor memory), B K-major or MN-major.
__host__ __device__ constexpr uint32_t idesc_16(int M, int N, bool bf16, bool b_mn_major) {
  return (1u << 4) /*D = f32*/ | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_mn_major ? (1u << 16) : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}
// Shared-memory descriptor of a 128-byte-swizzled operand whose rows are 128 bytes and whose 8-row groups are 1024 bytes apart. K-major use: rows =
// M/N index, the row's bytes = 64 K elements (lbo unused). MN-major use: rows = K index, the row's bytes = 64 M/N elements, lbo = distance
// to the next 64 M/N elements.
__device__ __forceinline__ uint64_t desc_sw128(uint32_t smem_addr, uint32_t lbo_bytes) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr >> 4) & 0x3FFF);
  d |= static_cast<uint64_t>((lbo_bytes >> 4) & 0x3FFF) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
constexpr int PP_CHUNK = 16;  // score columns of a step of the softmax
// 16 rows x 16 columns as a matrix fragment: lane 4g + t gets columns 8n + 2t, 8n + 2t + 1 of row g (r[4n], r[4n + 1]) and of row g + 8 (r[4n + 2], r[4n + 3]).
__device__ __forceinline__ void tmem_ld_frag(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
// The wait with the loaded registers as operands: every use of r stays behind it.
__device__ __forceinline__ void tmem_ld_wait_frag(uint32_t (&r)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
               :
               : "memory");
}
// 16 rows x 32 words, the counterpart: lane 4g + t has word 4n + t of row g (r[2n]) and of row g + 8 (r[2n + 1]).
__device__ __forceinline__ void tmem_st_frag(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// Exchanges between lanes l and l ^ m: the lane with the bit clear keeps a and receives the other's a as b, the other keeps b and receives b as a.
__device__ __forceinline__ void swap_halves(uint4& a, uint4& b, bool bit, int m) {
  uint4 t = bit ? a : b;
  t.x = __shfl_xor_sync(0xffffffffu, t.x, m), t.y = __shfl_xor_sync(0xffffffffu, t.y, m);
  t.z = __shfl_xor_sync(0xffffffffu, t.z, m), t.w = __shfl_xor_sync(0xffffffffu, t.w, m);
  if (bit)
    a = t;
  else
    b = t;
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// sum_{i=0}^{n-1} floor((a i + b) / 128) for a, b >= 0, by the Euclidean reduction of the lattice points under a line (the first step is by shifts).
__device__ int64_t floor_sum_128(int64_t n, int64_t a, int64_t b) {
  int64_t s = (a >> 7) * (n * (n - 1) / 2) + (b >> 7) * n;
  a &= 127, b &= 127;
  int64_t top = a * n + b;
  if (top < 128) return s;
  n = top >> 7;
  uint32_t m32 = static_cast<uint32_t>(a), a32 = 128, b32 = static_cast<uint32_t>(top & 127);  // all below 2^8 from here on
  for (;;) {
    s += static_cast<int64_t>(a32 / m32) * (n * (n - 1) / 2) + static_cast<int64_t>(b32 / m32) * n;
    a32 %= m32, b32 %= m32;
    top = a32 * n + b32;
    if (top < m32) return s;
    if (top < (1ll << 32)) {
      n = static_cast<uint32_t>(top) / m32, b32 = static_cast<uint32_t>(top) % m32;
    } else {
      n = top / m32, b32 = static_cast<uint32_t>(top % m32);
    }
    const uint32_t t = m32;
    m32 = a32, a32 = t;
  }
}

// The stretch of a worker as the roles walk it, item by item.
struct PpItem {
  int b, h, rt;         // sequence, KV head, row tile pair
  int n, len, row0, nt; // of the sequence: new rows, cached keys, first row, row tile pairs
  int base;             // cached keys before the new rows: len - n
  int tiles, j0, j1;    // key tiles of the item (the prefix first), and this worker's
  int u;                // unit where this worker's share begins (an item is PP_ITEM_UNITS units and its tiles)
};

template <bool DYN, bool POLL>
__global__ void __launch_bounds__(PP_THREADS, 1) paged_prefill_kernel(const PagedAttnParams p) {
  extern __shared__ uint8_t pp_raw[];
  uint8_t* smem = pp_raw + (-pq::smem_u32(pp_raw) & 1023u);  // (through an integer the compiler would lose sight of shared memory and use generic loads)
  uint8_t* q_buf = smem;                               // two Q tiles
  uint8_t* kv_buf = q_buf + 2 * PP_TILE;               // stage s: K tile, then V tile
  uint8_t* land = kv_buf + PP_STAGES * 2 * PP_TILE;    // packed rows of K or V
  PpSteps* steps_buf = reinterpret_cast<PpSteps*>(land + PP_LANDS * PP_LAND);
  PpBarriers* bars = reinterpret_cast<PpBarriers*>(steps_buf + PP_STAGES);

  const int warp = pq::warp_index(), lane = threadIdx.x & 31;
  const int G = p.G, RT = PP_ROWS / G, R = 2 * RT;     // tokens of a row tile and of an item
  const int has_prefix = p.n_prefix > 0 ? 1 : 0, pre_cols = p.n_prefix <= 16 ? 16 : PP_PREFIX;  // key rows of the prefix tile
  volatile int* abort_flag = &bars->abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < PP_LANDS; ++i) {
      pq::mbar_init(&bars->land_full[i], 1);
      pq::mbar_init(&bars->land_empty[i], PP_EXPAND_WARPS);
    }
    for (int i = 0; i < PP_STAGES; ++i) {
      pq::mbar_init(&bars->k_full[i], PP_EXPAND_WARPS);
      pq::mbar_init(&bars->k_empty[i], 1);
      pq::mbar_init(&bars->v_full[i], PP_EXPAND_WARPS);
      pq::mbar_init(&bars->v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      pq::mbar_init(&bars->s_full[i], 1);
      pq::mbar_init(&bars->p_full[i], PP_SOFTMAX_WARPS / 2);
      pq::mbar_init(&bars->o_final[i], 1);
      pq::mbar_init(&bars->q_ready[i], PP_SOFTMAX_WARPS / 2);
    }
    pq::mbar_init(&bars->drain, 1);
    bars->abort_flag = 0;
    for (int k = 0; k < 8; ++k) bars->pair_out[k >> 2][k & 3] = 0;
    pq::mbar_fence_init();
  }
  if (warp == PP_WARP_MMA) {
    pq::tmem_alloc(&bars->tmem_base, PP_TMEM_COLS);
    pq::tmem_relinquish();
  }
  pq::pdl_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the kernel for single tokens follows, which only needs what this wait waited for

  // ---- the sequences: number of key tiles of all row tiles of one KV head, prefix sums, and where this worker's stretch begins
  const int64_t capacity = static_cast<int64_t>(p.max_pages) << p.page_log2;
  auto load_seq = [&](PpItem& x, bool& odd) {  // n = 0 for a sequence that is not this kernel's
    const int r0 = pq::ld_dep(p.q_begin + x.b), r1 = pq::ld_dep(p.q_begin + x.b + 1), l = pq::ld_dep(p.len + x.b);
    const int64_t n = static_cast<int64_t>(r1) - r0;
    x.row0 = r0;
    x.len = l < 0 ? 0 : l > capacity ? static_cast<int>(capacity) : l;
    odd = n > p.max_new || n < 0 || (n > 0 && (r0 < 0 || r1 > p.n_rows || l != x.len));
    x.n = n >= 2 && n <= p.max_new && r0 >= 0 && r1 <= p.n_rows ? static_cast<int>(n) : 0;
    x.base = x.len - x.n;
    x.nt = (x.n + R - 1) / R;
  };
  // key tiles of row tile rt; an item with fewer cached keys than rows counts the tiles as if the keys began at zero
  auto tiles_of = [&](const PpItem& x, int rt) { return has_prefix + (max(x.base, 0) + min(x.n, (rt + 1) * R) + PP_KEYS - 1) / PP_KEYS; };
  auto units_before = [&](const PpItem& x, int rt) {  // of the row tiles 0 .. rt - 1, all of them full
    return static_cast<int64_t>(rt) * (has_prefix + PP_ITEM_UNITS) + (rt > 0 ? floor_sum_128(rt, R, static_cast<int64_t>(max(x.base, 0)) + R + PP_KEYS - 1) : 0);
  };
  int32_t* scan = reinterpret_cast<int32_t*>(kv_buf);
  __syncthreads();
  for (int b = threadIdx.x; b < p.B; b += PP_THREADS) {
    PpItem x;
    x.b = b;
    bool odd;
    load_seq(x, odd);
    int64_t t = 0;
    if (x.n > 0) {
      t = units_before(x, x.nt - 1) + PP_ITEM_UNITS + tiles_of(x, x.nt - 1);
    }
    if (odd || t * p.Hkv > 0x7fffffffll) {
      pq::report(p.status, PQ_ERR_SHAPE);
      t = t * p.Hkv > 0x7fffffffll ? 0 : t;  // (more work than any chip's memory holds keys for)
    }
    scan[b] = static_cast<int32_t>(t);
  }
  __syncthreads();
  const int64_t total = pq::block_scan<PP_THREADS>(scan, p.B, bars->part) * p.Hkv;
  if (warp < 2) {  // the two borders of this CTA's stretch, a warp each
    const bool too_many = total > 0x7fffffffll;
    if (too_many && threadIdx.x == 0) pq::report(p.status, PQ_ERR_SHAPE);
    PpStart st{};
    st.U = too_many ? 0 : static_cast<int>(total);
    st.workers = min(static_cast<int>(gridDim.x), max(1, st.U / (PP_ITEM_UNITS + 1)));  // as much as an item of one tile at least
    if (st.U > 0 && static_cast<int>(blockIdx.x) < st.workers) {
      int tiles = 0, at = 0;  // of the item: key tiles, and the unit's place in it (an item's own units come before its tiles)
      auto locate = [&](int u) {  // unit u into (b, h, rt, j0) and the tiles of its item; 32 row tiles are looked at at a time
        PpItem x;
        x.b = pq::find_segment(scan, p.B, u / p.Hkv);
        bool odd;
        load_seq(x, odd);
        const int per_head = scan[x.b + 1] - scan[x.b], rel = u - scan[x.b] * p.Hkv;
        st.b = x.b, st.h = rel / per_head;
        const int v = rel - st.h * per_head;
        int lo = 0, hi = x.nt;  // the item lies in [lo, hi)
        while (hi - lo > 1) {
          const int step = (hi - lo + 31) >> 5, mine = lo + lane * step;
          const uint32_t below = __ballot_sync(0xffffffffu, mine < hi && units_before(x, mine) <= v);  // lanes 0 .. k: ascending, and lane 0 always
          lo += (31 - __clz(below)) * step;
          hi = min(hi, lo + step);
        }
        at = v - static_cast<int>(units_before(x, lo)), tiles = tiles_of(x, lo);
        st.rt = lo, st.j0 = max(0, at - PP_ITEM_UNITS);
      };
      // where stretch w begins: inside a short item, or among an item's own units, an end of the item is taken, so that no partials are left for a few tiles
      auto border = [&](int w) {
        const int u = static_cast<int>(static_cast<int64_t>(st.U) * w / st.workers);
        if (w == st.workers) return u;
        locate(u);
        int to = u;
        if (st.j0 == 0)
          to = u - at;
        else if (tiles <= PP_SHORT)
          to = 2 * st.j0 < tiles ? u - at : u + tiles - st.j0;
        if (to > u && to < st.U) locate(to);
        if (to < u) st.j0 = 0;
        return to;
      };
      const int u = border(blockIdx.x + warp);
      if (lane == 0) {
        if (warp == 0)
          bars->start = st, bars->start.u0 = u;
        else
          bars->part[0] = u;
      }
    } else if (lane == 0) {
      if (warp == 0) bars->start = st;
      if (warp == 1) bars->part[0] = 0;
    }
  }
  pq::tc_fence_before();
  __syncthreads();
  pq::tc_fence_after();
  PpStart start = bars->start;
  start.u1 = static_cast<int>(bars->part[0]);
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, bars->tmem_base, 0);

  auto first_item = [&]() {
    PpItem x;
    x.b = start.b, x.h = start.h, x.rt = start.rt;
    bool odd;
    load_seq(x, odd);
    x.tiles = tiles_of(x, x.rt), x.j0 = start.j0, x.u = start.u0;
    x.j1 = min(x.tiles, x.j0 + (start.u1 - x.u) - (x.j0 == 0 ? PP_ITEM_UNITS : 0));
    return x;
  };
  auto next_item = [&](PpItem& x) {  // false at the end of the stretch
    x.u += x.j1 - x.j0 + (x.j0 == 0 ? PP_ITEM_UNITS : 0);
    if (x.u >= start.u1) return false;
    if (++x.rt == x.nt) {
      x.rt = 0;
      if (++x.h == p.Hkv) {
        x.h = 0;
        bool odd;
        do {
          ++x.b;
          load_seq(x, odd);
        } while (x.n == 0);
      }
    }
    x.tiles = tiles_of(x, x.rt), x.j0 = 0;
    x.j1 = min(x.tiles, start.u1 - x.u - PP_ITEM_UNITS);
    return true;
  };
  auto n_ctx_of = [&](const PpItem& x) { return min(x.len, max(x.base, 0) + min(x.n, (x.rt + 1) * R)); };  // cached keys a row of the item may see
  auto second_tile = [&](const PpItem& x) { return x.n > x.rt * R + RT; };  // does the second row tile have rows

  // Bounded wait; also gives up when another role of the CTA has raised the abort flag.
  auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
    if (pq::mbar_look<POLL>(bar, parity)) return true;
    const long long c0 = clock64();
    for (;;) {
      if (pq::mbar_look<POLL>(bar, parity)) return true;
      if (*abort_flag) return false;
      if (clock64() - c0 > p.wait_clocks) return false;
    }
  };
  auto wait_warp = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, wait(bar, parity)); };
  auto give_up = [&]() {
    bars->abort_flag = 1;
    pq::report(p.status, PQ_ERR_TIMEOUT);
  };

  const bool any = start.u0 < start.u1;
  int lands_issued = 0;  // loader only

  if (warp < PP_SOFTMAX_WARPS) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PP_REGS_SOFTMAX));
    // ================================================================== softmax warps: two threads per query row, one for each half of the key columns
    const int i = warp >> 3, set = (warp >> 2) & 1, row = (warp & 3) * 32 + lane;  // row tile, half of the columns, row of the tile
    const int tok_in = i * RT + row / G, g_in = row % G;  // token of the item and query head of the group (rows past RT * G have none)
    const bool row_used = row < RT * G;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem_base + lane_base + i * 128 + set * PP_HALF_KEYS, o_addr = tmem_base + lane_base + 256 + i * 128 + set * 64;
    const int pair_bar = 2 + i * 4 + (warp & 3);  // named barrier of the two warps of these rows
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory"); };
    auto pair_any = [&](bool v) {  // does any of the 64 threads say so
      uint32_t r;
      asm volatile(
          "{\n.reg .pred p, q;\nsetp.ne.u32 p, %2, 0;\nbarrier.cta.red.or.pred q, %1, 64, p;\nselp.u32 %0, 1, 0, q;\n}\n"
          : "=r"(r)
          : "r"(pair_bar), "r"(static_cast<uint32_t>(v))
          : "memory");
      return r != 0;
    };
    float* const mine = &bars->row[i][set][row];
    const volatile float* const other = &bars->row[i][set ^ 1][row];
    // While weights are formed a thread has the columns 2t, 2t + 1 of every eight of its set, of four rows: fr + 8k. What it needs per key is then read for four
    // rows at once.
    const int fg = lane >> 2, ft = lane & 3, fr = (warp & 3) * 32 + fg;
    uint32_t tok4 = 0;  // tokens of the four rows, a byte each
    for (int k = 0; k < 4; ++k) tok4 |= static_cast<uint32_t>(i * RT + (fr + 8 * k) / G) << (8 * k);
    auto of_lane = [&](const float (&v)[4]) {  // of the row of this lane, where the four lanes of a quad hold the same for their rows
      float r = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = __shfl_sync(0xffffffffu, v[k], (lane & 7) * 4);
        if (lane >> 3 == k) r = x;
      }
      return r;
    };
    bool ok = true;
    // A warp whose wait ran out still comes to the next barrier that the other warp of its rows may be at, and has left word before: named barriers have no
    // bound of their own. Both have passed the same barriers, so that the next one is the same for both.
    volatile uint32_t* const pair_out = &bars->pair_out[i][warp & 3];
    auto leave = [&]() {
      if (lane == 0) *pair_out = 1;
      __syncwarp();
      ok = false;
    };
    int n_tiles_done = 0, n_items_done = 0, c = 0, n_shared = 0;  // of this group: tiles, items; of the CTA: tiles
    PpItem x, ahead;
    // Q staging of the row tile: the warp brings 16 rows in, two rows (512 contiguous bytes) per load instruction
    float next_s_k = 1.0f, next_s_v = 1.0f;
    auto stage_q = [&](const PpItem& y) {
      if (!DYN) next_s_k = fmaxf(pq::ld_dep(p.s_k + y.h), 0x1p-60f), next_s_v = fmaxf(pq::ld_dep(p.s_v + y.h), 0x1p-60f);
      if (i == 1 && !second_tile(y)) return;
      {
        const uint32_t dst = pq::smem_u32(q_buf + i * PP_TILE);
        const int c16 = lane & 15, rw0 = (warp & 7) * 16;
        const __nv_bfloat16* base = p.q + static_cast<int64_t>(y.row0) * p.ldq + static_cast<int64_t>(y.h) * G * 128 + c16 * 8;
        int rq = rw0 + (lane >> 4), tq = rq / G, gq = rq % G;
        const int tq0 = y.rt * R + i * RT, tq_last = min(RT, y.n - tq0) - 1;  // rows that do not exist repeat the last token
        uint4 qv[8];
#pragma unroll
        for (int it = 0; it < 8; ++it) {
          qv[it] = pq::ld_dep(reinterpret_cast<const uint4*>(base + static_cast<int64_t>(tq0 + min(tq, tq_last)) * p.ldq + gq * 128));
          gq += 2;
          while (gq >= G) gq -= G, ++tq;
        }
#pragma unroll
        for (int it = 0; it < 8; ++it) sts128(dst + tile_off(rw0 + it * 2 + (lane >> 4), c16), permute8(qv[it]));
        pq::fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) pq::mbar_arrive(&bars->q_ready[i]);
    };
    if (any) {
      x = first_item();
      stage_q(x);
    }
    for (bool more = any; more && ok; x = ahead) {
      const bool active = i == 0 || second_tile(x);
      const int t0 = x.rt * R, tok = min(t0 + tok_in, x.n - 1), head = x.h * G + g_in;
      const float s_k = next_s_k, s_v = next_s_v;
      if (x.rt + 1 < x.nt) {  // the queries of the sequence's next row tiles into L2: a thread 128 bytes of them
        const int t_next = t0 + R + (threadIdx.x >> 1) / G, g_next = (threadIdx.x >> 1) % G;
        if (threadIdx.x < 2 * R * G && t_next < x.n)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(p.q + static_cast<int64_t>(x.row0 + t_next) * p.ldq + (x.h * G + g_next) * 128 + (threadIdx.x & 1) * 64));
      }
      const float scale_ctx = s_k * p.scale2, log2_sv = DYN ? 0.0f : pq::lg2_approx(s_v), inv_sv = DYN ? 1.0f : 1.0f / s_v;
      const int n_ctx = n_ctx_of(x), tile_min_tok = t0 + i * RT;
      float m_ref[4], l[4];  // l: of this thread's columns
#pragma unroll
      for (int k = 0; k < 4; ++k) m_ref[k] = -INFINITY, l[k] = 0.0f;
      for (int jt = x.j0; jt < x.j1; ++jt, ++c) {
        if (!active) continue;
        const bool is_pre = has_prefix && jt == 0;
        const int key0 = (jt - has_prefix) * PP_KEYS;
        if (__any_sync(0xffffffffu, !wait(&bars->s_full[i], n_tiles_done & 1) || (DYN && !wait(&bars->v_full[c % PP_STAGES], (c / PP_STAGES) & 1)))) {
          leave();
          pair_any(true);  // the other warp of the rows comes to its vote and learns of it there
          break;
        }
        pq::tc_fence_after();
        const int c0 = set * PP_HALF_KEYS;  // this thread's first column; the prefix tile has columns for the first set only
        const bool idle = is_pre && set == 1;
        const float scale = is_pre ? p.scale2 : scale_ctx, add = is_pre ? 0.0f : log2_sv;
        const bool need_mask = is_pre ? p.n_prefix < pre_cols : (key0 + PP_KEYS > x.base + tile_min_tok + 1 || key0 + PP_KEYS > n_ctx);
        const PpSteps* st = steps_buf + c % PP_STAGES;
        // w = 2^(exponent - m) against the reference so far, fp16, kept in registers until the whole tile has been looked at. Where an exponent is more than
        // PP_LAZY above the reference (or there is none yet), the reference is moved to a whole number, the sums and O_i are multiplied by the power
        // of two that makes, and the tile's weights are formed again. The scores stay where they are meanwhile: the weights overwrite them
        // at the end only. The next columns are requested before the current ones are worked on.
        const float2 scale2 = make_float2(scale, scale);
        uint32_t pk[2][16];  // the weights as they are stored: rows fr, fr + 8, then rows fr + 16, fr + 24
        float2 l2[4];
        for (bool again = false;; again = true) {
          float off[4], top[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float m_use = m_ref[k] == -INFINITY ? 0.0f : m_ref[k];
            off[k] = DYN ? pq::PQ_UP - m_use : add - m_use, top[k] = -INFINITY, l2[k] = make_float2(0.0f, 0.0f);
          }
          auto form = [&](auto chunks) {  // the weights of so many times sixteen columns
            uint32_t rr[2][8];
            tmem_ld_frag(s_addr, rr[0]);
#pragma unroll
            for (int cc = 0; cc < chunks.value; ++cc) {
              float4 key[2];
              float2 inv[2];
              if (DYN) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                  const int pair = ((c0 + cc * PP_CHUNK + n * 8) >> 1) + ft;
                  key[n] = st->key[pair], inv[n] = st->inv[pair];
                }
              }
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {  // rows fr, fr + 8; rows fr + 16, fr + 24
                uint32_t(&r)[8] = rr[hf];
                tmem_ld_wait_frag(r);
                if (hf == 0)
                  tmem_ld_frag(s_addr + (16u << 16) + cc * PP_CHUNK, rr[1]);
                else if (cc + 1 < chunks.value)
                  tmem_ld_frag(s_addr + (cc + 1) * PP_CHUNK, rr[0]);
                float2 ex[4];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                  for (int y = 0; y < 2; ++y) {
                    const float2 v = make_float2(__uint_as_float(r[4 * n + 2 * y]), __uint_as_float(r[4 * n + 2 * y + 1]));
                    const float2 off2 = make_float2(off[2 * hf + y], off[2 * hf + y]);
                    if (DYN)
                      ex[2 * n + y] = __fadd2_rn(__ffma2_rn(v, make_float2(key[n].x, key[n].y), make_float2(key[n].z, key[n].w)), off2);
                    else
                      ex[2 * n + y] = __ffma2_rn(v, scale2, off2);
                  }
                if (need_mask) {
#pragma unroll
                  for (int y = 0; y < 2; ++y) {
                    const int tk = min(t0 + static_cast<int>((tok4 >> (16 * hf + 8 * y)) & 255u), x.n - 1);
                    // visible columns of the row, counted from this thread's first
                    const int limit = (is_pre ? p.n_prefix : min(n_ctx - key0, x.base + tk - key0 + 1)) - c0 - 2 * ft;
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                      ex[2 * n + y].x = cc * PP_CHUNK + 8 * n < limit ? ex[2 * n + y].x : -INFINITY;
                      ex[2 * n + y].y = cc * PP_CHUNK + 8 * n + 1 < limit ? ex[2 * n + y].y : -INFINITY;
                    }
                  }
                }
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                  for (int y = 0; y < 2; ++y) {
                    const float2 x2 = ex[2 * n + y];
                    top[2 * hf + y] = max3f(top[2 * hf + y], x2.x, x2.y);
                    float2 w = make_float2(pq::ex2_approx(x2.x), pq::ex2_approx(x2.y));
                    if (DYN)
                      l2[2 * hf + y] = __ffma2_rn(w, inv[n], l2[2 * hf + y]), w = __fmul2_rn(w, make_float2(pq::PQ_DOWN, pq::PQ_DOWN));
                    else
                      l2[2 * hf + y] = __fadd2_rn(l2[2 * hf + y], w);
                    pk[hf][4 * cc + 2 * n + y] = pq::pack_f16(w.x, w.y);
                  }
              }
            }
          };
          if (is_pre && pre_cols == PP_CHUNK) {
            if (!idle) form(std::integral_constant<int, 1>());
          } else if (!idle) {
            form(std::integral_constant<int, PP_HALF_KEYS / PP_CHUNK>());
          }
          if (again) break;
          bool over = false;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (DYN) top[k] -= pq::PQ_UP;
            over |= top[k] > (m_ref[k] == -INFINITY ? -INFINITY : PP_LAZY);
          }
          if (x.j0 == 0 && jt == 1)  // (of the row's columns of this set)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float t = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
              t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
              over |= t < -PP_LOW && t != -INFINITY;
            }
          if (!pair_any(over)) break;
          if (*pair_out) {
            ok = false;
            break;
          }
          // the rows' maxima: over the four lanes, then over the two halves of the columns (the last reader of the exchange before is behind the vote)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
            top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
            if (ft == k) bars->row[i][set][fr + 8 * k] = top[k];
          }
          pair_sync();
          float alpha[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float most = fmaxf(top[k], *const_cast<const volatile float*>(&bars->row[i][set ^ 1][fr + 8 * k]));
            const bool first = m_ref[k] == -INFINITY, move = most > (first ? -INFINITY : PP_LAZY) || (most < -PP_LOW && most != -INFINITY && jt == 1 && x.j0 == 0);
            const float m_new = move ? ceilf(first ? most : m_ref[k] + fmaxf(most, has_prefix ? -PP_FAR_PREFIX : -PP_FAR_CACHED)) : m_ref[k];
            alpha[k] = move ? pq::ex2_approx(m_ref[k] - m_new) : 1.0f;  // 2^(-inf) = 0 for a row that had seen nothing
            l[k] = DYN && move ? pq::at_reference(l[k], m_ref[k] - m_new) : l[k] * alpha[k];
            m_ref[k] = m_new;
          }
          if (jt > x.j0) {  // S_i of this tile is complete, so O_i += P V of the tile before is, too
            const float f = of_lane(alpha);
            for (int k = 0; k < 4; ++k) {  // this set's half of the dims
              uint32_t q[16];
              tmem_ld_32x16(o_addr + k * 16, q);
#pragma unroll
              for (int e = 0; e < 16; ++e) q[e] = __float_as_uint(__uint_as_float(q[e]) * f);
              tmem_st_32x16(o_addr + k * 16, q);
            }
          }
        }
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float lt = l2[k].x + l2[k].y;
          l[k] += DYN || is_pre ? lt : lt * inv_sv;
        }
        if (!idle) tmem_st_frag(s_addr, pk[0]), tmem_st_frag(s_addr + (16u << 16), pk[1]);
        pq::tmem_st_wait();
        pq::tc_fence_before();
        __syncwarp();
        if (lane == 0) pq::mbar_arrive(&bars->p_full[i]);
        ++n_tiles_done;
      }
      if (!ok) break;
      // the scores of the item are done, its Q tile is free: the next item's queries come in under the last product, its scores under the epilogue
      ahead = x;
      more = next_item(ahead);
      if (more) stage_q(ahead);
      if (active) {
        if (__any_sync(0xffffffffu, !wait(&bars->o_final[i], n_items_done & 1))) {
          leave();
          pair_sync();
        } else {
          ++n_items_done;
          pq::tc_fence_after();
          const bool whole = x.j0 == 0 && x.j1 == x.tiles, live = row_used && t0 + tok_in < x.n;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
            l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
          }
          float sum = of_lane(l);
          *mine = sum;  // the sums of the two halves of the columns
          pair_sync();
          if (*pair_out) {
            ok = false;
            break;
          }
          sum += *other;
          const float norm = sum > 0.0f ? 1.0f / sum : 0.0f;
          // rows of the output as this lane stores them: piece `lane & 3` (16 bytes) of 64 bytes of the four rows of its quad
          const int64_t my_row = live ? static_cast<int64_t>(x.row0 + tok) * p.Hq + head : -1;
          int64_t out_row[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) out_row[k] = __shfl_sync(0xffffffffu, my_row, (lane & ~3) + k);
          const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (x.j0 == 0 ? 1 : 0);
          float4* part = reinterpret_cast<float4*>(p.ws_o + slot * PP_PARTIAL) + i * PP_ROWS + row;  // [dims / 4][256 rows]
          pair_sync();  // both have read before either writes again
          for (int cc = 2 * set; cc < 2 * set + 2; ++cc) {  // this set's half of the dims
            uint32_t r[32];
            pq::tmem_ld_32x32(o_addr + (cc & 1) * 32, r);
            pq::tmem_ld_wait_for(r);
            if (whole) {
              uint4 piece[4];
#pragma unroll
              for (int a = 0; a < 4; ++a) {  // columns 8a .. 8a+7 hold dims 0,4,1,5,2,6,3,7 of the group
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r[8 * a + e]) * norm;
                const __nv_bfloat162 d01 = __floats2bfloat162_rn(v[0], v[2]), d23 = __floats2bfloat162_rn(v[4], v[6]);
                const __nv_bfloat162 d45 = __floats2bfloat162_rn(v[1], v[3]), d67 = __floats2bfloat162_rn(v[5], v[7]);
                piece[a] = make_uint4(*reinterpret_cast<const uint32_t*>(&d01), *reinterpret_cast<const uint32_t*>(&d23), *reinterpret_cast<const uint32_t*>(&d45),
                                      *reinterpret_cast<const uint32_t*>(&d67));
              }
              swap_halves(piece[0], piece[1], lane & 1, 1), swap_halves(piece[2], piece[3], lane & 1, 1);
              swap_halves(piece[0], piece[2], lane & 2, 2), swap_halves(piece[1], piece[3], lane & 2, 2);
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (out_row[k] >= 0) *reinterpret_cast<uint4*>(p.out + out_row[k] * 128 + cc * 32 + (lane & 3) * 8) = piece[k];
            } else if (live) {
#pragma unroll
              for (int a = 0; a < 4; ++a) {
                part[(cc * 8 + a * 2) * 256] = make_float4(__uint_as_float(r[8 * a]), __uint_as_float(r[8 * a + 2]), __uint_as_float(r[8 * a + 4]), __uint_as_float(r[8 * a + 6]));
                part[(cc * 8 + a * 2 + 1) * 256] = make_float4(__uint_as_float(r[8 * a + 1]), __uint_as_float(r[8 * a + 3]), __uint_as_float(r[8 * a + 5]), __uint_as_float(r[8 * a + 7]));
              }
            }
            __syncwarp();
          }
          if (!whole) {
            const float m_row = of_lane(m_ref);
            if (live && set == 0) *reinterpret_cast<float2*>(p.ws_ml + (slot * 256 + i * PP_ROWS + row) * 2) = make_float2(m_row, sum);
          }
          pq::tc_fence_before();
        }
      }
      if (x.j0 != 0 || x.j1 != x.tiles) {
        if (threadIdx.x == 0) {
          const int u = x.j0 == 0 ? x.u + PP_ITEM_UNITS : x.u - x.j0;  // of the item's first tile
          auto worker_of = [&](int unit) { return static_cast<int>(((static_cast<int64_t>(unit) + 1) * start.workers - 1) / start.U); };
          bars->shared[n_shared & 1] = PpShared{worker_of(u), worker_of(u + x.tiles - 1), x.b, x.h, x.rt, x.row0, x.n};
        }
        ++n_shared;
      }
    }
    // ---- the last of the workers w0 .. w1 of a shared item to come here merges their partials, in that order
    if (!ok && lane == 0) give_up();
    __threadfence();
    asm volatile("bar.sync 1, 512;" ::: "memory");
    if (threadIdx.x < 2) {
      const bool go = !bars->abort_flag && static_cast<int>(threadIdx.x) < n_shared;
      const PpShared sh = bars->shared[threadIdx.x];
      bars->merge[threadIdx.x] = go && atomicAdd(p.tickets + PP_TICKET0 + sh.w0, 1u) == static_cast<uint32_t>(sh.w1 - sh.w0) ? 1 : 0;
    }
    asm volatile("bar.sync 1, 512;" ::: "memory");
    __threadfence();
    for (int k = 0; k < 2; ++k) {
      if (!bars->merge[k]) continue;
      const PpShared sh = bars->shared[k];
      const int tok = sh.rt * R + tok_in;
      if (row_used && tok < sh.n) {
        auto slot_of = [&](int w) { return 2 * static_cast<int64_t>(w) + (w == sh.w0 ? 1 : 0); };
        const int my = i * PP_ROWS + row;
        float m = -INFINITY, l = 0.0f;
        for (int w0 = sh.w0; w0 <= sh.w1; w0 += 4) {  // references and denominators, four requests at a time
          float2 ml[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            ml[k] = w0 + k <= sh.w1 ? __ldcg(reinterpret_cast<const float2*>(p.ws_ml) + slot_of(w0 + k) * 256 + my) : make_float2(-INFINITY, 0.0f);
          const float mn = fmaxf(m, fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)));
          l = m == -INFINITY ? 0.0f : DYN ? pq::at_reference(l, m - mn) : l * pq::ex2_approx(m - mn);
#pragma unroll
          for (int k = 0; k < 4; ++k) l = ml[k].x == -INFINITY ? l : DYN ? l + pq::at_reference(ml[k].y, ml[k].x - mn) : fmaf(ml[k].y, pq::ex2_approx(ml[k].x - mn), l);
          m = mn;
        }
        const float m_use = m == -INFINITY ? 0.0f : m, norm = l > 0.0f ? 1.0f / l : 0.0f;
        __nv_bfloat16* dst = p.out + (static_cast<int64_t>(sh.row0 + tok) * p.Hq + sh.h * G + g_in) * 128;
        for (int cc = 2 * set; cc < 2 * set + 2; ++cc) {  // 32 dims at a time, two partials requested together
          float4 acc[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          for (int w = sh.w0; w <= sh.w1; w += 2) {
            const bool two = w < sh.w1;
            const int64_t sa = slot_of(w), sb = two ? slot_of(w + 1) : sa;
            const float4 *pa = reinterpret_cast<const float4*>(p.ws_o + sa * PP_PARTIAL) + cc * 8 * 256 + my;
            const float4 *pb = reinterpret_cast<const float4*>(p.ws_o + sb * PP_PARTIAL) + cc * 8 * 256 + my;
            const float ma = __ldcg(p.ws_ml + (sa * 256 + my) * 2), mb = __ldcg(p.ws_ml + (sb * 256 + my) * 2);
            float4 va[8], vb[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) va[e] = __ldcg(pa + e * 256), vb[e] = __ldcg(pb + e * 256);
            const float fa = ma == -INFINITY ? 0.0f : pq::ex2_approx(ma - m_use) * norm, fb = !two || mb == -INFINITY ? 0.0f : pq::ex2_approx(mb - m_use) * norm;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              acc[e].x = fmaf(vb[e].x, fb, fmaf(va[e].x, fa, acc[e].x)), acc[e].y = fmaf(vb[e].y, fb, fmaf(va[e].y, fa, acc[e].y));
              acc[e].z = fmaf(vb[e].z, fb, fmaf(va[e].z, fa, acc[e].z)), acc[e].w = fmaf(vb[e].w, fb, fmaf(va[e].w, fa, acc[e].w));
            }
          }
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const __nv_bfloat162 a = __floats2bfloat162_rn(acc[e].x, acc[e].y), b = __floats2bfloat162_rn(acc[e].z, acc[e].w);
            const __nv_bfloat162 c2 = __floats2bfloat162_rn(acc[e + 1].x, acc[e + 1].y), d = __floats2bfloat162_rn(acc[e + 1].z, acc[e + 1].w);
            *reinterpret_cast<uint4*>(dst + cc * 32 + e * 4) = make_uint4(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b),
                                                                        *reinterpret_cast<const uint32_t*>(&c2), *reinterpret_cast<const uint32_t*>(&d));
          }
        }
      }
      if (threadIdx.x == 0) p.tickets[PP_TICKET0 + sh.w0] = 0;
    }
  } else if (warp < PP_WARP_MMA) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PP_REGS_OTHERS));
    // ================================================================== expansion warps
    const int tid_e = threadIdx.x & (PP_EXPAND_WARPS * 32 - 1);
    // A thread takes 16 packed bytes of a row at a time, 32 dims: four 16-byte chunks. Threads of the upper 64 dims begin with their third chunk, so that
    // the lanes of a store meet in no bank.
    const int part = tid_e & 3, turn = part & 2;
    bool ok = true;
    int c = 0, lc = 0;  // tile of the CTA, landing slot
    PpItem x;
    if (any) x = first_item();
    for (bool more = any; more && ok; more = next_item(x)) {
      const int n_ctx = n_ctx_of(x);
      for (int jt = x.j0; jt < x.j1 && ok; ++jt, ++c) {
        const int stage = c % PP_STAGES;
        const bool is_pre = has_prefix && jt == 0;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {  // keys, then values
          const int slot = lc % PP_LANDS;
          uint64_t *const full = kv ? bars->v_full : bars->k_full, *const empty = kv ? bars->v_empty : bars->k_empty;
          const uint32_t tile = pq::smem_u32(kv_buf + stage * 2 * PP_TILE + kv * PP_TILE);
          if ((!is_pre && __any_sync(0xffffffffu, !wait(&bars->land_full[slot], (lc / PP_LANDS) & 1))) ||
              __any_sync(0xffffffffu, !wait(&empty[stage], ((c / PP_STAGES) & 1) ^ 1))) {
            ok = false;
            break;
          }
          if (is_pre) {
            // full-precision rows (reordered inside groups of eight dims); rows past n_prefix are zero
            for (int unit = tid_e; unit < pre_cols * 16; unit += PP_EXPAND_WARPS * 32) {
              const int r = unit >> 4, c16 = unit & 15;
              uint4 v = make_uint4(0, 0, 0, 0);
              if (r < p.n_prefix)
                v = permute8(pq::ld_dep(reinterpret_cast<const uint4*>((kv ? p.prefix_v : p.prefix_k) + (static_cast<int64_t>(x.h) * p.n_prefix + r) * 128 + c16 * 8)));
              if (kv) {
                sts128(tile + tile_off(r, c16), v);
              } else {  // two bf16 terms: rows 0 .. and rows 64 ..
                sts128(tile + tile_off(r, c16), make_uint4(bf16_term(v.x, false), bf16_term(v.y, false), bf16_term(v.z, false), bf16_term(v.w, false)));
                sts128(tile + tile_off(PP_PREFIX + r, c16), make_uint4(bf16_term(v.x, true), bf16_term(v.y, true), bf16_term(v.z, true), bf16_term(v.w, true)));
              }
            }
          } else {
            const uint32_t src = pq::smem_u32(land + slot * PP_LAND) + tid_e * 16;
            uint4 w4[PP_KEYS * 4 / (PP_EXPAND_WARPS * 32)];
#pragma unroll
            for (int it = 0; it < PP_KEYS / PP_EXPAND_WARPS / 8; ++it) w4[it] = pq::lds128(src + it * (PP_EXPAND_WARPS * 32 * 16));
#pragma unroll
            for (int it = 0; it < PP_KEYS / PP_EXPAND_WARPS / 8; ++it) {
              const int r = it * (PP_EXPAND_WARPS * 8) + (tid_e >> 2);
              const uint32_t ww[4] = {turn ? w4[it].z : w4[it].x, turn ? w4[it].w : w4[it].y, turn ? w4[it].x : w4[it].z, turn ? w4[it].y : w4[it].w};
              if (kv) {
#pragma unroll
                for (int w = 0; w < 4; ++w) sts128(tile + tile_off(r, 4 * part + (w ^ turn)), expand8_f16(ww[w]));
              } else {
#pragma unroll
                for (int w = 0; w < 4; ++w) sts128(tile + tile_off(r, 4 * part + (w ^ turn)), expand8_bf16(ww[w]));
              }
            }
          }
          if (DYN && kv) {  // thread j: key j of the tile. A key that no row sees adds nothing.
            const float* st = reinterpret_cast<const float*>(land + slot * PP_LAND + PP_KEYS * 64);
            const int key = (jt - has_prefix) * PP_KEYS + tid_e;
            const bool in = !is_pre && key < n_ctx;
            const float k_step = in ? st[tid_e] : 1.0f, v_step = in ? st[PP_KEYS + tid_e] : 1.0f;
            float* key_out = reinterpret_cast<float*>(&steps_buf[stage].key[tid_e >> 1]) + (tid_e & 1);
            key_out[0] = k_step * p.scale2, key_out[2] = pq::lg2_approx(v_step);
            reinterpret_cast<float*>(steps_buf[stage].inv)[tid_e] = pq::rcp_approx(v_step) * pq::PQ_DOWN;
          }
          pq::fence_proxy_async_smem();  // generic-proxy writes -> visible to the tensor core's async proxy
          __syncwarp();
          if (lane == 0) {
            pq::mbar_arrive(&full[stage]);
            if (!is_pre) pq::mbar_arrive(&bars->land_empty[slot]);
          }
          if (!is_pre) ++lc;
        }
      }
    }
    if (!ok && lane == 0) give_up();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PP_REGS_OTHERS));
    if (warp == PP_WARP_LOAD) {
      // ================================================================== loader
      // A lane to a copy: lanes 0 .. 7 the pages of the tile (fewer for larger pages); with own steps lanes 8 .. 15 and 16 .. 23 the steps of their keys and
      // values, which go with the rows of V.
      const int pages = PP_KEYS >> p.page_log2, pg = lane & 7, kind = lane >> 3, page = 1 << p.page_log2;
      bool ok = true;
      PpItem x;
      if (any) x = first_item();
      for (bool more = any; more && ok; more = next_item(x)) {
        const int n_ctx = n_ctx_of(x);
        const int32_t* row = p.table + static_cast<int64_t>(x.b) * p.max_pages;
        for (int jt = max(x.j0, has_prefix); jt < x.j1 && ok; ++jt) {
          const int key0 = (jt - has_prefix) * PP_KEYS, n_here = min(pages, (n_ctx - key0 + page - 1) >> p.page_log2);  // pages with keys in them
          const bool mine = pg < n_here && kind < (DYN ? 3 : 1);
          int id = 0;
          if (mine) {
            id = pq::ld_dep(row + (key0 >> p.page_log2) + pg);
            if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(p.n_pages)) {  // an id that is none is reported and page 0 read in its place
              pq::report(p.status, PQ_ERR_SHAPE);
              id = 0;
            }
          }
          const int64_t vec = ((static_cast<int64_t>(id) * p.Hkv + x.h) * 2) << p.page_log2;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const int slot = lands_issued % PP_LANDS;
            if (!wait_warp(&bars->land_empty[slot], ((lands_issued / PP_LANDS) & 1) ^ 1)) {
              ok = false;
              break;
            }
            const uint32_t dst = pq::smem_u32(land + slot * PP_LAND);
            const uint32_t n_pages = static_cast<uint32_t>(max(n_here, 0));
            if (lane == 0) pq::mbar_arrive_expect_tx(&bars->land_full[slot], n_pages * page * (64 + (DYN && kv ? 8 : 0)));
            __syncwarp();
            if (mine && kind == 0)
              pq::bulk_load(dst + pg * page * 64, p.codes + (vec + kv * page) * 64, page * 64, &bars->land_full[slot]);
            else if (mine && kv)
              pq::bulk_load(dst + PP_KEYS * 64 + (kind - 1) * (PP_KEYS * 4) + pg * page * 4, p.steps + vec + (kind - 1) * page, page * 4, &bars->land_full[slot]);
            ++lands_issued;
          }
        }
      }
      if (!ok && lane == 0) give_up();
    } else if (warp == PP_WARP_MMA) {
      // ================================================================== MMA issuer: the whole warp runs the loop, the elected lane issues
      constexpr uint32_t IDESC_S = idesc_16(PP_ROWS, PP_KEYS, true, false);
      const uint32_t IDESC_S_PRE = idesc_16(PP_ROWS, pre_cols, true, false);
      constexpr uint32_t IDESC_O = idesc_16(PP_ROWS, 128, false, true);
      const bool leader = pq::elect_one();
      const uint64_t q_desc0 = desc_sw128(pq::smem_u32(q_buf), 16), k_desc0 = desc_sw128(pq::smem_u32(kv_buf), 16);
      const uint64_t v_desc0 = desc_sw128(pq::smem_u32(kv_buf + PP_TILE), PP_HALF);
      auto issue_s = [&](int i, int c, bool is_pre) {  // by the elected lane
        const uint64_t q_desc = q_desc0 + i * (PP_TILE >> 4), k_desc = k_desc0 + (c % PP_STAGES) * (2 * PP_TILE >> 4);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {  // 16 head dims per instruction
          const uint32_t off = ((kk >> 2) * PP_HALF + (kk & 3) * 32) >> 4;
          mma_ss(tmem_base + i * 128, q_desc + off, k_desc + off, is_pre ? IDESC_S_PRE : IDESC_S, kk ? 1u : 0u);
        }
        if (is_pre)  // the second terms of the prefix keys, 64 rows on
#pragma unroll
          for (int kk = 0; kk < 8; ++kk) {
            const uint32_t off = ((kk >> 2) * PP_HALF + (kk & 3) * 32) >> 4;
            mma_ss(tmem_base + i * 128, q_desc + off, k_desc + off + (PP_PREFIX * 128 >> 4), IDESC_S_PRE, 1u);
          }
        pq::mma_commit(&bars->s_full[i]);
      };
      auto issue_pv = [&](int i, int c, bool is_pre, bool first) {
        const uint32_t o_tm = tmem_base + 256 + i * 128, p_tm = tmem_base + i * 128;
        const uint64_t v_desc = v_desc0 + (c % PP_STAGES) * (2 * PP_TILE >> 4);
#pragma unroll
        for (int kk = 0; kk < PP_PREFIX / 16; ++kk)  // 16 keys per instruction
          if (!is_pre || kk * 16 < pre_cols) mma_ts(o_tm, p_tm + kk * 8, v_desc + kk * (2048 >> 4), IDESC_O, (!first || kk > 0) ? 1u : 0u);
        if (!is_pre)
#pragma unroll
          for (int kk = PP_PREFIX / 16; kk < PP_KEYS / 16; ++kk) mma_ts(o_tm, p_tm + PP_HALF_KEYS / 2 + kk * 8, v_desc + kk * (2048 >> 4), IDESC_O, 1u);
      };
      bool ok = true;
      int c = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};
      PpItem x;
      if (any) x = first_item();
      for (bool more = any; more && ok; more = next_item(x)) {
        const int groups = second_tile(x) ? 2 : 1;
        ok = wait_warp(&bars->k_full[c % PP_STAGES], (c / PP_STAGES) & 1);
        for (int i = 0; i < groups && ok; ++i) {
          if (!wait_warp(&bars->q_ready[i], n_q[i] & 1)) {
            ok = false;
            break;
          }
          ++n_q[i];
          pq::tc_fence_after();
          if (leader) {
            issue_s(i, c, has_prefix && x.j0 == 0);
            if (i == groups - 1) pq::mma_commit(&bars->k_empty[c % PP_STAGES]);
          }
          __syncwarp();
        }
        for (int jt = x.j0; jt < x.j1 && ok; ++jt, ++c) {
          const bool is_pre = has_prefix && jt == 0, last = jt + 1 == x.j1;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (i >= groups) break;
            if (!wait_warp(&bars->p_full[i], n_p[i] & 1) || (i == 0 && !wait_warp(&bars->v_full[c % PP_STAGES], (c / PP_STAGES) & 1))) {
              ok = false;
              break;
            }
            ++n_p[i];
            pq::tc_fence_after();
            if (leader) {
              issue_pv(i, c, is_pre, jt == x.j0);
              if (i == groups - 1) pq::mma_commit(&bars->v_empty[c % PP_STAGES]);
            }
            __syncwarp();
            if (!last) {
              if (i == 0 && !wait_warp(&bars->k_full[(c + 1) % PP_STAGES], ((c + 1) / PP_STAGES) & 1)) {
                ok = false;
                break;
              }
              pq::tc_fence_after();
              if (leader) {
                issue_s(i, c + 1, false);
                if (i == groups - 1) pq::mma_commit(&bars->k_empty[(c + 1) % PP_STAGES]);
              }
            } else if (leader) {
              pq::mma_commit(&bars->o_final[i]);
            }
            __syncwarp();
          }
        }
      }
      if (leader) {
        if (!ok) give_up();
        // whatever was issued has finished before tensor memory is released or shared memory given back
        pq::mma_commit(&bars->drain);
      }
      __syncwarp();
      pq::mbar_wait(&bars->drain, 0);
    }
  }

  pq::tc_fence_before();
  __syncthreads();
  if (warp == PP_WARP_LOAD && lane == 0 && bars->abort_flag) {
    // copies that nobody consumed must have landed before the CTA may exit
    for (int k = max(0, lands_issued - PP_LANDS); k < lands_issued; ++k) pq::mbar_wait(&bars->land_full[k % PP_LANDS], (k / PP_LANDS) & 1);
  }
  __syncthreads();
  if (warp == PP_WARP_MMA) {
    pq::tc_fence_after();
    pq::tmem_dealloc(tmem_base, PP_TMEM_COLS);
  }
}

}  // namespace

size_t pq_paged_prefill_ws_bytes(const pq_ctx* ctx) {
  return static_cast<size_t>(2) * ctx->sm_count * (PP_PARTIAL + 256 * 2) * sizeof(float);
}

pq_status pq_paged_prefill_launch(pq_ctx* ctx, PagedAttnParams p, void* ws, cudaStream_t st) {
  const bool dyn = p.steps != nullptr, poll = p.wait_clocks < PQ_SUSPENDED_CLOCKS;
  void (*const kern)(const PagedAttnParams) = poll ? (dyn ? paged_prefill_kernel<true, true> : paged_prefill_kernel<false, true>)
                                                   : (dyn ? paged_prefill_kernel<true, false> : paged_prefill_kernel<false, false>);
  static std::atomic<bool> attr_set[64][2][2] = {};
  if (ctx->device < 0 || ctx->device >= 64 || ctx->sm_count > PQ_PAGED_MAX_WORKERS) return PQ_ERR_UNSUPPORTED;
  if (!attr_set[ctx->device][dyn][poll].load(std::memory_order_relaxed)) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(PP_SMEM_BYTES)) != cudaSuccess) {
      cudaGetLastError();
      return PQ_ERR_CUDA;
    }
    attr_set[ctx->device][dyn][poll].store(true, std::memory_order_relaxed);
  }
  p.ws_o = static_cast<float*>(ws);
  p.ws_ml = p.ws_o + static_cast<size_t>(2) * ctx->sm_count * PP_PARTIAL;
  return pq_launch_pdl(kern, dim3(ctx->sm_count), PP_THREADS, PP_SMEM_BYTES, st, p);
}
