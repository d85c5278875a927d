// Attention of drafted trees: up to 128 new rows of a sequence, each of which sees the prefix, the cached keys before the new ones (through a window, where there is
// one) and, of the new ones, what its mask says.
//
// Few rows do not fill the 128 rows of an MMA, so the products are transposed: the keys, of which there are many, are the MMA's rows, a column is a (token, query head)
// pair, and both products cost what the columns are:
//     S^T[key, column] = K Q^T        O^T[dim, column] = V^T P^T
// The 4-bit codes are expanded into tensor memory, never into shared memory: K as exact bf16 integers (lane = key), V^T as exact fp16 integers (lane = head dim), each the
// A operand of its product. What passes through shared memory is the packed rows, Q and P (the B operands): at 64 columns 640 clocks of its bandwidth per key
// tile in place of 1660 with both operands there.
//
// An item is (sequence, KV head, floor(NC / G) tokens): NC = 32, 64 or 128 columns, by an estimate of the time (form_of). Work is counted in key tiles of 128 and ten more for
// every item. Where there are as many workers as items, and the items are of about one length, a worker takes an item; else every worker takes an equal stretch of the units
// of all items laid end to end. An item inside one stretch is final, one that several share leaves partials in the workspace, and the last CTA to finish merges them
// in the order of the CTAs. Up to 64 columns two CTAs share an SM, so that one's first and last tiles of an item go beside the other's work.
//   loader warp       a TMA box per page (K and V rows of a head, 64-byte-swizzled so that both readers meet no bank twice) into a ring of key tiles; own steps by
//                     asynchronous copies of 16 bytes, a lane to a copy
//   expansion warps   four: a warp expands its 32 keys of a tile, then its 32 head dims of all keys of the tile before (transposed matrix loads; lane 8j + g of a quadrant is
//                     dim 4g + j)
//   two MMA warps     S^T of a tile as soon as K and a buffer are there, O^T as soon as V and P are
//   softmax warps     eight (to 64 columns) or sixteen. A thread is a key, a set of four warps has 32 columns; with 32 columns two sets take the tiles in turn, each with sums
//                     and an O^T of its own, joined at the item's end. Own steps are constants of the thread; masks are a bit per column. A column's reference
//                     exponent m lies in shared memory and moves only when a score exceeds it by more than 15 (one vote of the set per tile): w = 2^(s + log2 step - m) goes
//                     to P in fp16, the denominator (sum of w / step, fp32) stays in the thread until the item ends.
//                     The tiles of an item are walked from the one behind the first keys on, those of the first keys last (TK_LIFT). What decides of
//                     masks is formed once per item (the item's fields read in shared memory for every tile: 12 x 64 rows 311 -> 346 us).
//   helper warp       queries and description of the next item; scores of the prefixed keys (bf16 MMA, the fp16 keys as two terms, fp32 sums), which join at the item's end
//                     and never set a reference
// Roundings to fewer bits: w to fp16 (2^-11; below 2^-14 in steps of 2^-24 of the reference's weight), the result to bf16. Every wait is bounded.
//
// What bounds it. In principle HBM while rows x heads of a KV head are few (128 bytes of codes for 256 D flops a column), the tensor core and the special-function units at
// 128 columns. In practice the instructions of the expansion and the softmax: a key tile takes 0.9 us of an SM with 32 columns, 1.15 with 64, 1.5 with 128 (own steps 1.1,
// 1.6, 2.1); issue slots are 43 - 60 % busy, and with 32 columns warps wait for instructions (3.3 of 15 clocks between two of a warp) as long as for anything else, which is why
// loops here are rolled where that costs nothing. 48 ragged x 5 rows at 6000 keys, own steps, 32 heads on 8: 90 us, 2.1 TB/s of codes; 12 ragged x 64 rows at 16000 keys,
// 64 heads on 8: 294 to 310 us, 675 to 710 TFLOP/s of visible pairs, 0.40 to 0.42 of the measured bf16 rate; 16 ragged x 33 rows through a window of 2048: 45; 1 x 26 rows at
// 1021 keys: 16.6 (17 rows 16.4), of which half are the sums and first loads (2.9 us), the first tile (3) and the end of an item (4); its eight tiles in turn are what keeps
// it there, since an item so short is not cut and 24 to 32 CTAs have all the work.
// The tiles of first keys behind the others, and references below a heavy first key, cost 1 to 3 %.
// In place of this kernel: the prompts' kernel with these masks takes 30, 258, 331 and 75 us for 1 x 26, 48 x 5, 12 x 64 and the windowed 16 x 33 rows.
// Tried and not kept: the softmax warps expand V for 32 columns (48 x 5: 99 us against 97), boxes issued by a lane each (three times as long), steps loaded by the
// softmax threads, one loop over both prefix sums (no difference), the first reference from a key of every warp in place of the largest of all (static 0.2 us less, own steps 2 %
// more), the packed rows read ahead of the waits for tensor memory (no difference), partials merged four columns at a time through a ring of asynchronous copies (large calls 2 to 3 %
// less, small ones up to 5 % more).
#include <limits.h>

#include <atomic>
#include <type_traits>

#include "pq_paged_mma.cuh"
#include "pq_tree_form.cuh"

namespace {

constexpr int TK_KEYS = pq_tree::KEYS;
constexpr int TK_COLS = 32;  // columns of a softmax thread
constexpr int TK_ITEM_UNITS = 10;  // units that an item costs besides its key tiles
constexpr int TK_SHORT = pq_tree::SHORT;
constexpr int TK_PIECE = 15;      // units that cutting an item costs
constexpr int TK_LEAST = 5;       // units of a stretch at least (eleven, an item of one tile: 3 x 26 rows at 1513 keys 23 us for 18, 2 x 18 at 3723 24 for 19)
constexpr float TK_LAZY = 15.0f;
// A first cached key often draws most of the weight and has a small value: what the others' weights keep of their bits is then what the output keeps. So the tiles of first
// keys are an item's last, and a reference that moves to a key so far above the others, or is set by a group's last tile or by one of first keys, stays TK_LIFT below
// it: nothing higher is expected, and the other keys of that tile keep all their bits to 2^-27 of its weight and multiples of 2^-37 of it below.
constexpr float TK_LIFT = 14.0f;
constexpr float TK_NONE = 3.0e38f;  // in place of -m of a column that has seen no key: whatever it sees first exceeds the reference
constexpr int TK_TICKET0 = PQ_PAGED_TICKET0 + PQ_PAGED_MAX_WORKERS;
constexpr int TK_LAND_CODES = TK_KEYS * 128;  // a key tile's packed rows of K and V
constexpr int TK_LAND_STEPS = TK_KEYS * 8;

// NC columns. Up to 64 two CTAs share an SM, so that one's first and last tiles of an item go beside the other's work.
template <int NC>
struct TkShape {
  static constexpr int CTAS = NC < 128 ? 2 : 1;            // of an SM
  static constexpr int SETS = NC < 128 ? 2 : 4;            // of four softmax warps
  static constexpr int GROUPS = SETS * TK_COLS / NC;       // a group of sets has all columns of every GROUPS-th tile
  static constexpr int NB = NC == 64 ? 1 : 2;              // buffers of S and of P
  static constexpr int LANDS = NC == 32 ? 4 : 3;           // landing slots, a key tile each
  static constexpr int P_ROW = NC < 64 ? 64 : 128;         // bytes of a key's row in a panel of P
  static constexpr int P_BYTES = NC * 2 * TK_KEYS;
  static constexpr int COL_O = NB * NC, COL_K = COL_O + GROUPS * NC, COL_V = COL_K + 64, TMEM_COLS = 512 / CTAS;
  static_assert(COL_V + 64 <= TMEM_COLS, "tensor memory");
  static constexpr int SOFTMAX_WARPS = 4 * SETS;
  static constexpr int WARP_EXPAND0 = SOFTMAX_WARPS, WARP_QK = WARP_EXPAND0 + 4, WARP_PV = WARP_QK + 1, WARP_LOAD = WARP_PV + 1, WARP_HELP = WARP_LOAD + 1;
  static constexpr int THREADS = (WARP_HELP + 1) * 32;
  // Registers: 512 threads at 64 (256 x 88 + 256 x 40), 768 at 80 (512 x 96 + 256 x 48).
  static constexpr int REGS_SOFTMAX = NC < 128 ? 88 : 96, REGS_OTHERS = NC < 128 ? 40 : 48;
};

struct TkShared {  // an item that several workers share
  int w0, w1, b, h, it, row0, n;
};
// The stretch of a worker as the roles walk it, item by item.
struct TkItem {
  int b, h, it;              // sequence, KV head, group of tokens
  int n, len, row0, nt;      // of the sequence: new rows, cached keys, first row, groups
  int base;                  // cached keys before the new rows
  int tiles, j0, j1;         // key tiles of the item, and this worker's
  int u;                     // unit where this worker's share begins
  int skip, lo;              // key tiles left out behind the first ones, and the first key of any row's window
};
struct TkStart {  // where a worker's stretch begins
  TkItem x;
  int U, workers;
};

template <int NC>
struct TkState {
  using Sh = TkShape<NC>;
  uint64_t land_full[Sh::LANDS], land_empty[Sh::LANDS];
  uint64_t k_full, k_empty, v_full, v_empty;
  uint64_t s_full[Sh::NB], s_empty[Sh::NB], p_full[Sh::NB], pv_done[Sh::NB];
  uint64_t q_full[2], q_empty[2], pre_full, pre_empty, drain[2];
  int64_t part[Sh::THREADS / 32];
  uint32_t tmem_base;
  volatile int abort_flag;
  int merge[2];
  int border;
  volatile int n_tiles;  // of this CTA, once the loader knows
  TkStart start;
  TkShared shared[2];
  int n_shared, most_units;
  uint32_t out[Sh::SETS];  // a warp of the set has given up
  TkItem item[2];         // as the softmax warps read it, beside its queries; no tiles: there are no more
  uint4 pre_key[8][32];   // prefixed keys as operand B
  alignas(16) float neg_m[Sh::SOFTMAX_WARPS][TK_COLS];  // -m of a column, TK_NONE while it has seen no key; every warp has its copy
  alignas(16) float moved[Sh::SOFTMAX_WARPS][2 * TK_COLS];  // 2^(m before its last move - m behind it), in two factors
  float red[Sh::GROUPS][4][NC];
  int lo[2][NC];  // first key of the window of an item's tokens
};

template <int NC>
constexpr size_t tk_smem_bytes(bool dyn, int n_prefix) {
  return 1024 /*alignment slack*/ + 2 * NC * 256 /*Q*/ + TkShape<NC>::NB * TkShape<NC>::P_BYTES + TkShape<NC>::LANDS * (TK_LAND_CODES + (dyn ? TK_LAND_STEPS : 0)) +
         sizeof(TkState<NC>) + static_cast<size_t>(NC) * ((n_prefix + 3) / 4 * 4) * 4;
}
static_assert(tk_smem_bytes<128>(true, PQ_PAGED_MAX_PREFIX) <= 227 * 1024, "shared memory budget");
// Two CTAs of an SM have 113 KB each: as long a prefix as the rule says, and none longer.
template <int NC, bool DYN>
constexpr bool tk_two_ctas() {
  return tk_smem_bytes<NC>(DYN, pq_tree::two_ctas_prefix(NC, DYN)) <= 113 * 1024 && tk_smem_bytes<NC>(DYN, pq_tree::two_ctas_prefix(NC, DYN) + 1) > 113 * 1024;
}
static_assert(tk_two_ctas<32, false>() && tk_two_ctas<32, true>() && tk_two_ctas<64, false>() && tk_two_ctas<64, true>(), "CTAs of an SM");
static_assert(2 * (PQ_PAGED_MAX_SEQS + 1) * 4 <= 16 * 1024 + 16 * 1024 + 4 * TK_LAND_CODES && 2 * (PQ_PAGED_MAX_SEQS + 1) * 4 <= 32 * 1024 + 16 * 1024 + 3 * TK_LAND_CODES,
              "the prefix sums lie in the buffers of Q, P and the packed rows before the pipeline starts");

// The landing ring's 64-byte swizzle: 16-byte piece c of row r (64 bytes a row, rows from a multiple of 512 bytes on).
__device__ __forceinline__ uint32_t land_off(uint32_t row_off, int c) { return row_off + ((c ^ ((row_off >> 7) & 3)) << 4); }
// Nibbles 0 and 4, nibbles 1 and 5 of a word as exact fp16 integers (the first half of expand8_f16).
__device__ __forceinline__ uint2 expand2_f16(uint32_t w) {
  return make_uint2(hfma2_u32(pq::and_xor<0x000F000Fu, 0x64086408u>(w), 0x3C003C00u, 0xE408E408u), hfma2_u32(pq::and_xor<0x00F000F0u, 0x64806480u>(w), 0x2C002C00u, 0xD480D480u));
}
// 16 rows x 16 words: lane 4g + t has word 4n + t of row g (r[2n]) and of row g + 8 (r[2n + 1]).
__device__ __forceinline__ void tmem_st_frag8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),
               "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_cols(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),
               "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
// An arrival of this thread once its copies so far have landed (counted among the expected ones).
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(pq::smem_u32(bar)) : "memory"); }
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* m, int x, int y, int z, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(m)), "r"(pq::smem_u32(bar)), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[32]) {
  pq::tmem_ld_32x32(taddr, r);
  pq::tmem_ld_wait_for(r);
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(taddr)
      : "memory");
}
// P as the MN-major B operand of the second product: rows = keys, of 64 columns (128-byte swizzle) or of 32 (64-byte swizzle: 8-row groups 512 bytes apart).
__device__ __forceinline__ uint64_t desc_p(uint32_t smem_addr, bool narrow) {
  if (!narrow) return desc_sw128(smem_addr, TK_KEYS * 128);
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr >> 4) & 0x3FFF);
  d |= static_cast<uint64_t>(1) << 16;
  d |= static_cast<uint64_t>(512 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(4) << 61;
  return d;
}
// N = 16 or 32 values of each of 32 lanes, joined over the lanes: lane l ends with value l % N.
template <int N, typename F>
__device__ __forceinline__ float lane_join(float (&v)[N], int lane, const F& f) {
#pragma unroll
  for (int s = N / 2; s >= 1; s >>= 1) {
#pragma unroll
    for (int i = 0; i < s; ++i) {
      const float keep = lane & s ? v[i + s] : v[i], send = lane & s ? v[i] : v[i + s];
      v[i] = f(keep, __shfl_xor_sync(0xffffffffu, send, s));
    }
  }
  if (N == 16) v[0] = f(v[0], __shfl_xor_sync(0xffffffffu, v[0], 16));
  return v[0];
}
__device__ __forceinline__ uint2 pack_bf16x4(const float4& v) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

template <int NC, bool DYN, bool POLL>
__global__ void __launch_bounds__(TkShape<NC>::THREADS, TkShape<NC>::CTAS) paged_tree_kernel(const __grid_constant__ CUtensorMap map, const PagedAttnParams p) {
  using Sh = TkShape<NC>;
  constexpr int LANDS = Sh::LANDS, NB = Sh::NB, T = Sh::GROUPS, SETS = Sh::SETS / T;  // sets of a group
  constexpr int TK_THREADS = Sh::THREADS, TK_SOFTMAX_WARPS = Sh::SOFTMAX_WARPS;
  extern __shared__ uint8_t tk_raw[];
  uint8_t* smem = tk_raw + (-pq::smem_u32(tk_raw) & 1023u);
  uint8_t* q_buf = smem;                                    // two: [half of the dims][column][128 bytes, swizzled]
  uint8_t* p_buf = q_buf + 2 * NC * 256;                    // [buffer][panel of 64 (32) columns][key][128 (64) bytes, swizzled]
  uint8_t* land = p_buf + NB * Sh::P_BYTES;                 // [slot][page][K rows, V rows]
  uint8_t* land_steps = land + LANDS * TK_LAND_CODES;       // [slot][page][steps of K, of V]
  TkState<NC>* st = reinterpret_cast<TkState<NC>*>(land_steps + LANDS * (DYN ? TK_LAND_STEPS : 0));
  float* pre = reinterpret_cast<float*>(st + 1);            // [column][prefixed key]
  static_assert(sizeof(TkState<NC>) % 16 == 0, "alignment");

  const int warp = pq::warp_index(), lane = threadIdx.x & 31;
  const int G = p.G, TI = NC / G;  // tokens of an item
  const int pre_stride = (p.n_prefix + 3) / 4 * 4;
  volatile int* abort_flag = &st->abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < LANDS; ++i) {
      pq::mbar_init(&st->land_full[i], DYN ? 1 + 32 : 1);
      pq::mbar_init(&st->land_empty[i], 4 + (DYN ? 4 * SETS : 0));
    }
    pq::mbar_init(&st->k_full, 4), pq::mbar_init(&st->k_empty, 1), pq::mbar_init(&st->v_full, 4), pq::mbar_init(&st->v_empty, 1);
    for (int i = 0; i < 2; ++i) pq::mbar_init(&st->q_full[i], 1), pq::mbar_init(&st->q_empty[i], 1 + TK_SOFTMAX_WARPS);
    for (int i = 0; i < NB; ++i) {
      pq::mbar_init(&st->s_full[i], 1), pq::mbar_init(&st->s_empty[i], 4 * SETS);
      pq::mbar_init(&st->p_full[i], 4 * SETS), pq::mbar_init(&st->pv_done[i], 1);
    }
    for (int i = 0; i < Sh::SETS; ++i) st->out[i] = 0;
    pq::mbar_init(&st->pre_full, 1), pq::mbar_init(&st->pre_empty, TK_SOFTMAX_WARPS);
    pq::mbar_init(&st->drain[0], 1), pq::mbar_init(&st->drain[1], 1);
    st->abort_flag = 0, st->n_tiles = 0x7fffffff, st->n_shared = 0, st->most_units = 0;
    pq::mbar_fence_init();
  }
  if (warp == Sh::WARP_QK) {
    pq::tmem_alloc(&st->tmem_base, Sh::TMEM_COLS);
    pq::tmem_relinquish();
  }
  if (warp == Sh::WARP_LOAD && lane == 0) pq::tma_prefetch_desc(&map);
  pq::pdl_wait();

  // ---- the sequences: units of work of all groups of one KV head, prefix sums, and where this worker's stretch begins
  const int64_t capacity = static_cast<int64_t>(p.max_pages) << p.page_log2;
  const int first_tiles = (p.n_sink + TK_KEYS - 1) / TK_KEYS;  // key tiles with keys that stay visible
  auto load_rows = [&](TkItem& x) {  // n = 0 for a sequence that is left out; false: something about it is odd
    const int r0 = pq::ld_dep(p.q_begin + x.b), r1 = pq::ld_dep(p.q_begin + x.b + 1), l = pq::ld_dep(p.len + x.b);
    const int64_t n = static_cast<int64_t>(r1) - r0;
    x.row0 = r0;
    x.len = l < 0 ? 0 : l > capacity ? static_cast<int>(capacity) : l;
    x.n = n >= 1 && n <= p.max_new && r0 >= 0 && r1 <= p.n_rows ? static_cast<int>(n) : 0;
    return !(n > p.max_new || n < 0 || (n > 0 && (r0 < 0 || r1 > p.n_rows || l != x.len)));
  };
  auto lay_out = [&](TkItem& x) {  // what follows from rows and length
    x.base = x.len - x.n;
    x.nt = (x.n + TI - 1) / TI;
    // rows lie at the root's place, `base`, or behind it: what all windows leave out
    x.lo = p.window > 0 ? max(0, x.base - p.window + 1) : 0;
    x.skip = max(0, x.lo - first_tiles * TK_KEYS) / TK_KEYS;
    x.tiles = max(1, (x.len + TK_KEYS - 1) / TK_KEYS - x.skip);
  };
  auto load_seq = [&](TkItem& x) {
    load_rows(x);
    lay_out(x);
  };
  // First key of an item's tile jt: the tiles behind the first ones, then those (without keys that stay visible the cache's first, where it is not left out).
  auto first_of = [&](const TkItem& x) { return min(x.tiles, first_tiles > 0 ? first_tiles : x.skip == 0 ? 1 : 0); };
  auto key_of = [&](const TkItem& x, int jt) {
    int at = jt + first_of(x);
    if (at >= x.tiles) at -= x.tiles;
    return (at >= first_tiles ? at + x.skip : at) * TK_KEYS;
  };
  int32_t *scan = reinterpret_cast<int32_t*>(smem), *items = scan + p.B + 1;  // units and items of one KV head before a sequence
  auto units_of = [&](const TkItem& x, bool fine) {
    const int64_t t = static_cast<int64_t>(x.nt) * (x.tiles + TK_ITEM_UNITS);
    const bool too_many = t * p.Hkv > 0x7fffffffll;
    if (!fine || too_many) pq::report(p.status, PQ_ERR_SHAPE);
    return too_many ? 0 : static_cast<int>(t);
  };
  // Up to 32 sequences are a lane each, of the two warps that need the sums: no barrier, and the sequence of the first item comes from a lane (1 x 26 rows at 1021 keys
  // 20 -> 17.5 us, with the end of the kernel that is left out where no item is shared).
  const bool few = p.B <= 32;
  TkItem mine;
  mine.b = lane, mine.n = mine.len = mine.row0 = 0;
  int64_t total = 0, n_items = 0;
  int most_units = 0;
  if (!few) {
    __syncthreads();
    for (int b = threadIdx.x; b < p.B; b += TK_THREADS) {
      TkItem x;
      x.b = b;
      const bool fine = load_rows(x);
      lay_out(x);
      scan[b] = units_of(x, fine);
      items[b] = scan[b] > 0 ? x.nt : 0;
      if (scan[b] > 0) atomicMax(&st->most_units, x.tiles + TK_ITEM_UNITS);
    }
    __syncthreads();
    total = pq::block_scan<TK_THREADS>(scan, p.B, st->part) * p.Hkv, n_items = pq::block_scan<TK_THREADS>(items, p.B, st->part) * p.Hkv;
    most_units = st->most_units;
  } else if (warp < 2) {
    const bool fine = lane < p.B ? load_rows(mine) : true;
    lay_out(mine);
    const int units = units_of(mine, fine || warp > 0), nt = units > 0 ? mine.nt : 0;
    int64_t units_to = units;
    int items_to = nt;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, units_to, d);
      const int v = __shfl_up_sync(0xffffffffu, items_to, d);
      if (lane >= d) units_to += u, items_to += v;
    }
    total = __shfl_sync(0xffffffffu, units_to, 31) * p.Hkv, n_items = static_cast<int64_t>(__shfl_sync(0xffffffffu, items_to, 31)) * p.Hkv;
    most_units = __reduce_max_sync(0xffffffffu, units > 0 ? mine.tiles + TK_ITEM_UNITS : 0);
    if (lane < p.B) {  // (both warps write the same)
      if (lane == 0) scan[0] = items[0] = 0;
      scan[lane + 1] = static_cast<int32_t>(units_to), items[lane + 1] = items_to;
    }
    __syncwarp();
  }
  // An item to a worker where there are enough workers and no item is much longer than an equal share: pieces of items cost their ends and the merge. (16 x 33 rows, window
  // 2048: 66 -> 48 us.)
  const bool direct = n_items <= gridDim.x && static_cast<int64_t>(most_units - TK_PIECE) * gridDim.x <= total;
  if (warp < 2) {  // the two borders of this CTA's stretch, a warp each
    const bool too_many = total > 0x7fffffffll;
    if (too_many && threadIdx.x == 0) pq::report(p.status, PQ_ERR_SHAPE);
    TkStart s{};
    s.U = too_many ? 0 : static_cast<int>(total);
    s.workers = direct ? static_cast<int>(n_items) : min(static_cast<int>(gridDim.x), max(1, s.U / TK_LEAST));
    int u = 0;
    TkItem& x = s.x;
    if (s.U > 0 && static_cast<int>(blockIdx.x) < s.workers) {
      int at = 0;
      auto sequence = [&](int b) {
        x.b = b;
        if (few)
          x.n = __shfl_sync(0xffffffffu, mine.n, b), x.len = __shfl_sync(0xffffffffu, mine.len, b), x.row0 = __shfl_sync(0xffffffffu, mine.row0, b);
        else
          load_rows(x);
        lay_out(x);
      };
      auto locate = [&](int v) {
        sequence(pq::find_segment(scan, p.B, v / p.Hkv));
        const int per_head = scan[x.b + 1] - scan[x.b], per = x.tiles + TK_ITEM_UNITS, rel = v - scan[x.b] * p.Hkv;
        x.h = rel / per_head, x.it = rel % per_head / per;
        at = rel % per_head % per, x.j0 = max(0, at - TK_ITEM_UNITS);
      };
      // inside a short item, or among an item's own units, an end of the item is taken, so that no partials are left for a few tiles
      const int w = blockIdx.x + warp;
      u = static_cast<int>(static_cast<int64_t>(s.U) * w / s.workers);
      if (direct && w < s.workers) {
        sequence(pq::find_segment(items, p.B, w / p.Hkv));
        const int rel = w - items[x.b] * p.Hkv;
        x.h = rel / x.nt, x.it = rel % x.nt, x.j0 = 0;
        u = scan[x.b] * p.Hkv + rel * (x.tiles + TK_ITEM_UNITS);
      } else if (w < s.workers) {
        locate(u);
        int to = u;
        if (x.j0 == 0)
          to = u - at;
        else if (x.tiles <= TK_SHORT)
          to = 2 * x.j0 < x.tiles ? u - at : u + x.tiles - x.j0;
        if (to > u && to < s.U) locate(to);
        if (to < u) x.j0 = 0;
        u = to;
      }
    }
    if (lane == 0) {
      x.u = u;
      if (warp == 0)
        st->start = s;
      else
        st->border = u;
    }
  }
  pq::fence_proxy_async_smem();  // (the sums have been read: copies may land over them)
  pq::tc_fence_before();
  __syncthreads();
  pq::tc_fence_after();
  const int u_end = st->border;
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, st->tmem_base, 0);

  auto first_item = [&]() {
    TkItem x = st->start.x;
    if (DYN) load_seq(x);  // (the same once more: with the copy alone the compiler's loops come out slower, 48 x 5 rows at 6000 keys 102 us for 91)
    x.j1 = min(x.tiles, x.j0 + (u_end - x.u) - (x.j0 == 0 ? TK_ITEM_UNITS : 0));
    return x;
  };
  auto next_item = [&](TkItem& x) {  // false at the end of the stretch
    x.u += x.j1 - x.j0 + (x.j0 == 0 ? TK_ITEM_UNITS : 0);
    if (x.u >= u_end) return false;
    if (++x.it == x.nt) {
      x.it = 0;
      if (++x.h == p.Hkv) {
        x.h = 0;
        do {
          ++x.b;
          load_seq(x);
        } while (x.n == 0);
      }
    }
    x.j0 = 0;
    x.j1 = min(x.tiles, u_end - x.u - TK_ITEM_UNITS);
    return true;
  };
  // Bounded wait of a warp; also gives up when another role of the CTA has raised the abort flag.
  auto wait_warp = [&](uint64_t* bar, uint32_t parity) -> bool {
    if (__builtin_expect(__all_sync(0xffffffffu, pq::mbar_look<POLL>(bar, parity)), 1)) return true;
    const long long c0 = clock64();
    for (;;) {
      const bool done = pq::mbar_look<POLL>(bar, parity);
      if (__all_sync(0xffffffffu, done)) return true;
      if (__any_sync(0xffffffffu, *abort_flag != 0 || clock64() - c0 > p.wait_clocks)) return false;
    }
  };
  auto wait_both = [&](uint64_t* bar, uint32_t parity, uint64_t* bar2, uint32_t parity2) -> bool {
    const bool one = pq::mbar_look<POLL>(bar, parity), two = pq::mbar_look<POLL>(bar2, parity2);
    if (__builtin_expect(__all_sync(0xffffffffu, one && two), 1)) return true;
    return wait_warp(bar, parity) && wait_warp(bar2, parity2);
  };
  auto give_up = [&]() {
    st->abort_flag = 1;
    pq::report(p.status, PQ_ERR_TIMEOUT);
  };
  const bool any = st->start.x.u < u_end;
  int lands_issued = 0;   // loader only
  bool said_all = false;  // loader only: a slot more than those holds its word that this was all

  // Queries of an item into shared memory, and the first keys of its tokens' windows; scores of the prefixed keys in fp32. The first item's by the softmax warps, which have
  // nothing else to do yet, later ones' by the helper.
  auto load_queries = [&](const TkItem& x, int buf, int tid, int threads, auto ahead) {
    const int t0 = x.it * TI, cols = min(TI, x.n - t0) * G;
    const __nv_bfloat16* q0 = p.q + static_cast<int64_t>(x.row0 + t0) * p.ldq + static_cast<int64_t>(x.h) * G * 128;
    const uint32_t dst = pq::smem_u32(q_buf + buf * NC * 256);
    for (int unit0 = tid; unit0 < NC * 16; unit0 += threads * ahead.value) {  // 16-byte pieces
      uint4 v[ahead.value];
#pragma unroll
      for (int i = 0; i < ahead.value; ++i) {
        const int unit = unit0 + i * threads, col = unit >> 4, tok = col / G;
        v[i] = make_uint4(0, 0, 0, 0);  // (columns that do not exist)
        if (col < cols) v[i] = pq::ld_dep(reinterpret_cast<const uint4*>(q0 + tok * p.ldq + (col - tok * G) * 128) + (unit & 15));
      }
#pragma unroll
      for (int i = 0; i < ahead.value; ++i) {
        const int unit = unit0 + i * threads, col = unit >> 4, c16 = unit & 15;
        if (unit < NC * 16) sts128(dst + (c16 >> 3) * (NC * 128) + col * 128 + (((c16 & 7) ^ (col & 7)) << 4), permute8(v[i]));
      }
    }
    if (p.window > 0)
      for (int tok = tid; tok < cols / G; tok += threads) {
        const uint32_t* mask = p.mask + static_cast<int64_t>(x.row0 + t0 + tok) * p.mask_words;
        int sees = 0;
        for (int w = 0; w * 32 < x.n; ++w) {
          uint32_t m = pq::ld_dep(mask + w) | ((t0 + tok) >> 5 == w ? 1u << ((t0 + tok) & 31) : 0u);
          if (x.n - w * 32 < 32) m &= (1u << (x.n - w * 32)) - 1;
          sees += __popc(m);
        }
        st->lo[buf][tok] = x.base + sees - p.window;  // (the row's place is base + sees - 1)
      }
    pq::fence_proxy_async_smem();
  };
  // scores of the prefixed keys, by one warp: columns on the 16-row side of the bf16 MMA (every query is exact), the fp16 keys as two bf16 terms
  auto prefix_scores = [&](const TkItem& x, int buf) {
    const int cols = min(TI, x.n - x.it * TI) * G, g = lane >> 2, t = lane & 3;
    const uint32_t q = pq::smem_u32(q_buf + buf * NC * 256);
    for (int j0 = 0; j0 < p.n_prefix; j0 += 8) {
      // operand B of 16 dims: key j0 + g, in the order of the queries (0,4) (1,5) (2,6) (3,7) of every eight dims
      const uint16_t* key = reinterpret_cast<const uint16_t*>(p.prefix_k) + (static_cast<int64_t>(x.h) * p.n_prefix + j0 + g) * 128 + t;
      __syncwarp();
#pragma unroll 4
      for (int kk = 0; kk < 8; ++kk) {
        uint32_t w[2] = {0, 0};
        if (j0 + g < p.n_prefix)
#pragma unroll
          for (int i = 0; i < 2; ++i) w[i] = __ldcg(key + kk * 16 + 8 * i) | static_cast<uint32_t>(__ldcg(key + kk * 16 + 8 * i + 4)) << 16;
        st->pre_key[kk][lane] = make_uint4(bf16_term(w[0], false), bf16_term(w[1], false), bf16_term(w[0], true), bf16_term(w[1], true));
      }
      __syncwarp();
      for (int col0 = 0; col0 < cols; col0 += 16) {
        float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const int row = col0 + (lane & 15);
#pragma unroll 4
        for (int kk = 0; kk < 8; ++kk) {
          const int c16 = 2 * kk + (lane >> 4);
          uint32_t a[4];
          ldmatrix_x4(q + (c16 >> 3) * (NC * 128) + row * 128 + (((c16 & 7) ^ (row & 7)) << 4), a);
          const uint4 b = st->pre_key[kk][lane];
          mma_bf16(c, a, b.x, b.y), mma_bf16(c, a, b.z, b.w);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = j0 + 2 * t + (i & 1);
          if (j < pre_stride) pre[(col0 + g + 8 * (i >> 1)) * pre_stride + j] = c[i] * p.scale2;
        }
      }
    }
  };

  if (warp < TK_SOFTMAX_WARPS) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::REGS_SOFTMAX));
    // ================================================================== softmax warps: a thread is a key; a set of four warps has 32 columns of every T-th tile
    const int set = warp >> 2, quad = warp & 3, group = set / SETS, col0 = set % SETS * TK_COLS, in_set = quad * 32 + lane;
    const uint32_t lane_base = static_cast<uint32_t>(quad * 32) << 16;
    auto set_sync = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(2 + set) : "memory"); };
    auto any_of = [&](int bar, int threads, bool v) {  // does any of them say so
      uint32_t r;
      asm volatile(
          "{\n.reg .pred p, q;\nsetp.ne.u32 p, %3, 0;\nbarrier.cta.red.or.pred q, %1, %2, p;\nselp.u32 %0, 1, 0, q;\n}\n"
          : "=r"(r)
          : "r"(bar), "r"(threads), "r"(static_cast<uint32_t>(v))
          : "memory");
      return r != 0;
    };
    auto all_sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(Sh::SOFTMAX_WARPS * 32) : "memory"); };
    // A warp whose wait ran out leaves word and still comes to the next vote, where the others learn of it: named barriers have no bound of their own.
    volatile uint32_t* const out_flag = &st->out[set];
    float* const neg_m = st->neg_m[warp];
    float* const moved = st->moved[warp];
    bool ok = true;
    auto leave = [&]() {
      if (lane == 0) *out_flag = 1, st->abort_flag = 1;
      __syncwarp();
      ok = false;
    };
    const uint32_t o_addr = tmem_base + lane_base + Sh::COL_O + group * NC + col0;
    const uint32_t p_row = pq::smem_u32(p_buf) + (col0 >> 6) * (TK_KEYS * 128) + in_set * Sh::P_ROW, p_turn = NC < 64 ? (in_set >> 1) & 3 : in_set & 7;
    const float* const step0 = reinterpret_cast<const float*>(land_steps) + ((in_set >> p.page_log2) << (p.page_log2 + 1)) + (in_set & ((1 << p.page_log2) - 1));
    int n_pre = 0;  // items with the prefix
    int k = 0;      // this group's tiles so far
    if (any) {
      const TkItem x = first_item();
      load_queries(x, 0, threadIdx.x, TK_SOFTMAX_WARPS * 32, std::integral_constant<int, NC / 8 / Sh::SETS>());
      if (threadIdx.x == 0) st->item[0] = x;
      all_sync();
      if (threadIdx.x == 0) pq::mbar_arrive(&st->q_full[0]);
    }
    if (any && !wait_warp(&st->q_full[0], 0)) leave();
    bool more = any;
    int turn = group;                 // this group's first tile of the item
    int slot = group, slot_phase = 0;  // the landing slot of its next tile
    for (int n_items = 0; more; ++n_items) {
      const TkItem& x = st->item[n_items & 1];
      const int n_tiles = x.j1 - x.j0;
      const float scale = DYN ? p.scale2 : fmaxf(pq::ld_dep(p.s_k + x.h), 0x1p-60f) * p.scale2;
      float2 l[TK_COLS / 2];  // of this thread's keys
#pragma unroll
      for (int i = 0; i < TK_COLS / 2; ++i) l[i] = make_float2(0.0f, 0.0f);
      // Tiles that need no masks: from the begin of the last row's window to the first new key (the cache ends behind it), and the first keys' at the end, where all rows see
      // all of them.
      int clear_a = 0, clear_n, clear_from = x.tiles - first_of(x) - x.j0;
      {
        const int first = first_of(x), tile_new = x.base < 0 ? 0 : x.base / TK_KEYS - x.skip;
        if (p.window > 0) {
          const int tile_lo = (max(0, x.base + x.n - p.window) + TK_KEYS - 1) / TK_KEYS - x.skip;
          clear_a = max(0, tile_lo - first);
          if (p.n_sink / TK_KEYS < min(tile_lo, first)) clear_from = INT_MAX;
        }
        clear_n = max(0, tile_new - first - clear_a), clear_a -= x.j0;
        if (tile_new < first) clear_from = INT_MAX;
      }
      for (int i0 = turn; i0 < n_tiles; i0 += T, ++k) {
        const int buf = T > 1 ? group : k % NB, phase = T > 1 ? k & 1 : (k / NB) & 1;
        const uint32_t s_addr = tmem_base + lane_base + buf * NC + col0;
        const bool need_mask = static_cast<uint32_t>(i0 - clear_a) >= static_cast<uint32_t>(clear_n) && i0 < clear_from;
        // what the key's score is multiplied by, log2 of the value's step PQ_UP octaves up, and what its weight counts in the denominator
        float a = scale, b = 0.0f, inv = 1.0f;
        if (DYN) {
          if (ok && !wait_warp(&st->land_full[slot], slot_phase)) leave();
          const float* step = step0 + slot * (TK_LAND_STEPS / 4);
          const float v_step = step[1 << p.page_log2];
          a = step[0] * p.scale2, b = pq::lg2_approx(v_step) + pq::PQ_UP, inv = pq::rcp_approx(v_step) * pq::PQ_DOWN;
          __syncwarp();
          if (lane == 0) pq::mbar_arrive(&st->land_empty[slot]);
          slot += T;
          if (slot >= LANDS) slot -= LANDS, slot_phase ^= 1;
        }
        uint32_t vis = ~0u;  // the columns that see the key
        if (need_mask) {
          vis = 0;
          const int t0 = x.it * TI, n_tok = min(TI, x.n - t0);
          const int key = key_of(x, x.j0 + i0) + in_set, u = key - x.base, tok0 = col0 / G, tok_end = min(n_tok, (col0 + TK_COLS - 1) / G + 1);
          const bool seen = key < x.len && (key >= x.lo || key < p.n_sink), new_key = seen && u >= 0;  // by any row of the sequence
          if (DYN && !seen) a = 0.0f, b = 0.0f, inv = 0.0f;  // (its steps may be anything)
          if (DYN && !(inv < INFINITY)) inv = 0.0f;          // (a draft's that is no number is in the exponents of those who see it; the others' weights are zero)
          if (key - in_set + TK_KEYS <= x.lo) {  // first keys alone, which all rows see
            vis = seen ? ~0u : 0u;
          } else {
            // a lane per token: what it sees of the warp's 32 keys, which lie in two words at most
            uint32_t sees = 0;
            if (__any_sync(0xffffffffu, new_key)) {
              const int u0 = u - lane, w = u0 >> 5;
              if (tok0 + lane < tok_end) {
                const uint32_t* word = p.mask + static_cast<int64_t>(x.row0 + t0 + tok0 + lane) * p.mask_words;
                sees = __funnelshift_r(w >= 0 ? pq::ld_dep(word + w) : 0u, (w + 1) * 32 < x.n ? pq::ld_dep(word + w + 1) : 0u, u0 & 31);
                const int own = t0 + tok0 + lane - u0;
                if (static_cast<uint32_t>(own) < 32) sees |= 1u << own;
              }
            }
#pragma unroll 1
            for (int tok = tok0; tok < tok_end; ++tok) {
              const uint32_t new_keys = __shfl_sync(0xffffffffu, sees, tok - tok0);
              bool see = seen;
              if (new_key)
                see = (new_keys >> lane) & 1;
              else if (p.window > 0)
                see = seen && (key < p.n_sink || key >= st->lo[n_items & 1][tok]);
              const uint32_t heads = (1u << G) - 1;
              const int at = tok * G - col0;
              if (see) vis |= at >= 0 ? heads << at : heads >> -at;
            }
          }
        }
        if (ok && !wait_warp(&st->s_full[buf], phase)) leave();
        pq::tc_fence_after();
        float2 v[TK_COLS / 2];
        auto scores = [&]() {  // less the references
          uint32_t r[TK_COLS];
          tmem_ld_cols(s_addr, r);
#pragma unroll
          for (int i = 0; i < TK_COLS / 2; i += 2) {
            const float4 m4 = *reinterpret_cast<const float4*>(neg_m + 2 * i);
            const float2 s0 = make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), s1 = make_float2(__uint_as_float(r[2 * i + 2]), __uint_as_float(r[2 * i + 3]));
            const float2 a2 = make_float2(a, a), b2 = make_float2(b, b), m0 = make_float2(m4.x, m4.y), m1 = make_float2(m4.z, m4.w);
            v[i] = DYN ? __fadd2_rn(__ffma2_rn(s0, a2, b2), m0) : __ffma2_rn(s0, a2, m0);
            v[i + 1] = DYN ? __fadd2_rn(__ffma2_rn(s1, a2, b2), m1) : __ffma2_rn(s1, a2, m1);
          }
          if (need_mask)
#pragma unroll
            for (int i = 0; i < TK_COLS / 2; ++i) {
              v[i].x = vis & (1u << (2 * i)) ? v[i].x : -INFINITY;
              v[i].y = vis & (2u << (2 * i)) ? v[i].y : -INFINITY;
            }
        };
        // The references go to the whole number above the columns' largest exponents over the set's keys (or TK_LIFT below it) where one lies more than TK_LAZY above, or there
        // is none yet.
        auto move = [&](bool first) {
#pragma unroll 1
          for (int e = 0; e < TK_COLS; e += 16) {
            uint32_t r[16];
            tmem_ld_32x16(s_addr + e, r);
            float f[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = (vis >> e) & (1u << i) ? fmaf(__uint_as_float(r[i]), a, b) : -INFINITY;
            const float most = lane_join(f, lane, [](float x, float y) { return fmaxf(x, y); });
            if (lane < 16) st->red[group][quad][col0 + e + lane] = most;
          }
          set_sync();
          const float(&red)[4][NC] = st->red[group];
          const int col = col0 + lane;  // a lane per column, all four warps alike
          const float top_c = fmaxf(fmaxf(red[0][col], red[1][col]), fmaxf(red[2][col], red[3][col])) - (DYN ? pq::PQ_UP : 0.0f), neg = first ? TK_NONE : neg_m[lane];
          const bool none = neg == TK_NONE, up = none ? top_c > -INFINITY : top_c + neg > TK_LAZY;
          const float m_new = ceilf(top_c) - (none && i0 + T < n_tiles && x.j0 + i0 + first_of(x) < x.tiles ? 0.0f : TK_LIFT);
          if (!first) {  // 2^d for the sums; those of own steps, whose references may lie further apart than fp32 reaches, take it in two factors
            const float d = up ? (none ? -INFINITY : -neg - m_new) : 0.0f;
            moved[lane] = pq::ex2_approx(DYN ? fmaxf(d, -120.0f) : d);
            if (DYN) moved[TK_COLS + lane] = pq::ex2_approx(fminf(d + 120.0f, 0.0f));
          }
          neg_m[lane] = up ? -m_new : neg;
          __syncwarp();
          if (first) return;  // (the tile's vote follows)
          set_sync();         // all four have read what the item's end may overwrite
#pragma unroll
          for (int i = 0; i < TK_COLS / 2; ++i) {
            l[i] = __fmul2_rn(l[i], *reinterpret_cast<const float2*>(moved + 2 * i));
            if (DYN) l[i] = __fmul2_rn(l[i], *reinterpret_cast<const float2*>(moved + TK_COLS + 2 * i));
          }
          const int prev = k - 1;
          if (!wait_warp(&st->pv_done[T > 1 ? group : prev % NB], T > 1 ? prev & 1 : (prev / NB) & 1)) return leave();
          pq::tc_fence_after();
#pragma unroll 1
          for (int e = 0; e < TK_COLS; e += 8) {
            uint32_t r[8];
            tmem_ld_cols(o_addr + e, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * moved[e + i] * (DYN ? moved[TK_COLS + e + i] : 1.0f));
            tmem_st_cols(o_addr + e, r);
          }
          pq::tmem_st_wait();
        };
        auto overflow = [&]() {  // does a score of any of the set's keys exceed its column's reference by too much
          scores();
          float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < TK_COLS / 2; ++i) top4[i & 3] = max3f(top4[i & 3], v[i].x, v[i].y);
          const float top = fmaxf(max3f(top4[0], top4[1], top4[2]), top4[3]) - (DYN ? pq::PQ_UP : 0.0f);
          return __builtin_expect(any_of(2 + set, 128, top > TK_LAZY || !ok), 0);
        };
        bool stop = false;  // a warp of the set has given up
        if (DYN) {  // one copy of the pass: its code is the largest of the kernel, and instructions are what its warps wait for (48 x 12 rows at 6000 keys 198 -> 166 us)
          for (bool fresh = i0 == turn;; fresh = false) {
            if (!fresh) {
              if (!overflow()) break;
              if (*out_flag) {
                stop = true;
                break;
              }
            }
            move(fresh);
          }
        } else {  // (two copies: in that form 12 x 64 rows at 16000 keys took 326 us, in this 298 then)
          if (i0 == turn) move(true);
          if (overflow()) {
            stop = *out_flag != 0;
            if (!stop) {
              move(false);
              scores();
            }
          }
        }
        if (stop) {
          ok = false;
          break;
        }
        pq::tc_fence_before();
        __syncwarp();
        if (lane == 0) pq::mbar_arrive(&st->s_empty[buf]);
        uint32_t pk[TK_COLS / 2];
#pragma unroll
        for (int i = 0; i < TK_COLS / 2; ++i) {
          float2 w = make_float2(pq::ex2_approx(v[i].x), pq::ex2_approx(v[i].y));
          if (DYN)
            l[i] = __ffma2_rn(w, make_float2(inv, inv), l[i]), w = __fmul2_rn(w, make_float2(pq::PQ_DOWN, pq::PQ_DOWN));
          else
            l[i] = __fadd2_rn(l[i], w);
          pk[i] = pq::pack_f16(w.x, w.y);
        }
        // what the buffer of P held before has been read
        if (ok && k >= (T > 1 ? 1 : NB) && !wait_warp(&st->pv_done[buf], phase ^ 1)) leave();
        if (!ok) continue;
        const uint32_t chunk0 = (col0 & 63) >> 3;
#pragma unroll
        for (int j = 0; j < TK_COLS / 8; ++j) sts128(p_row + buf * Sh::P_BYTES + (((chunk0 + j) ^ p_turn) << 4), make_uint4(pk[4 * j], pk[4 * j + 1], pk[4 * j + 2], pk[4 * j + 3]));
        pq::fence_proxy_async_smem();
        pq::tc_fence_before();
        __syncwarp();
        if (lane == 0) pq::mbar_arrive(&st->p_full[buf]);
      }
      // ---- the end of the item: the groups' sums and, where it begins here, the prefix come together
      {
        float s[TK_COLS];
#pragma unroll
        for (int i = 0; i < TK_COLS; ++i) s[i] = i & 1 ? l[i >> 1].y : l[i >> 1].x;
        const float sum = lane_join(s, lane, [](float x, float y) { return x + y; });
        st->red[group][quad][col0 + lane] = sum;
      }
      const float s_v = DYN ? 1.0f : pq::ld_dep(p.s_v + x.h);
      if (turn < n_tiles) {
        const int last = k - 1;
        if (ok && !wait_warp(&st->pv_done[T > 1 ? group : last % NB], T > 1 ? last & 1 : (last / NB) & 1)) leave();
      } else {
        neg_m[lane] = TK_NONE;
      }
      const bool has_prefix = x.j0 == 0 && p.n_prefix > 0;
      if (has_prefix) {
        if (ok && !wait_warp(&st->pre_full, n_pre & 1)) leave();
        ++n_pre;
      }
      // the next item lies beside the other queries
      const int next_turn = (turn - n_tiles) & (T - 1);
      const TkItem& y = st->item[(n_items + 1) & 1];
      if (ok && !wait_warp(&st->q_full[(n_items + 1) & 1], ((n_items + 1) >> 1) & 1)) leave();
      if (any_of(1, TK_SOFTMAX_WARPS * 32, !ok)) {
        ok = false;
        break;
      }
      pq::tc_fence_after();
      float y4[4];  // a head dim of the first prefixed values
      const int dim = 4 * (lane & 7) + (lane >> 3) + 32 * quad;
      const __half* const pv = p.prefix_v + static_cast<int64_t>(x.h) * p.n_prefix * 128 + dim;
      auto prefix_value = [&](int j) { return has_prefix && j < p.n_prefix ? __half2float(__ushort_as_half(__ldcg(reinterpret_cast<const unsigned short*>(pv + j * 128)))) : 0.0f; };
#pragma unroll
      for (int j = 0; j < 4; ++j) y4[j] = prefix_value(j);
      const bool whole = x.j0 == 0 && x.j1 == x.tiles;
      const int64_t part = (2 * static_cast<int64_t>(blockIdx.x) + (x.j0 == 0 ? 1 : 0)) * NC;
      // A warp takes the head dims of its quadrant of PART = 32 / T columns; of group g and column c of them lane g PART + c.
      constexpr int PART = NC / Sh::SETS;
      static_assert(PART * T == 32, "a lane per group and column");
      const int t0 = x.it * TI, cols = min(TI, x.n - t0) * G;
      float m, norm = 1.0f;
      {
        const int g = lane / PART, col = set * PART + lane % PART;
        const float neg = st->neg_m[(g * SETS + col / TK_COLS) * 4 + quad][col % TK_COLS], m_g = neg == TK_NONE ? -INFINITY : -neg;
        const float l_g = (st->red[g][0][col] + st->red[g][1][col]) + (st->red[g][2][col] + st->red[g][3][col]);
        const float* const e = pre + col * pre_stride;
        m = m_g;
        if (has_prefix)
          for (int j = g; j < p.n_prefix; j += T) m = fmaxf(m, e[j]);
#pragma unroll
        for (int d = PART; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        const float d = m_g == -INFINITY ? -INFINITY : m_g - m;
        // (what is no number stays none, also of a column whose scores never set a reference)
        float sum = l_g != l_g ? l_g : DYN ? pq::at_reference(l_g, d) : l_g * pq::ex2_approx(d);
        if (has_prefix)
          for (int j = g; j < p.n_prefix; j += T) sum += pq::ex2_approx(e[j] - m);
#pragma unroll
        for (int d = PART; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (whole)
          norm = sum > 0.0f ? 1.0f / sum : sum == sum ? 0.0f : sum;  // (zero: a column that sees nothing)
        else if (quad == 0 && g == 0)
          *reinterpret_cast<float2*>(p.ws_ml + (part + col) * 2) = make_float2(m, sum);
        moved[lane] = pq::ex2_approx(d) * norm * s_v;
      }
      if (has_prefix) {  // scores to weights, a quarter of the columns to a warp
        set_sync();
        for (int e0 = quad * (PART / 4); e0 < (quad + 1) * (PART / 4); ++e0) {
          const float m_c = __shfl_sync(0xffffffffu, m, e0), norm_c = __shfl_sync(0xffffffffu, norm, e0);
          float* const e = pre + (set * PART + e0) * pre_stride;
          for (int j = lane; j < p.n_prefix; j += 32) e[j] = pq::ex2_approx(e[j] - m_c) * norm_c;
        }
        set_sync();
      }
      __syncwarp();
      // a head dim of eight columns at a time
      int tok = set * PART / G, head = set * PART - tok * G;
      int64_t at = whole ? (static_cast<int64_t>(x.row0 + t0 + tok) * p.Hq + x.h * G + head) * 128 + dim : (part + set * PART) * 128 + dim;
#pragma unroll 1
      for (int e0 = 0; e0 < PART; e0 += 8) {
        const int first = set * PART + e0;  // column
        if (first >= cols) break;
        float acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
#pragma unroll
        for (int g = 0; g < T; ++g) {
          if (((g - group + turn) & (T - 1)) >= n_tiles) continue;  // (the group had no tile: its columns hold another item's)
          uint32_t r[8];
          tmem_ld_cols(tmem_base + lane_base + Sh::COL_O + g * NC + first, r);
          const float4 f0 = *reinterpret_cast<const float4*>(moved + g * PART + e0), f1 = *reinterpret_cast<const float4*>(moved + g * PART + e0 + 4);
          const float f[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] = fmaf(__uint_as_float(r[i]), f[i], acc[i]);
        }
        if (has_prefix)
          for (int j = 0; j < p.n_prefix; j += 4) {
            if (p.n_prefix > 4)
#pragma unroll
              for (int jj = 0; jj < 4; ++jj) y4[jj] = prefix_value(j + jj);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float4 e = *reinterpret_cast<const float4*>(pre + (first + i) * pre_stride + j);
              acc[i] = fmaf(e.x, y4[0], fmaf(e.y, y4[1], fmaf(e.z, y4[2], fmaf(e.w, y4[3], acc[i]))));
            }
          }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (first + i < cols) {
            if (whole)
              p.out[at] = __float2bfloat16_rn(acc[i]);
            else
              p.ws_o[at] = acc[i];
          }
          at += 128;
          if (whole && ++head == G) head = 0, at += static_cast<int64_t>(p.Hq - G) * 128;
        }
      }
      if (!whole && threadIdx.x == 0) {
        const int u = x.j0 == 0 ? x.u + TK_ITEM_UNITS : x.u - x.j0;  // of the item's first tile
        // (exact: the quotient is a whole number or at least 2^-31 from one)
        auto worker_of = [&](int unit) { return static_cast<int>((static_cast<double>(unit + 1ll) * st->start.workers - 1.0) / st->start.U); };
        st->shared[st->n_shared++] = TkShared{worker_of(u), worker_of(u + x.tiles - 1), x.b, x.h, x.it, x.row0, x.n};
      }
      turn = next_turn;
      more = y.j1 > y.j0;
      pq::tc_fence_before();
      all_sync();  // sums and references are used again, and the groups' O is written again
      if (lane == 0) {
        if (has_prefix) pq::mbar_arrive(&st->pre_empty);
        pq::mbar_arrive(&st->q_empty[n_items & 1]);  // (nobody looks at the item any more)
      }
    }
    // ---- the last of the workers w0 .. w1 of a shared item to come here merges their partials, in that order
    if (!ok && lane == 0) give_up();
    all_sync();
    if (st->n_shared > 0) {
      __threadfence();
      all_sync();
      if (threadIdx.x < 2) {
        const bool go = !st->abort_flag && static_cast<int>(threadIdx.x) < st->n_shared;  // (its first item and its last)
        const TkShared sh = st->shared[threadIdx.x];
        st->merge[threadIdx.x] = go && atomicAdd(p.tickets + TK_TICKET0 + sh.w0, 1u) == static_cast<uint32_t>(sh.w1 - sh.w0) ? 1 : 0;
      }
      all_sync();
      __threadfence();
      for (int i = 0; i < 2; ++i) {
        if (!st->merge[i]) continue;
        const TkShared sh = st->shared[i];
        const int t0 = sh.it * TI, cols = min(TI, sh.n - t0) * G;
        for (int col = warp; col < cols; col += TK_SOFTMAX_WARPS) {
          float m = -INFINITY, sum = 0.0f;
          float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          for (int w0 = sh.w0; w0 <= sh.w1; w0 += 32) {  // a lane per partial for the weights, then the partials in turn
            const int nw = min(32, sh.w1 - w0 + 1);
            auto slot_of = [&](int w) { return (2 * static_cast<int64_t>(w) + (w == sh.w0 ? 1 : 0)) * NC + col; };
            const float2 ml = lane < nw ? __ldcg(reinterpret_cast<const float2*>(p.ws_ml) + slot_of(w0 + lane)) : make_float2(-INFINITY, 0.0f);
            float4 o[4];  // the first partials are on their way while the weights are formed
            auto load = [&](int i) { return i < nw ? __ldcg(reinterpret_cast<const float4*>(p.ws_o + slot_of(w0 + i) * 128) + lane) : make_float4(0.0f, 0.0f, 0.0f, 0.0f); };
  #pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = load(i);
            float mc = ml.x;
  #pragma unroll
            for (int d = 1; d < 32; d <<= 1) mc = fmaxf(mc, __shfl_xor_sync(0xffffffffu, mc, d));
            const float mn = fmaxf(m, mc), keep = m == -INFINITY ? 0.0f : pq::ex2_approx(m - mn);
            const float w = ml.x == -INFINITY ? 0.0f : pq::ex2_approx(ml.x - mn);
            float lw = ml.y != ml.y ? ml.y : ml.x == -INFINITY ? 0.0f : DYN ? pq::at_reference(ml.y, ml.x - mn) : ml.y * w;
  #pragma unroll
            for (int d = 1; d < 32; d <<= 1) lw += __shfl_xor_sync(0xffffffffu, lw, d);
            sum = (m == -INFINITY ? 0.0f : DYN ? pq::at_reference(sum, m - mn) : sum * keep) + lw;
            m = mn;
            acc.x *= keep, acc.y *= keep, acc.z *= keep, acc.w *= keep;
            for (int i0 = 0; i0 < nw; i0 += 4) {
  #pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float wi = __shfl_sync(0xffffffffu, w, (i0 + i) & 31);
                acc.x = fmaf(o[i].x, wi, acc.x), acc.y = fmaf(o[i].y, wi, acc.y), acc.z = fmaf(o[i].z, wi, acc.z), acc.w = fmaf(o[i].w, wi, acc.w);
                o[i] = load(i0 + 4 + i);
              }
            }
          }
          const float norm = sum > 0.0f ? 1.0f / sum : sum == sum ? 0.0f : sum;
          const int tok = col / G;
          *reinterpret_cast<uint2*>(p.out + (static_cast<int64_t>(sh.row0 + t0 + tok) * p.Hq + sh.h * G + (col - tok * G)) * 128 + 4 * lane) =
              pack_bf16x4(make_float4(acc.x * norm, acc.y * norm, acc.z * norm, acc.w * norm));
        }
        if (threadIdx.x == 0) p.tickets[TK_TICKET0 + sh.w0] = 0;
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::REGS_OTHERS));
    if (warp < Sh::WARP_QK) {
      // ================================================================== expansion: keys of a tile, then values of the tile before
      const int quad = warp & 3;
      const uint32_t k_dst = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + Sh::COL_K, v_dst = k_dst + (Sh::COL_V - Sh::COL_K);
      // keys: this lane's row. values: this lane gives the address of a row of every 32 keys.
      const int page = 1 << p.page_log2;
      auto row_off = [&](int key) { return static_cast<uint32_t>(((key >> p.page_log2) << (p.page_log2 + 7)) + ((key & (page - 1)) << 6)); };
      const uint32_t land0 = pq::smem_u32(land);
      const uint32_t k_row = row_off(quad * 32 + lane), k_turn = ((k_row >> 7) & 3) << 4;
      uint32_t v_off[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v_off[i] = land0 + land_off(row_off(i * 32 + lane) + (page << 6), quad);
      bool ok = true;
      int slot = 0, slot_phase = 0, v_slot = 0;
      // (static steps: rolled loops keep the code small, 64 x 8 rows at 6000 keys 151 -> 140 us; own steps: unrolled ones are faster, 175 -> 166 in the case above)
      for (int c = 0;; ++c) {
        if (!wait_both(&st->land_full[slot], slot_phase, &st->k_empty, (c & 1) ^ 1)) {
          ok = false;
          break;
        }
        const bool last = c == st->n_tiles;  // (the loader's word that this was all)
        if (!last) {
          pq::tc_fence_after();
          const uint32_t at = land0 + slot * TK_LAND_CODES + k_row;
#pragma unroll (DYN ? 4 : 1)
          for (int i = 0; i < 4; ++i) {  // 32 head dims
            const uint4 w = pq::lds128(at + ((i << 4) ^ k_turn));
            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint4 e = expand8_bf16(ww[2 * j]), f = expand8_bf16(ww[2 * j + 1]);
              const uint32_t r[8] = {e.x, e.y, e.z, e.w, f.x, f.y, f.z, f.w};
              tmem_st_cols(k_dst + 16 * i + 8 * j, r);
            }
          }
          pq::tmem_st_wait();
          pq::tc_fence_before();
          __syncwarp();
          if (lane == 0) pq::mbar_arrive(&st->k_full);
          if (++slot == LANDS) slot = 0, slot_phase ^= 1;
        }
        if (c > 0) {
          if (!wait_warp(&st->v_empty, c & 1)) {
            ok = false;
            break;
          }
          pq::tc_fence_after();
          const uint32_t at = v_slot * TK_LAND_CODES;
          uint32_t w[2][4];
          ldmatrix_x4_trans(v_off[0] + at, w[0]);
#pragma unroll (DYN ? 4 : 2)
          for (int i = 0; i < 4; ++i) {  // 32 keys, the next ones' rows on their way
            if (i < 3) ldmatrix_x4_trans(v_off[i + 1] + at, w[(i + 1) & 1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {  // dims 4g, 4g + 1 (lanes 0 .. 15), dims 4g + 2, 4g + 3
              uint32_t r[8];
#pragma unroll
              for (int n = 0; n < 4; ++n) {
                const uint2 e = expand2_f16(j ? w[i & 1][n] >> 8 : w[i & 1][n]);
                r[2 * n] = e.x, r[2 * n + 1] = e.y;
              }
              tmem_st_frag8(v_dst + (static_cast<uint32_t>(16 * j) << 16) + 16 * i, r);
            }
          }
          pq::tmem_st_wait();
          pq::tc_fence_before();
          __syncwarp();
          if (lane == 0) pq::mbar_arrive(&st->v_full), pq::mbar_arrive(&st->land_empty[v_slot]);
          if (++v_slot == LANDS) v_slot = 0;
        }
        if (last) break;
      }
      if (!ok && lane == 0) give_up();
    } else if (warp == Sh::WARP_LOAD) {
      // ================================================================== loader: lanes 0 .. 7 the pages of a tile
      const int pages = TK_KEYS >> p.page_log2, page = 1 << p.page_log2, pg = lane & 7;
      const bool leader = pq::elect_one();
      bool ok = true;
      int slot = 0, slot_phase = 1;
      TkItem x;
      if (any) x = first_item();
      for (bool more = any; more && ok; more = next_item(x)) {
        const int32_t* table = p.table + static_cast<int64_t>(x.b) * p.max_pages;
        auto wanted = [&](int jt) {  // is page pg of the tile one with keys that some row sees
          const int key = key_of(x, jt) + (pg << p.page_log2);
          return pg < pages && key < x.len && (key + page > x.lo || key < p.n_sink);
        };
        // page ids of four tiles at a time, eight lanes to a tile, requested four tiles ahead
        auto request = [&](int jt) {
          const int mine = jt + (lane >> 3);
          return mine < x.j1 && wanted(mine) ? pq::ld_dep(table + (key_of(x, mine) >> p.page_log2) + pg) : 0;
        };
        int ids = request(x.j0), ahead = 0;
        for (int jt = x.j0; jt < x.j1; ++jt) {
          const int in4 = (jt - x.j0) & 3;
          if (in4 == 0) {
            if (jt > x.j0) ids = ahead;
            ahead = request(jt + 4);
          }
          int id = __shfl_sync(0xffffffffu, ids, in4 * 8 + pg);
          const bool mine = wanted(jt) && lane < 8;
          if (mine && static_cast<uint32_t>(id) >= static_cast<uint32_t>(p.n_pages)) {  // an id that is none is reported and page 0 read in its place
            pq::report(p.status, PQ_ERR_SHAPE);
            id = 0;
          }
          const uint32_t copies = __ballot_sync(0xffffffffu, mine);
          if (!wait_warp(&st->land_empty[slot], slot_phase)) {
            ok = false;
            break;
          }
          const int row = id * p.Hkv + x.h;
          if (leader) pq::mbar_arrive_expect_tx(&st->land_full[slot], __popc(copies) * page * 128);
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 8; ++i) {  // (a lane at a time would take three times as long)
            if (i >= pages) break;
            const int row_i = __shfl_sync(0xffffffffu, row, i);
            if (leader && ((copies >> i) & 1)) tma_load_3d(pq::smem_u32(land + slot * TK_LAND_CODES) + i * page * 128, &map, 0, 0, row_i, &st->land_full[slot]);
          }
          if (DYN) {  // own steps, 16 bytes to a lane and copy
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int piece = (e * 32 + lane) * 4, of_page = piece >> (p.page_log2 + 1);  // (floats)
              const int page_id = __shfl_sync(0xffffffffu, mine ? id : -1, of_page);
              if (page_id >= 0)
                cp_async_16(pq::smem_u32(land_steps + slot * TK_LAND_STEPS) + piece * 4,
                            p.steps + ((static_cast<int64_t>(page_id) * p.Hkv + x.h) << (p.page_log2 + 1)) + (piece & ((2 << p.page_log2) - 1)));
            }
            cp_async_arrive(&st->land_full[slot]);
          }
          ++lands_issued;
          if (++slot == LANDS) slot = 0, slot_phase ^= 1;
        }
      }
      if (ok) ok = wait_warp(&st->land_empty[slot], slot_phase);
      if (ok && lane == 0) {  // one slot more, with nothing in it: that was all
        st->n_tiles = lands_issued;
        __threadfence_block();
        for (int i = 0; i < (DYN ? 33 : 1); ++i) pq::mbar_arrive(&st->land_full[slot]);
      }
      said_all = ok;
      if (!ok && lane == 0) give_up();
    } else if (warp == Sh::WARP_QK || warp == Sh::WARP_PV) {
      // ================================================================== MMA issuers, a warp for each product: the whole warp runs the loop, the elected lane issues
      constexpr uint32_t IDESC_S = idesc_16(128, NC, true, false), IDESC_O = idesc_16(128, NC, false, true);
      const bool leader = pq::elect_one(), scores = warp == Sh::WARP_QK;
      bool ok = true;
      int buf = 0, phase = 0, tile_phase = 0, item = 0, group = 0;
      TkItem x;
      if (any) x = first_item();
      for (bool more = any; more && ok; more = next_item(x), ++item) {
        const int n_tiles = x.j1 - x.j0;
        if (scores && !wait_warp(&st->q_full[item & 1], (item >> 1) & 1)) {
          ok = false;
          break;
        }
        for (int i = 0; i < n_tiles; ++i) {
          if (scores) {
            if (!wait_both(&st->s_empty[buf], phase ^ 1, &st->k_full, tile_phase)) {
              ok = false;
              break;
            }
            pq::tc_fence_after();
            if (leader) {
              const uint64_t q_desc = desc_sw128(pq::smem_u32(q_buf), 16) + (item & 1) * (NC * 256 >> 4);
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)  // 16 head dims per instruction
                mma_ts(tmem_base + buf * NC, tmem_base + Sh::COL_K + kk * 8, q_desc + (((kk >> 2) * NC * 128 + (kk & 3) * 32) >> 4), IDESC_S, kk ? 1u : 0u);
              pq::mma_commit(&st->s_full[buf]);
              pq::mma_commit(&st->k_empty);
              if (i + 1 == n_tiles) pq::mma_commit(&st->q_empty[item & 1]);
            }
          } else {
            if (!wait_both(&st->v_full, tile_phase, &st->p_full[buf], phase)) {
              ok = false;
              break;
            }
            pq::tc_fence_after();
            if (leader) {
              const uint64_t p_desc = desc_p(pq::smem_u32(p_buf), NC < 64) + buf * (Sh::P_BYTES >> 4);
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)  // 16 keys per instruction
                mma_ts(tmem_base + Sh::COL_O + group * NC, tmem_base + Sh::COL_V + kk * 8, p_desc + (kk * 16 * Sh::P_ROW >> 4), IDESC_O, (i >= T || kk > 0) ? 1u : 0u);
              pq::mma_commit(&st->pv_done[buf]);
              pq::mma_commit(&st->v_empty);
            }
            if (++group == T) group = 0;
          }
          __syncwarp();
          if (++buf == NB) buf = 0, phase ^= 1;
          tile_phase ^= 1;
        }
      }
      if (leader) {
        if (!ok) give_up();
        pq::mma_commit(&st->drain[scores ? 0 : 1]);  // whatever was issued has finished before tensor memory is released or shared memory given back
      }
      __syncwarp();
      pq::mbar_wait(&st->drain[scores ? 0 : 1], 0);
    } else if (warp == Sh::WARP_HELP) {
      // ================================================================== helper: queries of the items behind the first, prefix scores of all
      bool ok = true;
      int n_pre = 0;
      TkItem x;
      if (any) x = first_item();
      bool more = any;
      for (int item = 0; any; more = next_item(x), ++item) {
        const int buf = item & 1;
        if (item > 0) {
          if (!wait_warp(&st->q_empty[buf], ((item >> 1) & 1) ^ 1)) {
            ok = false;
            break;
          }
          if (more) load_queries(x, buf, lane, 32, std::integral_constant<int, 4>());
          if (lane == 0) {
            if (!more) x.j1 = x.j0;  // (no more)
            st->item[buf] = x;
          }
          __syncwarp();
          if (lane == 0) pq::mbar_arrive(&st->q_full[buf]);
          if (!more) break;
        }
        if (x.j0 == 0 && p.n_prefix > 0) {
          if ((item == 0 && !wait_warp(&st->q_full[0], 0)) || !wait_warp(&st->pre_empty, (n_pre & 1) ^ 1)) {
            ok = false;
            break;
          }
          ++n_pre;
          prefix_scores(x, buf);
          __syncwarp();
          if (lane == 0) pq::mbar_arrive(&st->pre_full);
        }
      }
      if (!ok && lane == 0) give_up();
    }
  }

  pq::tc_fence_before();
  __syncthreads();
  if (warp == Sh::WARP_LOAD && lane == 0 && st->abort_flag) {
    // Copies that nobody consumed must have landed before the CTA may exit. The slot with the loader's word has gone on by a phase, in which it has the parity that would be
    // waited for; its copies have been read (the loader waited for that before it gave its word).
    for (int c = max(0, lands_issued - LANDS + (said_all ? 1 : 0)); c < lands_issued; ++c) pq::mbar_wait(&st->land_full[c % LANDS], (c / LANDS) & 1);
  }
  __syncthreads();
  if (warp == Sh::WARP_QK) {
    pq::tc_fence_after();
    pq::tmem_dealloc(tmem_base, Sh::TMEM_COLS);
  }
}

using TkKernel = void (*)(const CUtensorMap, const PagedAttnParams);
struct TkForm {
  TkKernel kern;
  int nc, ctas, threads;
  size_t smem, smem_most;  // of this prefix, and the most that any call takes
};
template <int NC, bool POLL>
TkForm form(bool dyn, int n_prefix) {
  return {dyn ? paged_tree_kernel<NC, true, POLL> : paged_tree_kernel<NC, false, POLL>, NC, pq_tree::ctas_of_sm(NC, dyn, n_prefix), TkShape<NC>::THREADS, tk_smem_bytes<NC>(dyn, n_prefix),
          tk_smem_bytes<NC>(dyn, PQ_PAGED_MAX_PREFIX)};
}
// Short wait limits take the polling form, of 128 columns whatever the rows.
TkForm form_of(const pq_ctx* ctx, const PagedAttnParams& p, int64_t max_len) {
  const bool dyn = p.steps != nullptr;
  if (p.wait_clocks < PQ_SUSPENDED_CLOCKS) return form<128, true>(dyn, p.n_prefix);
  const int columns = pq_tree::columns_of(dyn, p.n_prefix, ctx->sm_count, p.B, p.Hkv, p.G, p.max_new, max_len, p.window, p.n_sink);
  return columns == 32 ? form<32, false>(dyn, p.n_prefix) : columns == 64 ? form<64, false>(dyn, p.n_prefix) : form<128, false>(dyn, p.n_prefix);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

}  // namespace

size_t pq_paged_tree_ws_bytes(const pq_ctx* ctx) { return static_cast<size_t>(2) * ctx->sm_count * 128 * (128 + 2) * sizeof(float); }

pq_status pq_paged_tree_launch(pq_ctx* ctx, PagedAttnParams p, int64_t max_len, void* ws, cudaStream_t st) {
  const bool dyn = p.steps != nullptr, poll = p.wait_clocks < PQ_SUSPENDED_CLOCKS;
  const TkForm f = form_of(ctx, p, max_len);
  if (ctx->device < 0 || ctx->device >= 64 || 2 * ctx->sm_count > PQ_PAGED_MAX_WORKERS) return PQ_ERR_UNSUPPORTED;
  static std::atomic<bool> attr_set[64][2][4] = {};  // the largest there is, once per device and kernel
  std::atomic<bool>& set = attr_set[ctx->device][dyn][poll ? 3 : f.nc >> 6];
  if (!set.load(std::memory_order_relaxed)) {
    if (cudaFuncSetAttribute(f.kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(f.smem_most)) != cudaSuccess ||
        cudaFuncSetAttribute(f.kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess) {
      cudaGetLastError();
      return PQ_ERR_CUDA;
    }
    set.store(true, std::memory_order_relaxed);
  }
  // [page and head][K rows, V rows][64 bytes]; without pages nothing is ever copied
  const int64_t heads = static_cast<int64_t>(p.n_pages) * p.Hkv;
  if (heads > 0x7fffffffll) return PQ_ERR_SHAPE;  // (more than any device's memory)
  const cuuint32_t rows = 2u << p.page_log2;
  const cuuint64_t dims[3] = {64, rows, static_cast<cuuint64_t>(heads > 0 ? heads : 1)}, strides[2] = {64, rows * 64ull};
  const cuuint32_t box[3] = {64, rows, 1}, one[3] = {1, 1, 1};
  CUtensorMap map;
  const void* base = heads > 0 ? static_cast<const void*>(p.codes) : ws;
  if (reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, one,
                                                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return PQ_ERR_CUDA;
  p.ws_o = static_cast<float*>(ws);
  const int grid = f.ctas * ctx->sm_count;
  p.ws_ml = p.ws_o + static_cast<size_t>(2) * grid * f.nc * 128;
  return pq_launch_pdl(f.kern, dim3(grid), f.threads, f.smem, st, map, p);
}
