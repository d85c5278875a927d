// Device helpers of the tcgen05 attention kernels over the paged 4-bit cache: codes to 16-bit operands, descriptors and instructions of kind::f16, tensor memory.
#pragma once

#include "pq_paged_attn.cuh"

namespace {

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
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

}  // namespace
