// What a paged cache holds in 4 bits, and how it becomes bf16 again.
//
// 32 channels of a token have one scale s, the nearest number of five significant bits to max|x| / 7, and each a code q = rint(x / s), -7 .. 7, held as
// u = q + 8.  q s has 3 + 5 = 8 significant bits: every value that the cache stands for IS a bf16 number.  So nothing is rounded behind the codes, whoever reads
// them (a copy as bf16, either attention kernel) works on the same values, and taking a value out is two instructions a pair: with u at the top of a bf16
// mantissa under the exponent of 16 the pair is 16 + u, and fma(16 + u, s, -24 s) is (u - 8) s, exactly, because -24 s has 2 + 5 bits and the result is a bf16.
// (With the codes at the bottom of the mantissa the constant is -136 s, 5 + 5 bits: it would be rounded.)
//
// A token's codes are words of eight channels; channel 2i of a word is at bits 4i, channel 2i + 1 at bits 16 + 4i: a shift and a mask make a pair of neighbours.
// Sixteen tokens keep their codes next to each other, 16 x d/2 bytes, and their scales behind these, 16 x d/32 bf16: what a warp of the attention takes at a
// time is one piece of memory (1152 bytes with 128 channels, 4.5 bits a value).
#pragma once
#include "avsa_common.cuh"

namespace avsa {

constexpr int kQ4Group = 32;       // channels of a scale
constexpr int kQ4Tokens = 16;      // tokens of a block
constexpr __host__ __device__ int q4_token_bytes(int d) { return d / 2 + d / 16; }
constexpr __host__ __device__ int q4_block_bytes(int d) { return kQ4Tokens * q4_token_bytes(d); }
constexpr __host__ __device__ int q4_scales_at(int d) { return kQ4Tokens * (d / 2); }      // in a block

// Groups whose largest magnitude is below 2^-100 are held as zeros, those with one of 2^125 or more, an infinity or a NaN as NaN: 1 / s and 24 s stay normal numbers.
constexpr uint32_t kQ4Least = (127 - 100) << 7, kQ4Most = (127 + 125) << 7;      // as bf16 bits

__device__ __forceinline__ uint32_t hfma2_bf16(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t hmul2_bf16(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// -24 times a pair of scales.
__device__ __forceinline__ uint32_t q4_offset(uint32_t s2) { return hmul2_bf16(s2, 0xc1c0c1c0u); }
// Pair i of a word: s2 the scales of its two values, c2 = q4_offset(s2).  `sixteen` is kQ4Sixteen, from a register that the compiler cannot see through: an instruction
// takes one constant, and mask and exponent are two (the stream kernel had 64 instructions more a block).
constexpr uint32_t kQ4Sixteen = 0x41804180u;
__device__ __forceinline__ uint32_t q4_pair(uint32_t word, int i, uint32_t s2, uint32_t c2, uint32_t sixteen) {
  const uint32_t at = i == 0 ? word << 3 : word >> (4 * i - 3);
  uint32_t x;
  asm("lop3.b32 %0, %1, 0x00780078, %2, 0xea;" : "=r"(x) : "r"(at), "r"(sixteen));
  return hfma2_bf16(x, s2, c2);
}

// A pool as the kernels see it.
struct Q4Pool {
  uint8_t* ptr;
  int64_t stride_page, stride_head;      // bytes
  uint32_t sixteen;
};
inline Q4Pool q4_pool(const avsa_q4_pool& p) { return Q4Pool{static_cast<uint8_t*>(p.ptr), p.stride_page, p.stride_head, kQ4Sixteen}; }

inline bool q4_pool_ok(const avsa_q4_pool& p, int pages, int Hkv, int page, int d) {
  const int64_t head = static_cast<int64_t>(page) * q4_token_bytes(d);
  if (p.ptr == nullptr || !aligned16(p.ptr)) return false;
  if (Hkv > 1 && (p.stride_head < head || p.stride_head % 16 != 0)) return false;
  if (pages > 1 && (p.stride_page < head || p.stride_page % 16 != 0)) return false;
  return true;
}

// The pages that the batch of an attention call reads (`own`: not only the beginning's), as bf16: of head h at ((p*Hkv + h)*page)*d of `k` and `v`, with p the page's number or
// (with p.s.places) its place.
struct PrefixParams;
int launch_widen(const PrefixParams& p, Q4Pool k4, Q4Pool v4, void* k, void* v, bool own, int d, cudaStream_t st);

}  // namespace avsa
