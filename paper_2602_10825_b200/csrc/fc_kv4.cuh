// The 4-bit row format (see fc.h): helpers shared by the kernels that write it, read it and attend over it.
#pragma once

#include "fc_common.cuh"

namespace fc {

constexpr int kKv4Group = 32;  // elements that share a scale

// One store as a kernel sees it (K and V share strides).
struct Kv4View {
  const uint8_t *k_codes, *v_codes;
  const uint16_t *k_scales, *v_scales;  // bf16 bits
  int64_t code_hs, code_rs, scale_hs, scale_rs;
};

inline Kv4View kv4_view(const fc_kv4_cache& c) {
  return {(const uint8_t*)c.k_codes, (const uint8_t*)c.v_codes, (const uint16_t*)c.k_scales, (const uint16_t*)c.v_scales,
          c.code_hs, c.code_rs, c.scale_hs, c.scale_rs};
}

// Host check of a store of H heads: FC_OK or the error a call returns.
inline int kv4_check(const fc_kv4_cache* c, int d, int64_t rows_needed) {
  if (!c || !c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales) return FC_ERR_INVALID_ARG;
  if (c->rows < rows_needed) return FC_ERR_INVALID_ARG;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return FC_ERR_MISALIGNED;
  if (((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) % (d / kKv4Group * 2)) return FC_ERR_MISALIGNED;
  if (c->code_hs < 0 || c->code_rs < 0 || c->code_hs % 16 || c->code_rs % 16) return FC_ERR_MISALIGNED;
  const int groups = d / kKv4Group;
  if (c->scale_hs < 0 || c->scale_rs < 0 || c->scale_hs % groups || c->scale_rs % groups) return FC_ERR_MISALIGNED;
  if (c->code_rs < d / 2 || c->scale_rs < groups) return FC_ERR_INVALID_ARG;
  return FC_OK;
}

__device__ __forceinline__ uint32_t hfma2_bf16(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}

// (w & mask) | magic in one instruction
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t magic) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w), "r"(mask), "r"(magic));
  return d;
}

// Code i (0..3) of both halves of a word as a pair of bf16 numbers 16 + code: the code goes to the top four bits of a
// mantissa whose exponent says 16.  With the scale s, (16 + code) s - 24 s = (code - 8) s in one rounding-free fma: 24 s
// has two bits more than s, and the result at most eight.
template <int I>
__device__ __forceinline__ uint32_t kv4_pair16(uint32_t w) {
  const uint32_t x = I == 0 ? w << 3 : w >> (4 * I - 3);
  return and_or(x, 0x00780078u, 0x41804180u);
}

// The scale, and -24 times it, in both halves of a register.
__device__ __forceinline__ uint32_t kv4_scale2(uint32_t s16) { return s16 | (s16 << 16); }
__device__ __forceinline__ uint32_t kv4_bias2(uint32_t s2) {
  return hfma2_bf16(s2, 0xC1C0C1C0u, 0x80008000u);  // s * -24 + (-0)
}

// Eight values of one word as four bf16 pairs, in the order of the elements.
__device__ __forceinline__ void kv4_word(uint32_t w, uint32_t s2, uint32_t b2, uint32_t (&out)[4]) {
  out[0] = hfma2_bf16(kv4_pair16<0>(w), s2, b2);
  out[1] = hfma2_bf16(kv4_pair16<1>(w), s2, b2);
  out[2] = hfma2_bf16(kv4_pair16<2>(w), s2, b2);
  out[3] = hfma2_bf16(kv4_pair16<3>(w), s2, b2);
}

// Unpacks rows [row0, row0 + n) of K and V into [H, n, d] tensors (fc_kv4.cu); either destination may be NULL.  `clear`: a word that
// is set to zero on the way, or NULL.  A kernel launched by launch_pdl behind it may start early.
int kv4_unpack_launch(cudaStream_t st, const Kv4View& src, int H, int d, int64_t row0, int n, void* K_dst, void* V_dst, int dtype,
                      int64_t k_hs, int64_t k_rs, int64_t v_hs, int64_t v_rs, uint32_t* clear);

}  // namespace fc
