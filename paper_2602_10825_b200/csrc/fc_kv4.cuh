// The 4-bit row format (see fc.h): helpers shared by the kernels that write it, read it and attend over it.
#pragma once

#include <algorithm>

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

// Rows r < n of heads h < H, `width` bytes each from base + h hs + r rs on.
struct RowSet {
  uintptr_t base;
  int64_t hs, rs, width;  // bytes, not negative
  int64_t n;
  int32_t H;
};

// Whether two such sets, of the same number of heads, share a byte.  Exact where their strides are equal; otherwise whole heads
// (equal head strides) or whole sets are taken for contiguous.
inline bool rows_meet(RowSet a, RowSet b) {
  using I = __int128;  // strides are the caller's: no sum of them overflows here
  if (a.n <= 0 || b.n <= 0 || a.H <= 0) return false;
  if (a.H == 1) a.hs = b.hs = 0;
  if (a.n == 1) a.rs = b.rs;
  if (b.n == 1) b.rs = a.rs;
  const I off = (I)b.base - (I)a.base;  // of b's first row from a's
  const I a_head = (I)(a.n - 1) * a.rs + a.width, b_head = (I)(b.n - 1) * b.rs + b.width;
  const int64_t last = a.H - 1;
  constexpr I kAll = (I)1 << 62;  // no memory is that large: below, 64 bits do
  if (a_head > kAll || b_head > kAll || last * (I)a.hs > kAll || last * (I)b.hs > kAll) return true;
  if (off >= last * (I)a.hs + a_head || off + last * (I)b.hs + b_head <= 0) return false;
  if (a.hs != b.hs) return true;
  for (int64_t dh = -last; dh <= last; ++dh) {
    const I far = off + dh * (I)a.hs;  // of a head of b from a head of a
    if (far >= a_head || far + b_head <= 0) continue;
    if (a.rs != b.rs || a.rs == 0) return true;
    // a row of b starts x + dr rs behind a row of a, -a.n < dr < b.n, and they meet if that is above -b.width and below a.width
    const int64_t x = (int64_t)far, rs = a.rs, least = -b.width - x, most = a.width - x;  // least < dr rs < most
    int64_t lo = least / rs, hi = most / rs;
    while (lo * rs <= least) ++lo;
    while (hi * rs >= most) --hi;
    if (std::max(lo, 1 - a.n) <= std::min(hi, b.n - 1)) return true;
  }
  return false;
}

// Whether rows [a0, a0 + na) of one store and rows [b0, b0 + nb) of another share memory.
inline bool kv4_meet(const fc_kv4_cache& a, int64_t a0, int64_t na, const fc_kv4_cache& b, int64_t b0, int64_t nb, int H, int d) {
  auto sets = [&](const fc_kv4_cache& c, int64_t r0, int64_t n, RowSet (&out)[4]) {
    const void* p[4] = {c.k_codes, c.v_codes, c.k_scales, c.v_scales};
    for (int i = 0; i < 4; ++i) {
      const bool codes = i < 2;
      const int64_t hs = codes ? c.code_hs : 2 * c.scale_hs, rs = codes ? c.code_rs : 2 * c.scale_rs;
      out[i] = {(uintptr_t)p[i] + (uintptr_t)r0 * (uintptr_t)rs, hs, rs, codes ? d / 2 : d / kKv4Group * 2, n, H};
    }
  };
  RowSet x[4], y[4];
  sets(a, a0, na, x);
  sets(b, b0, nb, y);
  for (const RowSet& s : x)
    for (const RowSet& t : y)
      if (rows_meet(s, t)) return true;
  return false;
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
