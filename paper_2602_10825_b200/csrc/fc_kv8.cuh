// The paged 8-bit store (see fc.h): helpers shared by the kernels that write it, read it and attend over it.
#pragma once

#include "fc_common.cuh"

namespace fc {

constexpr int kMaxPages = INT32_MAX - 8192;  // counters of pages run past the end by a tile

// A pool as a kernel sees it (K and V share strides).
struct Kv8View {
  uint8_t *k_codes, *v_codes;
  float *k_scales, *v_scales;
  int64_t code_ps, code_hs, scale_ps, scale_hs;
  int32_t n_pages, page_log2;
};

inline int page_log2(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : -1; }

inline Kv8View kv8_view(const fc_kv8_pool& p) {
  return {(uint8_t*)p.k_codes, (uint8_t*)p.v_codes, p.k_scales, p.v_scales, p.code_ps, p.code_hs, p.scale_ps, p.scale_hs,
          p.n_pages, page_log2(p.page)};
}

// Whether n x m intervals of `width`, `a` and `b` apart, are disjoint: one of the axes walks over whole rows of the other.
inline bool grid_disjoint(int64_t n, int64_t a, int64_t m, int64_t b, int64_t width) {
  using I = __int128;
  if (n <= 1 && m <= 1) return true;
  if (n <= 1) return b >= width;
  if (m <= 1) return a >= width;
  return (b >= width && (I)a >= (I)(m - 1) * b + width) || (a >= width && (I)b >= (I)(n - 1) * a + width);
}

// Host check of a pool of H heads: FC_OK or the error a call returns.
inline int kv8_check(const fc_kv8_pool* p, int H, int d) {
  if (!p || !p->k_codes || !p->v_codes || !p->k_scales || !p->v_scales) return FC_ERR_INVALID_ARG;
  if (p->n_pages <= 0) return FC_ERR_INVALID_ARG;
  if (p->n_pages > kMaxPages) return FC_ERR_UNSUPPORTED;
  if (page_log2(p->page) < 0) return FC_ERR_UNSUPPORTED;
  if (!aligned16(p->k_codes) || !aligned16(p->v_codes) || ((uintptr_t)p->k_scales | (uintptr_t)p->v_scales) % 4) return FC_ERR_MISALIGNED;
  if (p->code_ps < 0 || p->code_hs < 0 || p->code_ps % 16 || p->code_hs % 16) return FC_ERR_MISALIGNED;
  if (p->scale_ps < 0 || p->scale_hs < 0) return FC_ERR_INVALID_ARG;
  // what 32 bits hold in units of 16 bytes, and of a scale
  if (p->code_ps >= (1ll << 36) || p->code_hs >= (1ll << 36) || p->scale_ps > INT32_MAX || p->scale_hs > INT32_MAX) return FC_ERR_UNSUPPORTED;
  if (!grid_disjoint(p->n_pages, p->code_ps, H, p->code_hs, (int64_t)p->page * d)) return FC_ERR_INVALID_ARG;
  if (!grid_disjoint(p->n_pages, p->scale_ps, H, p->scale_hs, 1)) return FC_ERR_INVALID_ARG;
  return FC_OK;
}

// First byte of a block, and its scale: one multiplication each.
__device__ __forceinline__ uint8_t* kv8_block(uint8_t* codes, const Kv8View& p, int page, int h) {
  return reinterpret_cast<uint8_t*>(reinterpret_cast<uint4*>(codes) + (uint64_t)(uint32_t)page * (uint32_t)(p.code_ps >> 4) +
                                    (uint64_t)(uint32_t)h * (uint32_t)(p.code_hs >> 4));
}
__device__ __forceinline__ float* kv8_scale(float* scales, const Kv8View& p, int page, int h) {
  return scales + (uint64_t)(uint32_t)page * (uint32_t)p.scale_ps + (uint64_t)(uint32_t)h * (uint32_t)p.scale_hs;
}

// Two codes (the low 16 bits) as two fp16 numbers: exact.
__device__ __forceinline__ uint32_t e4m3_to_half2(uint16_t x) {
  uint32_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"(x));
  return y;
}
__device__ __forceinline__ uint32_t e4m3_lo2(uint32_t w) { return e4m3_to_half2((uint16_t)(w & 0xffffu)); }
__device__ __forceinline__ uint32_t e4m3_hi2(uint32_t w) { return e4m3_to_half2((uint16_t)(w >> 16)); }
__device__ __forceinline__ float half_lo(uint32_t w) {
  float y;
  asm("{.reg .b16 a, b; mov.b32 {a, b}, %1; cvt.f32.f16 %0, a;}" : "=f"(y) : "r"(w));
  return y;
}
__device__ __forceinline__ float half_hi(uint32_t w) {
  float y;
  asm("{.reg .b16 a, b; mov.b32 {a, b}, %1; cvt.f32.f16 %0, b;}" : "=f"(y) : "r"(w));
  return y;
}

// Tokens first .. first + n - 1 of row `seq` of the table become rows dst_row .. of the destination.
struct Kv8Job {
  int32_t seq, first, n, dst_row;
};
constexpr int kKv8Jobs = 3 * FC_MAX_CHUNKS;  // what lies between the ends of as many windows, and of as many ranges from token 0 on
struct Kv8Jobs {
  int32_t n;
  Kv8Job job[kKv8Jobs];
  // With a list of active chunks (DEVICE, as in fc_chunk_attention), only the jobs are done that one of them needs: bit c of needed[j].
  const int32_t *active_ids, *n_active;
  int32_t W;
  uint64_t needed[kKv8Jobs];
};
static_assert(FC_MAX_CHUNKS <= 64, "a bit a chunk");

// Unpacks jobs into [H, dst_rows, d] tensors (fc_kv8.cu); either destination may be NULL.  `clear`: a word that is set to zero on the
// way, or NULL.  A kernel launched by launch_pdl behind it may start early.
int kv8_unpack_launch(cudaStream_t st, const Kv8View& src, int H, int d, const int32_t* table, int64_t table_cs, const Kv8Jobs& jobs,
                      void* K_dst, void* V_dst, int64_t dst_rows, int dtype, int64_t k_hs, int64_t k_rs, int64_t v_hs, int64_t v_rs,
                      uint32_t* status, uint32_t* clear);

}  // namespace fc
