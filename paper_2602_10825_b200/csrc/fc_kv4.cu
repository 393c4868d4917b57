// fc_kv4_pack and fc_kv4_unpack: rows into and out of the 4-bit store.
//
// Both are bound by HBM.  A thread owns one 32-bit word of codes, that is eight elements of a row: four threads share a
// scale, sixteen (eight) threads a row of 128 (64), so that a warp reads and writes whole sectors of every array.
// Quantising is exact: codes are round-half-even of the true quotient, whatever the type.
//   bf16 rows   x / s is either a tie or at least 2^-10 away from one (x has 8 significant bits, s 5); so x * (1/s), off by
//               2^-20 at most, rounded to a multiple of 2^-13 is exactly the tie where there is one, and on the right
//               side of it where there is none.
//   fp32 rows   the remainder x - n s of a first guess n is exact in fp32, and compared with s/2.
#include <climits>

#include "fc_kv4.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerThread = 4;  // rows whose loads are in flight together

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 v = fc::ld_stream16(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = fc::bf16_lo(w[i]);
    x[2 * i + 1] = fc::bf16_hi(w[i]);
  }
}

// round_half_even(x / s) in -7 .. 7 for a scale of five significant bits, r = 1 / s
template <typename T> __device__ __forceinline__ int quantise(float x, float s, float r);
template <> __device__ __forceinline__ int quantise<__nv_bfloat16>(float x, float s, float r) {
  float t = x * r;
  t = __fadd_rn(__fadd_rn(t, 1536.f), -1536.f);  // to a multiple of 2^-13
  return __float2int_rn(fminf(fmaxf(t, -7.f), 7.f));
}
template <> __device__ __forceinline__ int quantise<float>(float x, float s, float r) {
  float n = rintf(fminf(fmaxf(x * r, -7.f), 7.f));
  const float rest = fmaf(-n, s, x), half = 0.5f * s;
  const bool odd = ((int)n & 1) != 0;
  if (rest > half || (rest == half && odd)) n += 1.f;
  if (rest < -half || (rest == -half && odd)) n -= 1.f;
  return (int)fminf(fmaxf(n, -7.f), 7.f);
}

// The word of eight elements that this thread holds, and the scale of its group (the same in the group's four threads).
template <typename T>
__device__ __forceinline__ void pack8(const float (&x)[8], unsigned mask, uint32_t& word, uint32_t& scale, bool& bad) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(x[i]) & 0x7fffffffu);  // as integers, so that a NaN is the largest
  a = max(a, __shfl_xor_sync(mask, a, 1));
  a = max(a, __shfl_xor_sync(mask, a, 2));
  bad = a >= 0x7f800000u;
  float s = __uint_as_float((__float_as_uint(__fdiv_rn(__uint_as_float(a), 7.f)) + 0x7ffffu) & ~0x7ffffu);
  s = a == 0 ? 0.f : fminf(fmaxf(s, 0x1p-126f), 0x1p122f);
  const float r = a == 0 ? 0.f : __fdiv_rn(1.f, s);
  word = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    word |= (uint32_t)(quantise<T>(x[2 * i], s, r) + 8) << (4 * i);
    word |= (uint32_t)(quantise<T>(x[2 * i + 1], s, r) + 8) << (16 + 4 * i);
  }
  scale = __float_as_uint(s) >> 16;
  if (bad) {
    word = 0x88888888u;
    scale = 0x7fc0u;
  }
}

struct PackGeom {
  int32_t n_old, n_new, n_out;
  int64_t dst_row, k_hs, k_rs, v_hs, v_rs, kept_hs;
  fc::Kv4View old;
  uint8_t *k_codes, *v_codes;
  uint16_t *k_scales, *v_scales;
  int64_t code_hs, code_rs, scale_hs, scale_rs;
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
kv4_pack_kernel(const T* __restrict__ K, const T* __restrict__ V, const int32_t* __restrict__ kept,
                const __grid_constant__ PackGeom g, uint32_t* __restrict__ status) {
  constexpr int W = D / 8, R = kThreads / W;  // words per row, rows per block and step
  const int w = threadIdx.x % W, h = blockIdx.y;
  const unsigned mask = 0xfu << (threadIdx.x & 28);  // the four threads of a group
  bool bad = false, bad_index = false;
#pragma unroll
  for (int u = 0; u < kRowsPerThread; ++u) {
    const int64_t r = ((int64_t)blockIdx.x * kRowsPerThread + u) * R + threadIdx.x / W;
    if (r >= g.n_out) break;
    const int64_t i = kept ? kept[h * g.kept_hs + r] : r;
    if (i < 0 || i >= (int64_t)g.n_old + g.n_new) {
      bad_index = true;
      continue;
    }
    uint32_t word[2], scale[2];
    if (i < g.n_old) {
      const int64_t c = h * g.old.code_hs + i * g.old.code_rs + 4 * w, s = h * g.old.scale_hs + i * g.old.scale_rs + w / 4;
      word[0] = __ldg(reinterpret_cast<const uint32_t*>(g.old.k_codes + c));
      word[1] = __ldg(reinterpret_cast<const uint32_t*>(g.old.v_codes + c));
      scale[0] = __ldg(g.old.k_scales + s);
      scale[1] = __ldg(g.old.v_scales + s);
    } else {
      const int64_t j = i - g.n_old;
      float x[8], y[8];
      load8<T>(K + h * g.k_hs + j * g.k_rs + 8 * w, x);
      load8<T>(V + h * g.v_hs + j * g.v_rs + 8 * w, y);
      bool b;
      pack8<T>(x, mask, word[0], scale[0], b);
      bad |= b;
      pack8<T>(y, mask, word[1], scale[1], b);
      bad |= b;
    }
    const int64_t c = h * g.code_hs + (g.dst_row + r) * g.code_rs + 4 * w;
    *reinterpret_cast<uint32_t*>(g.k_codes + c) = word[0];
    *reinterpret_cast<uint32_t*>(g.v_codes + c) = word[1];
    if (w % 4 == 0) {
      const int64_t s = h * g.scale_hs + (g.dst_row + r) * g.scale_rs + w / 4;
      g.k_scales[s] = (uint16_t)scale[0];
      g.v_scales[s] = (uint16_t)scale[1];
    }
  }
  if (status) {
    if (bad) atomicOr(status, (uint32_t)FC_DEV_NONFINITE);
    if (bad_index) atomicOr(status, (uint32_t)FC_DEV_BAD_INDEX);
  }
}

struct UnpackGeom {
  int32_t n;
  int64_t row0, k_hs, k_rs, v_hs, v_rs;
  fc::Kv4View src;
};

__device__ __forceinline__ void store8(__nv_bfloat16* p, const uint32_t (&v)[4]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store8(float* p, const uint32_t (&v)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(fc::bf16_lo(v[0]), fc::bf16_hi(v[0]), fc::bf16_lo(v[1]), fc::bf16_hi(v[1]));
  *reinterpret_cast<float4*>(p + 4) = make_float4(fc::bf16_lo(v[2]), fc::bf16_hi(v[2]), fc::bf16_lo(v[3]), fc::bf16_hi(v[3]));
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
kv4_unpack_kernel(T* __restrict__ K, T* __restrict__ V, const __grid_constant__ UnpackGeom g) {
  constexpr int W = D / 8, R = kThreads / W;
  const int w = threadIdx.x % W, h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  T* dst = is_v ? V : K;
  if (!dst) return;
  const uint8_t* codes = is_v ? g.src.v_codes : g.src.k_codes;
  const uint16_t* scales = is_v ? g.src.v_scales : g.src.k_scales;
  const int64_t hs = is_v ? g.v_hs : g.k_hs, rs = is_v ? g.v_rs : g.k_rs;
  uint32_t word[kRowsPerThread], scale[kRowsPerThread];
  const int64_t r0 = (int64_t)blockIdx.x * kRowsPerThread * R + threadIdx.x / W;
#pragma unroll
  for (int u = 0; u < kRowsPerThread; ++u) {
    const int64_t r = r0 + u * R;
    if (r < g.n) {
      word[u] = __ldg(reinterpret_cast<const uint32_t*>(codes + h * g.src.code_hs + (g.row0 + r) * g.src.code_rs + 4 * w));
      scale[u] = __ldg(scales + h * g.src.scale_hs + (g.row0 + r) * g.src.scale_rs + w / 4);
    }
  }
#pragma unroll
  for (int u = 0; u < kRowsPerThread; ++u) {
    const int64_t r = r0 + u * R;
    if (r < g.n) {
      const uint32_t s2 = fc::kv4_scale2(scale[u]);
      uint32_t v[4];
      fc::kv4_word(word[u], s2, fc::kv4_bias2(s2), v);
      store8(dst + h * hs + r * rs + 8 * w, v);
    }
  }
}

int check_rows(const void* p, int d, int es, int64_t hs, int64_t rs) {
  if (!fc::aligned16(p)) return FC_ERR_MISALIGNED;
  if (hs < 0 || rs < 0 || (hs * es) % 16 || (rs * es) % 16) return FC_ERR_MISALIGNED;
  return rs < d ? FC_ERR_INVALID_ARG : FC_OK;
}

}  // namespace

namespace fc {

int kv4_unpack_launch(fc_ctx* ctx, cudaStream_t st, const Kv4View& src, int H, int d, int64_t row0, int n, void* K_dst, void* V_dst,
                      int dtype, int64_t k_hs, int64_t k_rs, int64_t v_hs, int64_t v_rs) {
  (void)ctx;
  if (n == 0 || (!K_dst && !V_dst)) return FC_OK;
  UnpackGeom g = {n, row0, k_hs, k_rs, v_hs, v_rs, src};
  const int rows = kRowsPerThread * kThreads / (d / 8);
  const dim3 grid((unsigned)((n + rows - 1) / rows), (unsigned)H, 2);
#define FC_UNPACK(T, D) kv4_unpack_kernel<T, D><<<grid, kThreads, 0, st>>>((T*)K_dst, (T*)V_dst, g)
  if (dtype == FC_F32) { if (d == 128) FC_UNPACK(float, 128); else FC_UNPACK(float, 64); }
  else { if (d == 128) FC_UNPACK(__nv_bfloat16, 128); else FC_UNPACK(__nv_bfloat16, 64); }
#undef FC_UNPACK
  FC_LAUNCH_CHECK("kv4_unpack_kernel");
  return FC_OK;
}

}  // namespace fc

extern "C" int fc_kv4_pack(fc_ctx* ctx, void* stream, const fc_kv4_pack_desc* desc, const void* K_src, const void* V_src, int dtype,
                           const fc_kv4_cache* old, const int32_t* kept_idx, int64_t kept_hs, const fc_kv4_cache* dst,
                           uint32_t* status) {
  if (!ctx || !desc) return FC_ERR_INVALID_ARG;
  if (dtype != FC_BF16 && dtype != FC_F32) return FC_ERR_UNSUPPORTED;
  if (desc->d != 64 && desc->d != 128) return FC_ERR_UNSUPPORTED;
  if (desc->H <= 0 || desc->n_old < 0 || desc->n_new < 0 || desc->n_out < 0 || desc->dst_row < 0) return FC_ERR_INVALID_ARG;
  if (desc->n_old > INT32_MAX - desc->n_new) return FC_ERR_INVALID_ARG;
  if (desc->H > 65535) return FC_ERR_UNSUPPORTED;
  if (desc->n_out == 0) return FC_OK;
  if (!dst || (desc->n_new > 0 && (!K_src || !V_src))) return FC_ERR_INVALID_ARG;
  if (!kept_idx && desc->n_out > desc->n_old + desc->n_new) return FC_ERR_INVALID_ARG;
  if (kept_idx && kept_hs < desc->n_out) return FC_ERR_INVALID_ARG;
  const int es = fc::elem_size(dtype);
  int rc;
  if (desc->n_new > 0) {
    if ((rc = check_rows(K_src, desc->d, es, desc->k_hs, desc->k_rs)) != FC_OK) return rc;
    if ((rc = check_rows(V_src, desc->d, es, desc->v_hs, desc->v_rs)) != FC_OK) return rc;
  }
  if (desc->n_old > 0 && (rc = fc::kv4_check(old, desc->d, desc->n_old)) != FC_OK) return rc;
  if (desc->dst_row > INT64_MAX - desc->n_out) return FC_ERR_INVALID_ARG;
  if ((rc = fc::kv4_check(dst, desc->d, desc->dst_row + desc->n_out)) != FC_OK) return rc;

  PackGeom g = {};
  g.n_old = desc->n_old; g.n_new = desc->n_new; g.n_out = desc->n_out; g.dst_row = desc->dst_row;
  g.k_hs = desc->k_hs; g.k_rs = desc->k_rs; g.v_hs = desc->v_hs; g.v_rs = desc->v_rs; g.kept_hs = kept_hs;
  if (desc->n_old > 0) g.old = fc::kv4_view(*old);
  g.k_codes = (uint8_t*)dst->k_codes; g.v_codes = (uint8_t*)dst->v_codes;
  g.k_scales = (uint16_t*)dst->k_scales; g.v_scales = (uint16_t*)dst->v_scales;
  g.code_hs = dst->code_hs; g.code_rs = dst->code_rs; g.scale_hs = dst->scale_hs; g.scale_rs = dst->scale_rs;
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
  const int rows = kRowsPerThread * kThreads / (desc->d / 8);
  const dim3 grid((unsigned)((desc->n_out + rows - 1) / rows), (unsigned)desc->H);
#define FC_PACK(T, D) kv4_pack_kernel<T, D><<<grid, kThreads, 0, st>>>((const T*)K_src, (const T*)V_src, kept_idx, g, status)
  if (dtype == FC_F32) { if (desc->d == 128) FC_PACK(float, 128); else FC_PACK(float, 64); }
  else { if (desc->d == 128) FC_PACK(__nv_bfloat16, 128); else FC_PACK(__nv_bfloat16, 64); }
#undef FC_PACK
  FC_LAUNCH_CHECK("kv4_pack_kernel");
  return FC_OK;
}

extern "C" int fc_kv4_unpack(fc_ctx* ctx, void* stream, const fc_kv4_unpack_desc* desc, const fc_kv4_cache* src, void* K_dst,
                             void* V_dst, int dtype) {
  if (!ctx || !desc) return FC_ERR_INVALID_ARG;
  if (dtype != FC_BF16 && dtype != FC_F32) return FC_ERR_UNSUPPORTED;
  if (desc->d != 64 && desc->d != 128) return FC_ERR_UNSUPPORTED;
  if (desc->H <= 0 || desc->n < 0 || desc->src_row < 0) return FC_ERR_INVALID_ARG;
  if (desc->H > 65535) return FC_ERR_UNSUPPORTED;
  if (desc->n == 0) return FC_OK;
  if (!K_dst && !V_dst) return FC_ERR_INVALID_ARG;
  const int es = fc::elem_size(dtype);
  int rc;
  if (desc->src_row > INT64_MAX - desc->n) return FC_ERR_INVALID_ARG;
  if ((rc = fc::kv4_check(src, desc->d, desc->src_row + desc->n)) != FC_OK) return rc;
  if (K_dst && (rc = check_rows(K_dst, desc->d, es, desc->k_hs, desc->k_rs)) != FC_OK) return rc;
  if (V_dst && (rc = check_rows(V_dst, desc->d, es, desc->v_hs, desc->v_rs)) != FC_OK) return rc;
  FC_DEVICE_GUARD(ctx);
  return fc::kv4_unpack_launch(ctx, (cudaStream_t)stream, fc::kv4_view(*src), desc->H, desc->d, desc->src_row, desc->n, K_dst,
                               V_dst, dtype, desc->k_hs, desc->k_rs, desc->v_hs, desc->v_rs);
}
