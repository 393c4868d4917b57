// fc_kv4_pack and fc_kv4_unpack: rows into and out of the 4-bit store.
//
// Unpacking and the copying of old rows are bound by HBM, new rows by the quantising.  Unpacking moves 2.56 bytes an element for bf16 and is
// four loads in flight and one store a word (6.3 TB/s; to fp32, 4.56 bytes and two stores, 4.8).  Packing has two halves, and a warp that owns 32 output rows of a head does them one after the other:
//   old rows   whole 16-byte pieces, eight rows (D = 128) to an access, all of the warp's loads in flight at once;
//   new rows   a thread owns one 32-bit word of codes, that is eight elements of a row; four threads share a scale,
//              sixteen (eight) threads a row of 128 (64), several rows' loads in flight.  4680 rows of 24 heads of 128 take 20.5 us
//              in a replayed graph (their bytes 11.2), in fp32 52.2 (20.0), with the ALU pipe 61 % and 80 % busy.
// Quantising is exact: codes are round-half-even of the true quotient, whatever the type.
//   bf16 rows   x / s is either a tie or at least 2^-10 away from one (x has 8 significant bits, s 5); so x * (1/s), off by
//               2^-20 at most, rounded to a multiple of 2^-13 is exactly the tie where there is one, and on the right
//               side of it where there is none.  Rounding is adding and subtracting a large number, two elements an
//               instruction; the codes of four elements are put together as digits of an fp32 number below 2^16.
//   fp32 rows   the remainder x - n s of a first guess n is exact in fp32, and compared with s/2.
#include <climits>

#include "fc_kv4.cuh"
#include "fc_tcgen05.cuh"

namespace {

using fc::sm100::add2;
using fc::sm100::fma2;
using fc::sm100::pack2;
using fc::sm100::unpack2;

constexpr int kThreads = 256;
constexpr int kRowsPerThread = 4;  // rows whose loads are in flight together

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {  // bf16 pairs; a NaN is the largest
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

__device__ __forceinline__ float reciprocal(float x) {  // to one unit
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Eight elements as they lie in memory.
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> { uint4 w; };
template <> struct Eight<float> { float4 a, b; };
__device__ __forceinline__ void load8(const __nv_bfloat16* p, Eight<__nv_bfloat16>& x) { x.w = fc::ld_stream16(p); }
__device__ __forceinline__ void load8(const float* p, Eight<float>& x) {
  x.a = *reinterpret_cast<const float4*>(p);
  x.b = *reinterpret_cast<const float4*>(p + 4);
}

// Bits of the largest magnitude; above those of infinity for a NaN.
__device__ __forceinline__ uint32_t largest(const Eight<__nv_bfloat16>& x) {
  constexpr uint32_t kAbs = 0x7fff7fffu;
  const uint32_t m = max2_nan(max2_nan(x.w.x & kAbs, x.w.y & kAbs), max2_nan(x.w.z & kAbs, x.w.w & kAbs));
  return max(m << 16, m & 0xffff0000u);
}
__device__ __forceinline__ uint32_t largest(const Eight<float>& x) {
  const float v[8] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y, x.b.z, x.b.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);  // as integers
  return m;
}

// The word of codes 8 + round_half_even(x / s) for a scale of five significant bits, r = 1 / s; |x / s| <= 7 unless `clip`.
__device__ __forceinline__ uint32_t codes8(const Eight<__nv_bfloat16>& x, float s, float r, bool clip) {
  (void)s;
  const uint64_t r2 = pack2(r, r), snap = pack2(1536.f, 1536.f), unsnap = pack2(-1536.f, -1536.f);
  const uint64_t magic = pack2(12582920.f, 12582920.f), unmagic = pack2(-12582912.f, -12582912.f);  // 1.5 2^23 (+ 8)
  const uint32_t w[4] = {x.w.x, x.w.y, x.w.z, x.w.w};
  uint64_t digits = 0;
#pragma unroll
  for (int i = 3; i >= 0; --i) {
    uint64_t t = mul2(pack2(fc::bf16_lo(w[i]), fc::bf16_hi(w[i])), r2);
    if (clip) {
      float a, b;
      unpack2(t, a, b);
      t = pack2(fminf(fmaxf(a, -7.f), 7.f), fminf(fmaxf(b, -7.f), 7.f));
    }
    t = add2(add2(t, snap), unsnap);
    t = add2(add2(t, magic), unmagic);
    digits = i == 3 ? t : fma2(digits, pack2(16.f, 16.f), t);
  }
  float even, odd;
  unpack2(digits, even, odd);
  return (uint32_t)even | ((uint32_t)odd << 16);
}
__device__ __forceinline__ uint32_t codes8(const Eight<float>& x, float s, float r, bool) {
  const float v[8] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y, x.b.z, x.b.w};
  const float half = 0.5f * s;
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float n = rintf(fminf(fmaxf(v[i] * r, -7.f), 7.f));
    const float rest = fmaf(-n, s, v[i]);
    const bool odd = ((int)n & 1) != 0;
    if (rest > half || (rest == half && odd)) n += 1.f;
    if (rest < -half || (rest == -half && odd)) n -= 1.f;
    word |= (uint32_t)((int)fminf(fmaxf(n, -7.f), 7.f) + 8) << (4 * (i / 2) + 16 * (i & 1));
  }
  return word;
}

// The word of eight elements that this thread holds, and the scale of its group (the same in the group's four threads).
template <typename T>
__device__ __forceinline__ void pack8(const Eight<T>& x, unsigned mask, uint32_t& word, uint32_t& scale, bool& bad) {
  uint32_t a = largest(x);
  a = max(a, __shfl_xor_sync(mask, a, 1));
  a = max(a, __shfl_xor_sync(mask, a, 2));
  // the least five-bit number that is not below a / 7: an upper bound of the quotient cut to five bits is it, or the one before
  const uint32_t low = __float_as_uint(__fmul_ru(__uint_as_float(a), 0x1.24924ap-3f)) & ~0x7ffffu;
  const float s_free = __uint_as_float(7.f * __uint_as_float(low) >= __uint_as_float(a) ? low : low + 0x80000u);
  const float s = a == 0 ? 0.f : fminf(fmaxf(s_free, 0x1p-126f), 0x1p122f);
  const float r = a == 0 ? 0.f : reciprocal(s);
  word = codes8(x, s, r, s_free > 0x1p122f);
  scale = __float_as_uint(s) >> 16;
  if (a >= 0x7f800000u) {
    bad = true;
    word = 0x88888888u;
    scale = 0x7fc0u;
  }
}

struct PackGeom {
  int32_t n_old, n_new, n_out, rows_per_warp;
  int64_t dst_row, k_hs, k_rs, v_hs, v_rs, kept_hs;
  fc::Kv4View old;
  uint8_t *k_codes, *v_codes;
  uint16_t *k_scales, *v_scales;
  int64_t code_hs, code_rs, scale_hs, scale_rs;
};

template <int B> struct Bytes;  // a row's scales
template <> struct Bytes<8> { using type = uint2; };
template <> struct Bytes<4> { using type = uint32_t; };

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 3)
kv4_pack_kernel(const T* __restrict__ K, const T* __restrict__ V, const int32_t* __restrict__ kept,
                const __grid_constant__ PackGeom g, uint32_t* __restrict__ status) {
  constexpr int kWarps = kThreads / 32;
  const int lane = threadIdx.x % 32, h = blockIdx.y;
  const int64_t r0 = ((int64_t)blockIdx.x * kWarps + threadIdx.x / 32) * g.rows_per_warp;
  if (r0 >= g.n_out) return;
  const int rows = (int)min((int64_t)g.rows_per_warp, g.n_out - r0);
  const int64_t n_in = (int64_t)g.n_old + g.n_new;

  // lane L knows where output row r0 + L comes from
  int64_t from = -1;
  if (lane < rows) from = kept ? kept[h * g.kept_hs + r0 + lane] : r0 + lane;
  const bool bad_index = lane < rows && (from < 0 || from >= n_in);
  const bool is_new = lane < rows && !bad_index && from >= g.n_old;
  const bool is_old = lane < rows && !bad_index && !is_new;
  const uint32_t news = __ballot_sync(0xffffffffu, is_new), olds = __ballot_sync(0xffffffffu, is_old);
  const int32_t index = (int32_t)(is_new ? from - g.n_old : from);
  const int64_t code_out = h * g.code_hs + (g.dst_row + r0) * g.code_rs, scale_out = h * g.scale_hs + (g.dst_row + r0) * g.scale_rs;

  if (olds) {
    constexpr int kLanes = D / 32, kAt = 32 / kLanes, kIter = 32 / kAt;  // lanes of a row's codes, rows at once, accesses
    using S = typename Bytes<D / 16>::type;
    uint4 k[kIter], v[kIter];
    S s[kIter];
    const int piece = lane % kLanes;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int r = i * kAt + lane / kLanes;
      const int64_t src = __shfl_sync(0xffffffffu, index, r);
      if (!(olds >> r & 1)) continue;
      const int64_t c = h * g.old.code_hs + src * g.old.code_rs + 16 * piece;
      k[i] = fc::ld_stream16(g.old.k_codes + c);
      v[i] = fc::ld_stream16(g.old.v_codes + c);
      if (piece < 2) s[i] = __ldg(reinterpret_cast<const S*>((piece ? g.old.v_scales : g.old.k_scales) + h * g.old.scale_hs + src * g.old.scale_rs));
    }
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int r = i * kAt + lane / kLanes;
      if (!(olds >> r & 1)) continue;
      const int64_t c = code_out + r * g.code_rs + 16 * piece;
      *reinterpret_cast<uint4*>(g.k_codes + c) = k[i];
      *reinterpret_cast<uint4*>(g.v_codes + c) = v[i];
      if (piece < 2) *reinterpret_cast<S*>((piece ? g.v_scales : g.k_scales) + scale_out + r * g.scale_rs) = s[i];
    }
  }

  bool bad = false;
  if (news) {
    constexpr int W = D / 8, kAt = 32 / W, kUnroll = 4 / (int)sizeof(T) * 2;  // words of a row, rows at once, accesses in flight
    __shared__ uint8_t list_s[kWarps][32];
    uint8_t* list = list_s[threadIdx.x / 32];
    if (is_new) list[__popc(news & ((1u << lane) - 1u))] = (uint8_t)lane;
    __syncwarp();
    const int w = lane % W, n = __popc(news);
    const unsigned mask = 0xfu << (lane & 28);  // the four threads of a group
    for (int j0 = lane / W; j0 - lane / W < n; j0 += kUnroll * kAt) {
      Eight<T> x[kUnroll], y[kUnroll];
      int row[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int j = j0 + u * kAt;
        row[u] = list[min(j, n - 1)];
        const int64_t src = __shfl_sync(0xffffffffu, index, row[u]);
        if (j < n) {
          load8(K + h * g.k_hs + src * g.k_rs + 8 * w, x[u]);
          load8(V + h * g.v_hs + src * g.v_rs + 8 * w, y[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (j0 + u * kAt >= n) break;
        uint32_t word[2], scale[2];
        pack8<T>(x[u], mask, word[0], scale[0], bad);
        pack8<T>(y[u], mask, word[1], scale[1], bad);
        const int64_t c = code_out + row[u] * g.code_rs + 4 * w, s = scale_out + row[u] * g.scale_rs + w / 4;
        *reinterpret_cast<uint32_t*>(g.k_codes + c) = word[0];
        *reinterpret_cast<uint32_t*>(g.v_codes + c) = word[1];
        if (w % 4 == 0) {
          g.k_scales[s] = (uint16_t)scale[0];
          g.v_scales[s] = (uint16_t)scale[1];
        }
      }
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
  uint32_t* clear;
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
  fc::pdl_launch_dependents();
  const int w = threadIdx.x % W, h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  if (g.clear && threadIdx.x == 0 && blockIdx.x == 0 && h == 0 && !is_v) *g.clear = 0;
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

int kv4_unpack_launch(cudaStream_t st, const Kv4View& src, int H, int d, int64_t row0, int n, void* K_dst, void* V_dst, int dtype,
                      int64_t k_hs, int64_t k_rs, int64_t v_hs, int64_t v_rs, uint32_t* clear) {
  if (n == 0 || (!K_dst && !V_dst)) return FC_OK;
  UnpackGeom g = {n, row0, k_hs, k_rs, v_hs, v_rs, src, clear};
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
  if (desc->n_old > 0 && fc::kv4_meet(*old, 0, desc->n_old, *dst, desc->dst_row, desc->n_out, desc->H, desc->d))
    return FC_ERR_INVALID_ARG;  // rows would be read and written at once
  if (desc->H > 1 && (dst->code_hs < desc->d / 2 || dst->scale_hs < desc->d / fc::kKv4Group)) return FC_ERR_INVALID_ARG;  // overlap

  PackGeom g = {};
  g.n_old = desc->n_old; g.n_new = desc->n_new; g.n_out = desc->n_out; g.dst_row = desc->dst_row;
  g.k_hs = desc->k_hs; g.k_rs = desc->k_rs; g.v_hs = desc->v_hs; g.v_rs = desc->v_rs; g.kept_hs = kept_hs;
  if (desc->n_old > 0) g.old = fc::kv4_view(*old);
  g.k_codes = (uint8_t*)dst->k_codes; g.v_codes = (uint8_t*)dst->v_codes;
  g.k_scales = (uint16_t*)dst->k_scales; g.v_scales = (uint16_t*)dst->v_scales;
  g.code_hs = dst->code_hs; g.code_rs = dst->code_rs; g.scale_hs = dst->scale_hs; g.scale_rs = dst->scale_rs;
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
  // 32 rows a warp, fewer where that would leave the device with less than 32 warps an SM (4680 new rows of 24 heads: 24 us
  // with 16 rows a warp, 28 with 32)
  g.rows_per_warp = 32;
  while (g.rows_per_warp > 4 && (int64_t)desc->H * desc->n_out < 32ll * ctx->sm_count * g.rows_per_warp) g.rows_per_warp /= 2;
  const int rows = g.rows_per_warp * kThreads / 32;
  const dim3 grid((unsigned)((desc->n_out + (int64_t)rows - 1) / rows), (unsigned)desc->H);
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
  if (desc->H > 1 && ((K_dst && desc->k_hs < desc->d) || (V_dst && desc->v_hs < desc->d))) return FC_ERR_INVALID_ARG;  // overlap
  FC_DEVICE_GUARD(ctx);
  return fc::kv4_unpack_launch((cudaStream_t)stream, fc::kv4_view(*src), desc->H, desc->d, desc->src_row, desc->n, K_dst,
                               V_dst, dtype, desc->k_hs, desc->k_rs, desc->v_hs, desc->v_rs, nullptr);
}
