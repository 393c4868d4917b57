// fc_kv8_append and fc_kv8_unpack: rows into and out of the paged 8-bit store.
//
// Both are bound by HBM: appending moves es + 1 bytes an element, unpacking 1 + es.
//   append   a block of threads owns one block of the store (page and head; K or V), whose rows it holds in registers between the
//            one read, the maximum that gives the scale, and the one write.  Rows that were there before are read only
//            where the scale grows.
//   unpack   a 16-byte store a thread and access, several rows' loads in flight.
//
// Codes are the nearest ones to the true quotient, whatever the type.  A tie between two codes is a number t of at most five
// significant bits, and a scale s has four.
//   bf16 rows   (8 significant bits: x is either t s or at least 2^-9 of it away) x (1/s) is off by 2^-23 at most, so that it is
//               rounded to fp16 first, which puts a tie where it belongs and crosses none.
//   fp32 rows   q = x (1/s) and one correction, q + (x - q s)(1/s), whose remainder is exact: t itself where x = t s, since what is left of q's
//               error is 2^-46 of it; otherwise x is an ulp or more from t s, and the quotient 0.53 ulp or more from t, so that
//               it stays on its side.  The remainder has to be a normal number: below a scale of 2^-90 the quotient is divided.
//   codes that are rounded again: divided.
#include <algorithm>
#include <climits>

#include "fc_kv8.cuh"
#include "fc_tcgen05.cuh"

namespace {

using fc::sm100::cvt_bf16x2;
using fc::sm100::pack2;
using fc::sm100::unpack2;

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// a in the low byte
__device__ __forceinline__ uint32_t cvt_e4m3x2(float a, float b) {
  uint16_t d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(b), "f"(a));
  return d;
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
__device__ __forceinline__ void get8(const Eight<__nv_bfloat16>& x, float (&v)[8]) {
  const uint32_t w[4] = {x.w.x, x.w.y, x.w.z, x.w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = fc::bf16_lo(w[i]), v[2 * i + 1] = fc::bf16_hi(w[i]);
}
__device__ __forceinline__ void get8(const Eight<float>& x, float (&v)[8]) {
  v[0] = x.a.x; v[1] = x.a.y; v[2] = x.a.z; v[3] = x.a.w;
  v[4] = x.b.x; v[5] = x.b.y; v[6] = x.b.z; v[7] = x.b.w;
}

__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {  // bf16 pairs; a NaN is the largest
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Bits of the largest magnitude; at or above those of infinity if an element is not finite.
__device__ __forceinline__ uint32_t largest(const Eight<__nv_bfloat16>& x) {
  constexpr uint32_t kAbs = 0x7fff7fffu;
  const uint32_t m = max2_nan(max2_nan(x.w.x & kAbs, x.w.y & kAbs), max2_nan(x.w.z & kAbs, x.w.w & kAbs));
  return max(m << 16, m & 0xffff0000u);
}
__device__ __forceinline__ uint32_t largest(const Eight<float>& x) {
  float v[8];
  get8(x, v);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);  // as integers
  return m;
}
// The same of the finite elements alone.
template <typename T>
__device__ __noinline__ uint32_t largest_finite(const Eight<T> x) {
  float v[8];
  get8(x, v);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
    m = max(m, a >= 0x7f800000u ? 0u : a);
  }
  return m;
}

// The least number of four significant bits whose 448-fold is not below a (bits of a finite magnitude): an upper bound of the
// quotient cut to four bits is it, or the one before.  448 times a number of four bits is exact.
__device__ __forceinline__ float scale_of(uint32_t a) {
  if (a == 0) return 0.f;
  const float x = fmaxf(__uint_as_float(a), 0x1.cp-109f);  // 448 2^-117
  const uint32_t low = __float_as_uint(__fmul_ru(x, 0x1.24924ap-9f)) & ~0xfffffu;  // 1/448, rounded up
  return fminf(__uint_as_float(448.f * __uint_as_float(low) >= x ? low : low + 0x100000u), 0x1p119f);
}

// Two codes of x / s: r = 1 / s, rounded.  See the head of the file for why this meets every tie.  An infinity would be cut to 448.
__device__ __forceinline__ uint32_t codes2_short(float x0, float x1, uint64_t r2) {
  float a, b;
  unpack2(mul2(pack2(x0, x1), r2), a, b);
  uint32_t h;
  uint16_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(d) : "r"(h));
  return d;
}
__device__ __forceinline__ uint2 codes8_finite(const Eight<__nv_bfloat16>& x, float, float r) {
  float v[8];
  get8(x, v);
  const uint64_t r2 = pack2(r, r);
  return make_uint2(__byte_perm(codes2_short(v[0], v[1], r2), codes2_short(v[2], v[3], r2), 0x5410),
                    __byte_perm(codes2_short(v[4], v[5], r2), codes2_short(v[6], v[7], r2), 0x5410));
}
template <bool kFinite>
__device__ __forceinline__ uint2 codes8_of(const float (&x)[8], float s) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = s > 0.f ? __fdiv_rn(x[i], s) : x[i];
    if (!kFinite) v[i] = fmaf(x[i], 0.f, v[i]);  // an infinity becomes a NaN
  }
  return make_uint2(cvt_e4m3x2(v[0], v[1]) | cvt_e4m3x2(v[2], v[3]) << 16, cvt_e4m3x2(v[4], v[5]) | cvt_e4m3x2(v[6], v[7]) << 16);
}
// s at least 2^-90, so that nothing below is too small for a remainder.
__device__ __forceinline__ uint2 codes8_finite(const Eight<float>& x, float s, float r) {
  float v[8];
  get8(x, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = v[i] * r;
    v[i] = copysignf(fmaf(fmaf(-q, s, v[i]), r, q), v[i]);  // a zero keeps its sign
  }
  return make_uint2(cvt_e4m3x2(v[0], v[1]) | cvt_e4m3x2(v[2], v[3]) << 16, cvt_e4m3x2(v[4], v[5]) | cvt_e4m3x2(v[6], v[7]) << 16);
}
// Any elements and scales, as quotients: what the two above give where they may be used.
template <typename T>
__device__ __noinline__ uint2 codes8_any(const Eight<T> x, float s) {
  float v[8];
  get8(x, v);
  return codes8_of<false>(v, s);
}
// Eight codes of scale s_old as codes of a larger scale s.
__device__ __noinline__ uint2 again8(uint2 c, float s_old, float s) {
  const uint32_t h[4] = {fc::e4m3_lo2(c.x), fc::e4m3_hi2(c.x), fc::e4m3_lo2(c.y), fc::e4m3_hi2(c.y)};
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = fc::half_lo(h[i]) * s_old, v[2 * i + 1] = fc::half_hi(h[i]) * s_old;  // eight bits: exact
  return codes8_of<true>(v, s);  // a NaN stays one
}

struct AppendGeom {
  int32_t W, H;
  int32_t block_end[FC_MAX_CHUNKS];  // running count of the pages that sequences write to
  int32_t row_off[FC_MAX_CHUNKS + 1], pos[FC_MAX_CHUNKS];
  int64_t k_hs, k_rs, v_hs, v_rs, table_cs;
  fc::Kv8View pool;
  const int32_t *table, *ref;
};

constexpr int kAppendThreads = 256;

// A group of kGroup threads owns a block of page x d elements, kVec vectors of eight elements a thread; the groups of a block of threads own
// neighbouring heads' ones.
template <typename T, int D, int kGroup, int kVec>
__global__ void __launch_bounds__(kAppendThreads)
kv8_append_kernel(const T* __restrict__ K, const T* __restrict__ V, const __grid_constant__ AppendGeom g, uint32_t* __restrict__ status) {
  constexpr int kRowVecs = D / 8, kGroups = kAppendThreads / kGroup;
  __shared__ uint32_t largest_s[kAppendThreads / 32];
  const int group = threadIdx.x / kGroup, tid = threadIdx.x % kGroup, h = blockIdx.y * kGroups + group;
  const bool is_v = blockIdx.z != 0;
  int c = 0;
  while (c + 1 < g.W && (int)blockIdx.x >= g.block_end[c]) ++c;
  const int entry = g.pos[c] / (1 << g.pool.page_log2) + (int)blockIdx.x - (c > 0 ? g.block_end[c - 1] : 0);
  const int page_id = g.table[c * g.table_cs + entry];
  if (h >= g.H) return;  // a whole group
  // rows lo .. hi - 1 of the block are new; row r of it is row src0 + r of the source
  const int64_t token0 = (int64_t)entry << g.pool.page_log2, src0 = g.row_off[c] + token0 - g.pos[c];
  const int page = 1 << g.pool.page_log2;
  const int lo = (int)max(g.pos[c] - token0, (int64_t)0);
  const int hi = (int)min((int64_t)page, g.pos[c] + (int64_t)(g.row_off[c + 1] - g.row_off[c]) - token0);
  // the thread's first row, and from one of its rows to the next
  constexpr int kRowsApart = kGroup / kRowVecs;
  static_assert(kGroup % kRowVecs == 0, "a thread keeps its columns");
  const int64_t rs = is_v ? g.v_rs : g.k_rs;
  const int row0 = tid / kRowVecs;
  const T* src = (is_v ? V + h * g.v_hs : K + h * g.k_hs) + (src0 + row0) * rs + tid % kRowVecs * 8;
  Eight<T> x[kVec];
  bool bad = false;
  uint32_t a = 0;
  const int64_t step = kRowsApart * rs;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int row = row0 + i * kRowsApart;
    if (row >= lo && row < hi) load8(src, x[i]);
    src += step;
  }
  // the rows are on their way whether or not there is a page for them
  if (page_id < 0 || page_id >= g.pool.n_pages || (g.ref && g.ref[page_id] != 1)) {
    if (threadIdx.x == 0 && status) atomicOr(status, (uint32_t)FC_DEV_BAD_INDEX);
    return;
  }
  uint8_t* codes = fc::kv8_block(is_v ? g.pool.v_codes : g.pool.k_codes, g.pool, page_id, h);
  float* scale_p = fc::kv8_scale(is_v ? g.pool.v_scales : g.pool.k_scales, g.pool, page_id, h);
  const float s_old = lo > 0 ? *scale_p : 0.f;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int row = row0 + i * kRowsApart;
    if (row >= lo && row < hi) a = max(a, largest(x[i]));
  }
  if (a >= 0x7f800000u) {
    bad = true;
    a = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int row = row0 + i * kRowsApart;
      if (row >= lo && row < hi) a = max(a, largest_finite<T>(x[i]));
    }
  }
  a = __reduce_max_sync(0xffffffffu, a);
  if constexpr (kGroup > 32) {
    if (tid % 32 == 0) largest_s[threadIdx.x / 32] = a;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(kGroup) : "memory");
#pragma unroll
    for (int i = 0; i < kGroup / 32; ++i) a = max(a, largest_s[group * (kGroup / 32) + i]);
  }
  const float s = fmaxf(scale_of(a), s_old), r = s > 0.f ? __frcp_rn(s) : 0.f;
  const bool slow = bad || (sizeof(T) == 4 && s < 0x1p-90f);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int row = row0 + i * kRowsApart;
    uint2* at = reinterpret_cast<uint2*>(codes) + tid + i * kGroup;
    if (row < hi && !fc::bounds_ok(row < page && tid + i * kGroup < page * kRowVecs, status)) continue;
    if (row >= lo && row < hi) *at = slow ? codes8_any<T>(x[i], s) : codes8_finite(x[i], s, r);
    else if (row < lo && s > s_old) *at = again8(*at, s_old, s);
  }
  if (tid == 0 && (lo == 0 || s > s_old)) *scale_p = s;  // every thread of the group has read the old one
  if (bad && status) atomicOr(status, (uint32_t)FC_DEV_NONFINITE);
}

struct UnpackGeom {
  fc::Kv8Jobs jobs;
  int32_t block_end[fc::kKv8Jobs];  // running count of the jobs' blocks, so that a short one beside a long one has no empty blocks
  int64_t k_hs, k_rs, v_hs, v_rs, table_cs, rows;  // rows of a head of the destination
  fc::Kv8View src;
  const int32_t* table;
  uint32_t *status, *clear;
};

constexpr int kUnpackThreads = 256;
constexpr int kUnpackRows = 4;  // rows whose loads are in flight together

// The codes of a 16-byte store, and their values.
__device__ __forceinline__ void store_values(__nv_bfloat16* p, uint2 c, float s) {
  const uint32_t h[4] = {fc::e4m3_lo2(c.x), fc::e4m3_hi2(c.x), fc::e4m3_lo2(c.y), fc::e4m3_hi2(c.y)};
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = cvt_bf16x2(fc::half_lo(h[i]) * s, fc::half_hi(h[i]) * s);
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_values(float* p, uint32_t c, float s) {
  const uint32_t a = fc::e4m3_lo2(c), b = fc::e4m3_hi2(c);
  *reinterpret_cast<float4*>(p) = make_float4(fc::half_lo(a) * s, fc::half_hi(a) * s, fc::half_lo(b) * s, fc::half_hi(b) * s);
}
template <typename T> struct Codes;
template <> struct Codes<__nv_bfloat16> { using type = uint2; };
template <> struct Codes<float> { using type = uint32_t; };

template <typename T, int D>
__global__ void __launch_bounds__(kUnpackThreads)
kv8_unpack_kernel(T* __restrict__ K, T* __restrict__ V, const __grid_constant__ UnpackGeom g) {
  using C = typename Codes<T>::type;
  constexpr int kVec = sizeof(C), kRowVecs = D / kVec, R = kUnpackThreads / kRowVecs;
  fc::pdl_launch_dependents();
  const int w = threadIdx.x % kRowVecs, h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  if (g.clear && threadIdx.x == 0 && blockIdx.x == 0 && h == 0 && blockIdx.z == 0) *g.clear = 0;
  T* dst = is_v ? V : K;
  if (!dst) return;
  int j = 0;  // the first job whose end is behind this block
  for (int end = g.jobs.n - 1; j < end;) {
    const int mid = (j + end) / 2;
    if (g.block_end[mid] > (int)blockIdx.x) end = mid;
    else j = mid + 1;
  }
  const fc::Kv8Job job = g.jobs.job[j];
  if (g.jobs.active_ids) {
    const int lane = threadIdx.x % 32, n = min(max(*g.jobs.n_active, 0), g.jobs.W);
    uint64_t mine = 0;
    for (int i = lane; i < n; i += 32) {
      const int c = g.jobs.active_ids[i];
      if (c >= 0 && c < g.jobs.W) mine |= 1ull << c;
    }
    const uint32_t lo = __reduce_or_sync(0xffffffffu, (uint32_t)mine), hi = __reduce_or_sync(0xffffffffu, (uint32_t)(mine >> 32));
    if (!(((uint64_t)hi << 32 | lo) & g.jobs.needed[j])) return;
  }
  const int r0 = ((int)blockIdx.x - (j > 0 ? g.block_end[j - 1] : 0)) * (kUnpackRows * R) + threadIdx.x / kRowVecs;  // below 2^31, as the tokens are
  if (r0 >= job.n) return;
  uint8_t* codes = fc::kv8_block(is_v ? g.src.v_codes : g.src.k_codes, g.src, 0, h);
  float* scales = fc::kv8_scale(is_v ? g.src.v_scales : g.src.k_scales, g.src, 0, h);
  const int64_t rs = is_v ? g.v_rs : g.k_rs;
  const int32_t* table = g.table + job.seq * g.table_cs;
  int32_t page_id[kUnpackRows];
  C word[kUnpackRows];
  float scale[kUnpackRows];
#pragma unroll
  for (int u = 0; u < kUnpackRows; ++u) page_id[u] = r0 + u * R < job.n ? __ldg(table + ((job.first + r0 + u * R) >> g.src.page_log2)) : -1;
  bool bad = false;
#pragma unroll
  for (int u = 0; u < kUnpackRows; ++u) {
    word[u] = C{};
    scale[u] = 0.f;
    const bool there = (uint32_t)page_id[u] < (uint32_t)g.src.n_pages;
    if (there) {
      const int in_page = (job.first + r0 + u * R) & ((1 << g.src.page_log2) - 1);
      word[u] = __ldg(reinterpret_cast<const C*>(fc::kv8_block(codes, g.src, page_id[u], 0)) + in_page * kRowVecs + w);
      scale[u] = __ldg(fc::kv8_scale(scales, g.src, page_id[u], 0));
    }
    bad |= !there && r0 + u * R < job.n;
  }
  T* out = dst + h * (is_v ? g.v_hs : g.k_hs) + (job.dst_row + r0) * rs + kVec * w;
  const int64_t step = R * rs;
#pragma unroll
  for (int u = 0; u < kUnpackRows; ++u) {
    const int r = r0 + u * R;
    if (r < job.n && fc::bounds_ok(job.dst_row + r < g.rows, g.status)) store_values(out, word[u], scale[u]);
    out += step;
  }
  if (bad && g.status) atomicOr(g.status, (uint32_t)FC_DEV_BAD_INDEX);
}

int check_rows(const void* p, int d, int es, int64_t hs, int64_t rs) {
  if (!fc::aligned16(p)) return FC_ERR_MISALIGNED;
  if (hs < 0 || rs < 0 || (hs * es) % 16 || (rs * es) % 16) return FC_ERR_MISALIGNED;
  return rs < d ? FC_ERR_INVALID_ARG : FC_OK;
}

// What append and unpack ask of their common arguments: `at` is the first token of each sequence's rows.
int check_common(const fc_kv8_rows* desc, int dtype, const int32_t* row_off, const int32_t* at) {
  if (dtype != FC_BF16 && dtype != FC_F32) return FC_ERR_UNSUPPORTED;
  if (desc->d != 64 && desc->d != 128) return FC_ERR_UNSUPPORTED;
  if (desc->H <= 0 || desc->W <= 0 || !row_off || !at) return FC_ERR_INVALID_ARG;
  if (desc->H > 65535 || desc->W > FC_MAX_CHUNKS) return FC_ERR_UNSUPPORTED;
  for (int c = 0; c < desc->W; ++c) {
    if (row_off[c] < 0 || row_off[c + 1] < row_off[c] || at[c] < 0) return FC_ERR_INVALID_ARG;
    if ((int64_t)at[c] + (row_off[c + 1] - row_off[c]) > INT32_MAX - 4096) return FC_ERR_UNSUPPORTED;
  }
  return FC_OK;
}

}  // namespace

namespace fc {

int kv8_unpack_launch(cudaStream_t st, const Kv8View& src, int H, int d, const int32_t* table, int64_t table_cs, const Kv8Jobs& jobs,
                      void* K_dst, void* V_dst, int64_t dst_rows, int dtype, int64_t k_hs, int64_t k_rs, int64_t v_hs, int64_t v_rs,
                      uint32_t* status, uint32_t* clear) {
  int64_t blocks = 0;
  UnpackGeom g = {jobs, {}, k_hs, k_rs, v_hs, v_rs, table_cs, dst_rows, src, table, status, clear};
  const int rows = kUnpackRows * kUnpackThreads / (d / (dtype == FC_F32 ? 4 : 8));
  for (int i = 0; i < jobs.n; ++i) g.block_end[i] = (int32_t)(blocks += ((int64_t)jobs.job[i].n + rows - 1) / rows);
  if (blocks == 0 || (!K_dst && !V_dst)) return FC_OK;
  const dim3 grid((unsigned)blocks, (unsigned)H, 2);
#define FC_UNPACK(T, D) kv8_unpack_kernel<T, D><<<grid, kUnpackThreads, 0, st>>>((T*)K_dst, (T*)V_dst, g)
  if (dtype == FC_F32) { if (d == 128) FC_UNPACK(float, 128); else FC_UNPACK(float, 64); }
  else { if (d == 128) FC_UNPACK(__nv_bfloat16, 128); else FC_UNPACK(__nv_bfloat16, 64); }
#undef FC_UNPACK
  FC_LAUNCH_CHECK("kv8_unpack_kernel");
  return FC_OK;
}

}  // namespace fc

extern "C" int fc_kv8_append(fc_ctx* ctx, void* stream, const fc_kv8_rows* desc, const void* K_src, const void* V_src, int dtype,
                             const int32_t* row_off, const int32_t* pos, const fc_kv8_pool* pool, const int32_t* table,
                             int64_t table_cs, const int32_t* ref, uint32_t* status) {
  if (!ctx || !desc) return FC_ERR_INVALID_ARG;
  int rc = check_common(desc, dtype, row_off, pos);
  if (rc != FC_OK) return rc;
  if (row_off[desc->W] == row_off[0]) return FC_OK;
  if (!K_src || !V_src || !table || table_cs < 0) return FC_ERR_INVALID_ARG;
  const int es = fc::elem_size(dtype);
  if ((rc = check_rows(K_src, desc->d, es, desc->k_hs, desc->k_rs)) != FC_OK) return rc;
  if ((rc = check_rows(V_src, desc->d, es, desc->v_hs, desc->v_rs)) != FC_OK) return rc;
  if ((rc = fc::kv8_check(pool, desc->H, desc->d)) != FC_OK) return rc;
  AppendGeom g = {};
  g.W = desc->W;
  g.H = desc->H;
  g.pool = fc::kv8_view(*pool);
  int64_t blocks = 0;
  for (int c = 0; c < g.W; ++c) {
    const int64_t n = row_off[c + 1] - row_off[c], end = ((int64_t)pos[c] + n + pool->page - 1) / pool->page;
    if (n > 0) {
      if (g.W > 1 && table_cs < end) return FC_ERR_INVALID_ARG;  // rows of the table would overlap
      blocks += end - pos[c] / pool->page;
    }
    if (blocks > INT32_MAX) return FC_ERR_UNSUPPORTED;
    g.block_end[c] = (int32_t)blocks;
    g.row_off[c] = row_off[c];
    g.pos[c] = pos[c];
  }
  g.row_off[g.W] = row_off[g.W];
  g.k_hs = desc->k_hs; g.k_rs = desc->k_rs; g.v_hs = desc->v_hs; g.v_rs = desc->v_rs;
  g.table = table; g.table_cs = table_cs; g.ref = ref;
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
#define FC_APPEND(T, D, GROUP, VEC)                                                                                              \
  kv8_append_kernel<T, D, GROUP, VEC><<<dim3((unsigned)blocks, (unsigned)((desc->H + kAppendThreads / GROUP - 1) / (kAppendThreads / GROUP)), 2), \
                                        kAppendThreads, 0, st>>>((const T*)K_src, (const T*)V_src, g, status)
#define FC_APPEND_PICK(T)                                                                                                        \
  do {                                                                                                                           \
    if (desc->d == 128) switch (pool->page) {                                                                                    \
      case 16: FC_APPEND(T, 128, 64, 4); break;                                                                                  \
      case 32: FC_APPEND(T, 128, 128, 4); break;                                                                                 \
      case 64: FC_APPEND(T, 128, 256, 4); break;                                                                                 \
      default: FC_APPEND(T, 128, 256, 8);                                                                                        \
    } else switch (pool->page) {                                                                                                 \
      case 16: FC_APPEND(T, 64, 32, 4); break;                                                                                   \
      case 32: FC_APPEND(T, 64, 64, 4); break;                                                                                   \
      case 64: FC_APPEND(T, 64, 128, 4); break;                                                                                  \
      default: FC_APPEND(T, 64, 256, 4);                                                                                         \
    }                                                                                                                            \
  } while (0)
  if (dtype == FC_F32) FC_APPEND_PICK(float);
  else FC_APPEND_PICK(__nv_bfloat16);
#undef FC_APPEND_PICK
#undef FC_APPEND
  FC_LAUNCH_CHECK("kv8_append_kernel");
  return FC_OK;
}

extern "C" int fc_kv8_unpack(fc_ctx* ctx, void* stream, const fc_kv8_rows* desc, const fc_kv8_pool* pool, const int32_t* table,
                             int64_t table_cs, const int32_t* first, const int32_t* row_off, void* K_dst, void* V_dst, int dtype,
                             uint32_t* status) {
  if (!ctx || !desc) return FC_ERR_INVALID_ARG;
  int rc = check_common(desc, dtype, row_off, first);
  if (rc != FC_OK) return rc;
  if (row_off[desc->W] == row_off[0]) return FC_OK;
  if ((!K_dst && !V_dst) || !table || table_cs < 0) return FC_ERR_INVALID_ARG;
  const int es = fc::elem_size(dtype);
  if (K_dst && (rc = check_rows(K_dst, desc->d, es, desc->k_hs, desc->k_rs)) != FC_OK) return rc;
  if (V_dst && (rc = check_rows(V_dst, desc->d, es, desc->v_hs, desc->v_rs)) != FC_OK) return rc;
  const int64_t rows = row_off[desc->W];
  if (K_dst && !fc::grid_disjoint(desc->H, desc->k_hs, rows, desc->k_rs, desc->d)) return FC_ERR_INVALID_ARG;  // rows overlap
  if (V_dst && !fc::grid_disjoint(desc->H, desc->v_hs, rows, desc->v_rs, desc->d)) return FC_ERR_INVALID_ARG;
  if ((rc = fc::kv8_check(pool, desc->H, desc->d)) != FC_OK) return rc;
  fc::Kv8Jobs jobs = {};
  for (int c = 0; c < desc->W; ++c)
    if (row_off[c + 1] > row_off[c]) jobs.job[jobs.n++] = {c, first[c], row_off[c + 1] - row_off[c], row_off[c]};
  FC_DEVICE_GUARD(ctx);
  return fc::kv8_unpack_launch((cudaStream_t)stream, fc::kv8_view(*pool), desc->H, desc->d, table, table_cs, jobs, K_dst, V_dst,
                               rows, dtype, desc->k_hs, desc->k_rs, desc->v_hs, desc->v_rs, status, nullptr);
}
