// fc_qk_norm_rope: RMS norm of every head of queries and keys, and the rotation over (time, height, width), in one pass.
//
// A head's row is spread over 16-byte pieces, one per lane (16 lanes for a bf16 row of 128): each element is read and
// written once and everything between is in registers.  A group of lanes owns a token and walks over some of its heads,
// so that the token's cosines and sines, which all heads share, are computed once per group and not once per row.
// Angles: a pair's frequency is held in turns as a 64-bit fixed-point fraction, so position x frequency is one wrapping
// integer product whose overflow is exactly the reduction modulo a full turn; its top 32 bits go to sincospif.
#include <climits>
#include <cmath>

#include "fc_common.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // heads whose loads are in flight together

struct RopeGeom {
  int32_t H_q, H_kv, T, heads_per_item;
  int64_t q_hs, q_rs, k_hs, k_rs, qo_hs, qo_rs, ko_hs, ko_rs;
  int32_t axis_dim[3];
  int32_t norm;
  float eps;
  int32_t t0, gh, gw;
  int64_t n_items;
  uint64_t turns[64];  // per pair, in the order of the sections: turns per position, modulo one, times 2^64
};

template <typename T> struct Piece;  // 16 bytes of a row
template <> struct Piece<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const void* p, float (&x)[N]) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = fc::bf16_lo(w[i]);
      x[2 * i + 1] = fc::bf16_hi(w[i]);
    }
  }
  static __device__ __forceinline__ void store(void* p, const float (&x)[N]) {
    uint4 v;
    uint32_t* w = &v.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = v;
  }
};
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(const void* p, float (&x)[N]) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  }
  static __device__ __forceinline__ void store(void* p, const float (&x)[N]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  }
};

// Element e of a head: the pair it belongs to (-1: it does not turn), its partner and whether it is the pair's first.
template <bool kHalves>
__device__ __forceinline__ void place(const RopeGeom& g, int e, int& pair, int& axis, int& partner, bool& first) {
  int start = 0, pair0 = 0;
  pair = -1; axis = 0; partner = e; first = true;
#pragma unroll
  for (int a = 0; a < 3; ++a) {
    const int n = g.axis_dim[a], o = e - start;
    if (o >= 0 && o < n) {
      axis = a;
      if (kHalves) {
        first = o < n / 2;
        pair = pair0 + (first ? o : o - n / 2);
        partner = first ? e + n / 2 : e - n / 2;
      } else {
        first = (o & 1) == 0;
        pair = pair0 + o / 2;
        partner = e ^ 1;
      }
    }
    start += n;
    pair0 += n / 2;
  }
}

template <typename T, int D, bool kHalves>
__global__ void __launch_bounds__(kThreads)
qk_norm_rope_kernel(const T* Q, const T* K, T* Q_out, T* K_out, const float* __restrict__ q_weight,
                    const float* __restrict__ k_weight, const int32_t* __restrict__ pos, const __grid_constant__ RopeGeom g) {
  using P = Piece<T>;
  constexpr int E = P::N, L = D / E;  // elements per lane, lanes per row
  __shared__ uint64_t turns_s[64];
  __shared__ float row_s[kHalves ? kThreads * E : 1];  // the normed row, where partners sit in other lanes
  const int tid = threadIdx.x;
  if (tid < 64) turns_s[tid] = g.turns[tid];
  __syncthreads();

  const int lane = tid % L, grp = tid / L;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / L) + grp;
  const bool live = item < g.n_items;
  const int n = live ? (int)(item % g.T) : 0;
  const int h0 = live ? (int)(item / g.T) * g.heads_per_item : 0;
  const int h1 = live ? min(h0 + g.heads_per_item, g.H_q + g.H_kv) : 0;

  int p[3];
  if (pos) {
#pragma unroll
    for (int a = 0; a < 3; ++a) p[a] = pos[3ll * n + a];
  } else {
    const int frame = g.gh * g.gw;
    p[0] = g.t0 + n / frame;
    p[1] = n % frame / g.gw;
    p[2] = n % g.gw;
  }
  // out[i] = y[i] * c[i] + y[partner of i] * s[i]
  float c[E], s[E];
  int partner[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    int pair, axis;
    bool first;
    place<kHalves>(g, lane * E + i, pair, axis, partner[i], first);
    c[i] = 1.f;
    s[i] = 0.f;
    if (!kHalves && (i & 1)) {  // the pair's angle is that of the element before
      c[i] = c[i - 1];
      s[i] = -s[i - 1];
    } else if (pair >= 0) {
      const int at = axis == 0 ? p[0] : axis == 1 ? p[1] : p[2];
      const uint64_t phase = (uint64_t)(int64_t)at * turns_s[pair] + 0x80000000ull;
      float sn;
      sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &sn, &c[i]);
      s[i] = first ? -sn : sn;
    }
  }

  auto walk = [&](const T* src, T* dst, int64_t hs, int64_t rs, int64_t ohs, int64_t ors, const float* weight, int a, int b) {
    float w[E];
#pragma unroll
    for (int i = 0; i < E; ++i) w[i] = weight && g.norm ? weight[lane * E + i] : 1.f;
    const T* in = src + (int64_t)n * rs + lane * E;
    T* out = dst + (int64_t)n * ors + lane * E;
    for (int h = a; h < b; h += kUnroll) {
      float x[kUnroll][E];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (h + u < b) P::load(in + (int64_t)(h + u) * hs, x[u]);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (h + u >= b) break;
        if (g.norm) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < E; ++i) sum = fmaf(x[u][i], x[u][i], sum);
          const unsigned mask = L == 32 ? 0xffffffffu : ((1u << L) - 1u) << (tid & 31 & ~(L - 1));
#pragma unroll
          for (int k = 1; k < L; k <<= 1) sum += __shfl_xor_sync(mask, sum, k);
          const float r = 1.f / sqrtf(sum * (1.f / D) + g.eps);
#pragma unroll
          for (int i = 0; i < E; ++i) x[u][i] *= r * w[i];
        }
        float y[E];
        if (kHalves) {
          float* row = row_s + grp * D;
          const unsigned mask = L == 32 ? 0xffffffffu : ((1u << L) - 1u) << (tid & 31 & ~(L - 1));
#pragma unroll
          for (int i = 0; i < E; ++i) row[lane * E + i] = x[u][i];
          __syncwarp(mask);
#pragma unroll
          for (int i = 0; i < E; ++i) y[i] = fmaf(x[u][i], c[i], row[partner[i]] * s[i]);
          __syncwarp(mask);
        } else {
#pragma unroll
          for (int i = 0; i < E; ++i) y[i] = fmaf(x[u][i], c[i], x[u][i ^ 1] * s[i]);
        }
        P::store(out + (int64_t)(h + u) * ohs, y);
      }
    }
  };
  if (h0 < g.H_q) walk(Q, Q_out, g.q_hs, g.q_rs, g.qo_hs, g.qo_rs, q_weight, h0, min(h1, g.H_q));
  if (h1 > g.H_q) walk(K, K_out, g.k_hs, g.k_rs, g.ko_hs, g.ko_rs, k_weight, max(h0 - g.H_q, 0), h1 - g.H_q);
}

// f radians per position -> turns per position modulo one, times 2^64
uint64_t turns_of(double f) {
  long double t = (long double)f * 0.159154943091895335768883763372514362L;
  if (!(t >= 0.0L && t < 1.0L)) t -= floorl(t);
  return t < 1.0L ? (uint64_t)(t * 0x1p64L) : 0;
}

}  // namespace

extern "C" int fc_qk_norm_rope(fc_ctx* ctx, void* stream, const fc_rope_desc* desc, const void* Q, const void* K, int dtype,
                               const float* q_weight, const float* k_weight, const int32_t* pos, const double* inv_freq,
                               void* Q_out, void* K_out) {
  if (!ctx || !desc) return FC_ERR_INVALID_ARG;
  if (dtype != FC_BF16 && dtype != FC_F32) return FC_ERR_UNSUPPORTED;
  if (desc->d != 64 && desc->d != 128) return FC_ERR_UNSUPPORTED;
  if (desc->H_q < 0 || desc->H_kv < 0 || desc->T < 0 || desc->H_q > INT32_MAX - desc->H_kv) return FC_ERR_INVALID_ARG;
  if (desc->T > 0 && desc->H_q > 0 && (!Q || !Q_out)) return FC_ERR_INVALID_ARG;
  if (desc->T > 0 && desc->H_kv > 0 && (!K || !K_out)) return FC_ERR_INVALID_ARG;
  if (desc->pairing != FC_ROPE_PAIRS && desc->pairing != FC_ROPE_HALVES) return FC_ERR_INVALID_ARG;
  if (desc->norm != FC_NORM_NONE && desc->norm != FC_NORM_RMS) return FC_ERR_INVALID_ARG;
  if (!(desc->eps >= 0.f)) return FC_ERR_INVALID_ARG;
  int64_t turning = 0;
  for (int a = 0; a < 3; ++a) {
    if (desc->axis_dim[a] < 0 || desc->axis_dim[a] % 2) return FC_ERR_INVALID_ARG;
    turning += desc->axis_dim[a];
  }
  if (turning > desc->d) return FC_ERR_INVALID_ARG;
  RopeGeom g = {};
  if (turning > 0) {
    if (!inv_freq && !(desc->theta > 0.0 && std::isfinite(desc->theta))) return FC_ERR_INVALID_ARG;
    if (!pos) {
      if (desc->grid_h <= 0 || desc->grid_w <= 0) return FC_ERR_INVALID_ARG;
      const int64_t frame = (int64_t)desc->grid_h * desc->grid_w;
      if (frame > INT32_MAX || desc->grid_t0 + (int64_t)(desc->T > 0 ? desc->T - 1 : 0) / frame > INT32_MAX) return FC_ERR_INVALID_ARG;
    }
    int k = 0;
    for (int a = 0; a < 3; ++a) {
      const int half = desc->axis_dim[a] / 2;
      const bool same = !inv_freq && a > 0 && desc->axis_dim[a] == desc->axis_dim[a - 1];  // height and width, as a rule
      for (int i = 0; i < half; ++i, ++k) {
        if (same) {
          g.turns[k] = g.turns[k - half];
          continue;
        }
        const double f = inv_freq ? inv_freq[k] : pow(desc->theta, -2.0 * i / desc->axis_dim[a]);
        if (!std::isfinite(f)) return FC_ERR_INVALID_ARG;
        g.turns[k] = turns_of(f);
      }
    }
  }
  const int es = fc::elem_size(dtype);
  const struct { int heads; const void *in, *out; int64_t s[4]; } side[2] = {
      {desc->H_q, Q, Q_out, {desc->q_hs, desc->q_rs, desc->qo_hs, desc->qo_rs}},
      {desc->H_kv, K, K_out, {desc->k_hs, desc->k_rs, desc->ko_hs, desc->ko_rs}}};
  for (const auto& x : side) {
    if (x.heads == 0) continue;
    if (!fc::aligned16(x.in) || !fc::aligned16(x.out)) return FC_ERR_MISALIGNED;
    for (int64_t s : x.s)
      if (s < 0 || (s * es) % 16) return FC_ERR_MISALIGNED;
  }
  const int64_t heads = (int64_t)desc->H_q + desc->H_kv;
  if (heads == 0 || desc->T == 0) return FC_OK;

  g.H_q = desc->H_q; g.H_kv = desc->H_kv; g.T = desc->T;
  g.q_hs = desc->q_hs; g.q_rs = desc->q_rs; g.k_hs = desc->k_hs; g.k_rs = desc->k_rs;
  g.qo_hs = desc->qo_hs; g.qo_rs = desc->qo_rs; g.ko_hs = desc->ko_hs; g.ko_rs = desc->ko_rs;
  for (int a = 0; a < 3; ++a) g.axis_dim[a] = desc->axis_dim[a];
  g.norm = desc->norm; g.eps = desc->eps;
  if (turning == 0) pos = nullptr;
  const bool grid_used = turning > 0 && !pos;
  g.t0 = grid_used ? desc->grid_t0 : 0;
  g.gh = grid_used ? desc->grid_h : 1;
  g.gw = grid_used ? desc->grid_w : 1;
  // heads per item: as many as leave the device one full set of resident groups; a lone token gets a group per head
  const int lanes = desc->d * es / 16, groups = kThreads / lanes;
  const int64_t resident = (int64_t)ctx->sm_count * 2048 / lanes;
  int64_t per = heads * desc->T / resident;
  per = per < 1 ? 1 : per > heads ? heads : per;
  g.heads_per_item = (int32_t)per;
  g.n_items = (heads + per - 1) / per * desc->T;
  const int64_t blocks = (g.n_items + groups - 1) / groups;
  if (blocks > INT32_MAX) return FC_ERR_UNSUPPORTED;
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
#define FC_ROPE_LAUNCH(T, D, HALVES)                                                                                  \
  qk_norm_rope_kernel<T, D, HALVES><<<(unsigned)blocks, kThreads, 0, st>>>((const T*)Q, (const T*)K, (T*)Q_out, (T*)K_out, \
                                                                           q_weight, k_weight, pos, g)
#define FC_ROPE_PICK(T)                                                                                      \
  if (desc->d == 128) {                                                                                      \
    if (desc->pairing == FC_ROPE_HALVES) FC_ROPE_LAUNCH(T, 128, true); else FC_ROPE_LAUNCH(T, 128, false);   \
  } else {                                                                                                   \
    if (desc->pairing == FC_ROPE_HALVES) FC_ROPE_LAUNCH(T, 64, true); else FC_ROPE_LAUNCH(T, 64, false);     \
  }
  if (dtype == FC_F32) { FC_ROPE_PICK(float) } else { FC_ROPE_PICK(__nv_bfloat16) }
#undef FC_ROPE_PICK
#undef FC_ROPE_LAUNCH
  FC_LAUNCH_CHECK("qk_norm_rope_kernel");
  return FC_OK;
}
