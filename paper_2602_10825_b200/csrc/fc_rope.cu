// fc_qk_norm_rope: RMS norm of every head of queries and keys, and the rotation over (time, height, width), in one pass.
//
// Bound by HBM: every element is read and written once (4680 tokens of 48 bf16 heads of 128 at 4.7 TB/s, launch included; a
// plain copy of the same bytes takes 21 us).  A head's row is spread over 16-byte pieces, one per lane (16 lanes for a
// bf16 row of 128), and everything between the load and the store is in registers.  A group of lanes owns a token and walks
// over some of its heads, four rows' loads in flight.  What it takes to stay under the copy rate is few instructions:
//   - The cosines and sines of a token serve all its heads.  A block computes them once for its tokens, a pair a thread, and
//     leaves them in shared memory; a group keeps its own in registers, multiplied by the norm's weights, so that the
//     normed, weighted and rotated pair is (x0 cw0 - x1 sw1, x1 cw1 + x0 sw0) / rms.
//   - Even and odd elements are held as pairs of fp32, so that squares, rotation and scaling are two-wide instructions.
//   - With FC_ROPE_HALVES the partner of an element sits in another lane at an odd distance: the rows go through shared
//     memory as they are, and the partners are read one by one.
// Angles: a pair's frequency is held in turns as a 64-bit fixed-point fraction, so position x frequency is one wrapping
// integer product whose overflow is exactly the reduction modulo a full turn; its top 32 bits, rounded to an fp32 number, go to
// sincospif (2^-24 of the angle, as much as the fp32 products behind it are off by).
//
// Measured, one call among others with the launch: 4680 tokens of 48 bf16 heads of 128 in 24.6 us, 18719 tokens of 8 fp32 heads of 64 with
// far pairs in 18.4.  In replayed graphs the first takes 21.0 us, with far pairs 31.7, which is the cost of reading each
// partner by itself, two bytes at a time, from shared memory (fp32: 38.6 and 40.3).  When the sizes were chosen: blocks of 128 threads
// 25.0 us (35.7 with far pairs, fp32 heads of 64 19.2), of 256 threads 25.2, 37.2 and 20.8; without sending for the first rows before
// the angles 27.4 and 22.8; with two rows in flight, or the next rows sent for before the arithmetic, slower still.
#include <climits>
#include <cmath>

#include "fc_common.cuh"
#include "fc_tcgen05.cuh"

namespace {

using fc::sm100::add2;
using fc::sm100::cvt_bf16x2;
using fc::sm100::fma2;
using fc::sm100::pack2;
using fc::sm100::unpack2;

// Small blocks: a block's angles hold up only its own rows.
constexpr int kThreads = 128;
constexpr int kUnroll = 4;  // heads whose loads are in flight together

struct RopeGeom {
  int32_t H_q, H_kv, T;
  int32_t tokens, heads_per_group;  // tokens of a block; heads that a group of lanes walks over
  int64_t q_hs, q_rs, k_hs, k_rs, qo_hs, qo_rs, ko_hs, ko_rs;
  int32_t axis_dim[3];
  int32_t norm;
  float eps;
  int32_t t0, gh, gw;
  uint64_t turns[64];  // per pair, in the order of the sections: turns per position, modulo one, times 2^64
};

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// 16 bytes of a row as even and odd elements, two of each to a register pair: e[i] = (x[4i], x[4i+2]), o[i] = (x[4i+1], x[4i+3]).
template <typename T> struct Piece;
template <> struct Piece<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void split(const uint4& v, uint64_t (&e)[2], uint64_t (&o)[2]) {
    e[0] = pack2(fc::bf16_lo(v.x), fc::bf16_lo(v.y));
    o[0] = pack2(fc::bf16_hi(v.x), fc::bf16_hi(v.y));
    e[1] = pack2(fc::bf16_lo(v.z), fc::bf16_lo(v.w));
    o[1] = pack2(fc::bf16_hi(v.z), fc::bf16_hi(v.w));
  }
  static __device__ __forceinline__ uint4 join(const uint64_t (&e)[2], const uint64_t (&o)[2]) {
    float a[4], b[4];
    unpack2(e[0], a[0], a[1]);
    unpack2(o[0], b[0], b[1]);
    unpack2(e[1], a[2], a[3]);
    unpack2(o[1], b[2], b[3]);
    return make_uint4(cvt_bf16x2(a[0], b[0]), cvt_bf16x2(a[1], b[1]), cvt_bf16x2(a[2], b[2]), cvt_bf16x2(a[3], b[3]));
  }
};
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void split(const uint4& v, uint64_t (&e)[1], uint64_t (&o)[1]) {
    e[0] = pack2(__uint_as_float(v.x), __uint_as_float(v.z));
    o[0] = pack2(__uint_as_float(v.y), __uint_as_float(v.w));
  }
  static __device__ __forceinline__ uint4 join(const uint64_t (&e)[1], const uint64_t (&o)[1]) {
    float a[2], b[2];
    unpack2(e[0], a[0], a[1]);
    unpack2(o[0], b[0], b[1]);
    return make_uint4(__float_as_uint(a[0]), __float_as_uint(b[0]), __float_as_uint(a[1]), __float_as_uint(b[1]));
  }
};

// FC_ROPE_HALVES: the pair element e of a head belongs to (-1: it does not turn), its partner and whether it is the first.
__device__ __forceinline__ void place(const RopeGeom& g, int e, int& pair, int& partner, bool& first) {
  int start = 0;
  pair = -1; partner = e; first = true;
#pragma unroll
  for (int a = 0; a < 3; ++a) {
    const int n = g.axis_dim[a], o = e - start;
    if (o >= 0 && o < n) {
      first = o < n / 2;
      pair = start / 2 + (first ? o : o - n / 2);
      partner = first ? e + n / 2 : e - n / 2;
    }
    start += n;
  }
}

// kPass: the sections leave elements that pass through.  An instance of its own, since the others have no register to spare (4680 tokens of
// 48 bf16 heads of 128 in a replayed graph: 19.7 us, where half the elements pass through 20.5).
template <typename T, int D, bool kHalves, bool kPass>
__global__ void __launch_bounds__(kThreads, kHalves && sizeof(T) == 2 ? 6 : 8)  // 80 registers where eight partners are looked up, else 64
qk_norm_rope_kernel(const T* Q, const T* K, T* Q_out, T* K_out, const float* __restrict__ q_weight,
                    const float* __restrict__ k_weight, const int32_t* __restrict__ pos, const __grid_constant__ RopeGeom g) {
  using P = Piece<T>;
  constexpr int E = P::N, L = D / E, G = kThreads / L, V = E / 4;  // elements per lane, lanes per row, rows per block, pairs of pairs
  __shared__ float2 cs_s[G * (D / 2)];                     // (cos, sin) of the block's tokens and pairs
  __shared__ __align__(16) T row_s[kHalves ? kUnroll * kThreads * E : 1];  // the rows in flight, where partners sit in other lanes
  const int tid = threadIdx.x, lane = tid % L, grp = tid / L;
  const int first_token = blockIdx.x * g.tokens;

  const int t = grp % g.tokens, n = first_token + t;
  const int h0 = (blockIdx.y * (G / g.tokens) + grp / g.tokens) * g.heads_per_group;
  const int h1 = min(h0 + g.heads_per_group, g.H_q + g.H_kv);
  const bool idle = n >= g.T || h0 >= h1;
  // the first rows are sent for before the angles are worked out
  uint4 raw[kUnroll];
  if (!idle) {
    const bool q = h0 < g.H_q;
    const T* in = (q ? Q + (int64_t)n * g.q_rs + h0 * g.q_hs : K + (int64_t)n * g.k_rs + (h0 - g.H_q) * g.k_hs) + lane * E;
    const int rows = (q ? min(h1, g.H_q) : h1) - h0;
    const int64_t hs = q ? g.q_hs : g.k_hs;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (u < rows) raw[u] = *reinterpret_cast<const uint4*>(in + u * hs);
  }

  const int turning = g.axis_dim[0] + g.axis_dim[1] + g.axis_dim[2], pairs = turning / 2;
  for (int x = tid; x < g.tokens * (D / 2); x += kThreads) {
    const int t = x / (D / 2), pair = x % (D / 2), n = min(first_token + t, g.T - 1);
    if (pair >= pairs) {  // what does not turn, in the order of FC_ROPE_PAIRS
      cs_s[x] = make_float2(1.f, 0.f);
      continue;
    }
    const int axis = pair < g.axis_dim[0] / 2 ? 0 : pair < (g.axis_dim[0] + g.axis_dim[1]) / 2 ? 1 : 2;
    int at;
    if (pos) {
      at = pos[3ll * n + axis];
    } else {
      const int frame = g.gh * g.gw;
      at = axis == 0 ? g.t0 + n / frame : axis == 1 ? n % frame / g.gw : n % g.gw;
    }
    const uint64_t phase = (uint64_t)(int64_t)at * g.turns[pair] + 0x80000000ull;
    float2 cs;
    sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &cs.y, &cs.x);
    cs_s[x] = cs;
  }
  __syncthreads();

  if (idle) return;
  const unsigned mask = L == 32 ? 0xffffffffu : ((1u << L) - 1u) << (tid & 31 & ~(L - 1));

  auto walk = [&](const T* src, T* dst, int64_t hs, int64_t rs, int64_t ohs, int64_t ors, const float* weight, int a, int b, bool loaded) {
    // out[i] = x[i] c[i] + x[partner] s[i], with the weights of the elements it takes
    uint64_t ce[V], co[V], se[V], so[V];
    int partner[kHalves ? E : 1];  // where an element's partner lies in the rows of row_s
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float c[4], s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = lane * E + 4 * v + i;
        int other = e ^ 1;
        if (kHalves) {
          int pair;
          bool first;
          place(g, e, pair, other, first);
          partner[4 * v + i] = grp * D + other;
          const float2 cs = pair >= 0 ? cs_s[t * (D / 2) + pair] : make_float2(1.f, 0.f);
          c[i] = cs.x;
          s[i] = first ? -cs.y : cs.y;
        } else {
          const float2 cs = cs_s[t * (D / 2) + e / 2];
          c[i] = cs.x;
          s[i] = i & 1 ? cs.y : -cs.y;
        }
        if (weight && g.norm) {
          c[i] *= weight[e];
          s[i] *= weight[other];
        }
        if (kPass && e >= turning) s[i] = -0.f;
      }
      ce[v] = pack2(c[0], c[2]);
      co[v] = pack2(c[1], c[3]);
      se[v] = pack2(s[0], s[2]);
      so[v] = pack2(s[1], s[3]);
    }
    const T* in = src + (int64_t)n * rs + lane * E + a * hs;
    T* out = dst + (int64_t)n * ors + lane * E + a * ohs;
    for (int h = a; h < b; h += kUnroll, in += kUnroll * hs, out += kUnroll * ohs) {
      if (h > a || !loaded) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (h + u < b) raw[u] = *reinterpret_cast<const uint4*>(in + u * hs);
      }
      if (kHalves) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (h + u < b) *reinterpret_cast<uint4*>(&row_s[(u * G + grp) * D + lane * E]) = raw[u];
        __syncwarp(mask);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (h + u >= b) break;
        uint64_t e[V], o[V], pe[V], po[V];
        P::split(raw[u], e, o);
        if (kHalves) {
          const T* row = &row_s[u * G * D];
#pragma unroll
          for (int v = 0; v < V; ++v) {
            pe[v] = pack2(fc::to_float<T>(row[partner[4 * v]]), fc::to_float<T>(row[partner[4 * v + 2]]));
            po[v] = pack2(fc::to_float<T>(row[partner[4 * v + 1]]), fc::to_float<T>(row[partner[4 * v + 3]]));
          }
        }
        uint64_t r2 = pack2(1.f, 1.f);
        if (g.norm) {
          uint64_t sum2 = mul2(e[0], e[0]);
          sum2 = fma2(o[0], o[0], sum2);
#pragma unroll
          for (int v = 1; v < V; ++v) sum2 = fma2(o[v], o[v], fma2(e[v], e[v], sum2));
          float sum, other;
          unpack2(sum2, sum, other);
          sum += other;
#pragma unroll
          for (int k = 1; k < L; k <<= 1) sum += __shfl_xor_sync(mask, sum, k);
          const float r = rsqrtf(fmaf(sum, 1.f / D, g.eps));
          r2 = pack2(r, r);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          uint64_t p0 = kHalves ? pe[v] : o[v], p1 = kHalves ? po[v] : e[v];  // the partners
          if (kPass) {  // what passes through gets a partner of 0 in place of a perhaps infinite one: 0 times -0 adds nothing, even to a -0
            const bool k0 = lane * E + 4 * v < turning, k1 = lane * E + 4 * v + 2 < turning;
            float a[4];
            unpack2(p0, a[0], a[1]);
            unpack2(p1, a[2], a[3]);
            p0 = pack2(k0 ? a[0] : 0.f, k1 ? a[1] : 0.f);
            p1 = pack2(k0 ? a[2] : 0.f, k1 ? a[3] : 0.f);
          }
          const uint64_t y0 = fma2(e[v], ce[v], mul2(p0, se[v]));
          const uint64_t y1 = fma2(o[v], co[v], mul2(p1, so[v]));
          e[v] = mul2(y0, r2);
          o[v] = mul2(y1, r2);
        }
        *reinterpret_cast<uint4*>(out + u * ohs) = P::join(e, o);
      }
      if (kHalves) __syncwarp(mask);
    }
  };
  if (h0 < g.H_q) walk(Q, Q_out, g.q_hs, g.q_rs, g.qo_hs, g.qo_rs, q_weight, h0, min(h1, g.H_q), true);
  if (h1 > g.H_q) walk(K, K_out, g.k_hs, g.k_rs, g.ko_hs, g.ko_rs, k_weight, max(h0 - g.H_q, 0), h1 - g.H_q, h0 >= g.H_q);
}

// f radians per position -> turns per position modulo one, times 2^64
uint64_t turns_of(long double f) {
  long double t = f * 0.159154943091895335768883763372514362L;
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
    if (!pos && desc->T > 0) {  // no tokens, no places: their array may well be NULL
      if (desc->grid_h <= 0 || desc->grid_w <= 0) return FC_ERR_INVALID_ARG;
      const int64_t frame = (int64_t)desc->grid_h * desc->grid_w;
      if (frame > INT32_MAX || desc->grid_t0 + (int64_t)(desc->T - 1) / frame > INT32_MAX) return FC_ERR_INVALID_ARG;
    }
    int k = 0;
    for (int a = 0; a < 3; ++a) {
      const int half = desc->axis_dim[a] / 2;
      // theta^(-2i/n) as powers of one ratio: 64 bits of mantissa leave 58 after as many products
      const long double ratio = inv_freq || half == 0 ? 0.0L : powl(desc->theta, -1.0L / half);
      long double f = 1.0L;
      for (int i = 0; i < half; ++i, ++k, f *= ratio) {
        if (inv_freq) f = inv_freq[k];
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
    if ((x.heads > 1 && x.s[2] < desc->d) || (desc->T > 1 && x.s[3] < desc->d)) return FC_ERR_INVALID_ARG;  // rows would overlap
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
  // A group of lanes takes as many heads as leave the device half a set of resident groups (more heads amortise the group's
  // constants, fewer leave loads in flight); a lone token gets a group per head.  A block then takes as few tokens as its groups
  // have use for.
  const int lanes = desc->d * es / 16, groups = kThreads / lanes;
  const int64_t resident = (int64_t)ctx->sm_count * 1024 / lanes;
  int64_t per = heads * desc->T / resident;
  per = per < 1 ? 1 : per > heads ? heads : per;
  int parts = 1;  // of the heads, in a block
  while (parts < groups && parts * per < heads) parts *= 2;
  while (groups / parts > 1 && groups / parts / 2 >= desc->T) parts *= 2;
  if (parts * per >= heads) per = (heads + parts - 1) / parts;  // the same number for every group
  g.tokens = groups / parts;
  g.heads_per_group = (int32_t)per;
  const int64_t blocks = ((int64_t)desc->T + g.tokens - 1) / g.tokens, splits = (heads + parts * per - 1) / (parts * per);
  if (splits > 65535) return FC_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)blocks, (unsigned)splits);
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
#define FC_ROPE_LAUNCH(T, D, HALVES)                                                                                     \
  do {                                                                                                                   \
    auto kernel = turning < D ? qk_norm_rope_kernel<T, D, HALVES, true> : qk_norm_rope_kernel<T, D, HALVES, false>;      \
    kernel<<<grid, kThreads, 0, st>>>((const T*)Q, (const T*)K, (T*)Q_out, (T*)K_out, q_weight, k_weight, pos, g);       \
  } while (0)
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
