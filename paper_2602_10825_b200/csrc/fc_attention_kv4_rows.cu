// Attention of few query rows over [4-bit clean region | window], bf16: one pass over the keys, cut into parts that a
// second kernel joins.
//
// Bound by the bytes of the clean region and, next to it, by the issue slots that unpacking takes: 4.5 bits an element leave an
// SM about 46 elements per clock to unpack at the copy rate.  So nothing goes through shared memory: a warp loads the codes
// of 16 keys straight into the registers of its tensor-core operands, and every element costs about 1.6 instructions.
//   S^T = K Q^T   m16n8k16, keys as rows, up to 8 NT query rows as columns.  The order of the head's elements along the
//                 contraction is free as long as K and Q agree: lane (key, q) takes elements [q D/4, (q+1) D/4) of its key, which
//                 is one load and one scale.
//   O^T = V^T P^T dims as rows.  Again the order of the rows is free: lane (n, q) takes dims [n D/8, (n+1) D/8) of keys 2q,
//                 2q+1, 2q+8, 2q+9; the codes of two keys are brought into one register before they are unpacked, so that
//                 the pair along the contraction is a pair of 16-bit halves.
// P^T goes from the accumulator layout of the first product to the operand layout of the second by movmatrix.
// The maximum is lazy (it moves when a logit passes it by 2^8), so that the usual step has no shuffles and no rescaling.
// The four warps of a block take 16-key steps in turn and join their sums through shared memory at the end.
#include <algorithm>
#include <cmath>

#include "fc_attention_kv4.cuh"
#include "fc_tcgen05.cuh"

namespace {

using namespace fc::sm100;  // ex2, cvt_bf16x2, max3

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStep = 16;  // keys per warp and step
constexpr float kRescaleThreshold = 8.f;

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// The operands of one step as they lie in memory.
template <int D> struct Raw {
  static constexpr int WK = D / 32, WV = D / 64;  // words of codes per lane and key
  uint32_t k[2][WK], ks[2], v[4][WV], vs[4];
};

template <int N> __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(p));
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else if constexpr (N == 2) {
    const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
    w[0] = x.x; w[1] = x.y;
  } else {
    w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
  }
}

// What a warp carries along its keys: O^T, the maxima (log2 units) and this lane's share of the sums.
template <int D, int NT> struct State {
  float o[NT][D / 16][4];
  float m[NT][2], l[NT][2];
};

// S^T (log2 units, masked) -> P^T operands; moves the maxima where they have to move.
template <int D, int NT>
__device__ __forceinline__ void softmax_step(State<D, NT>& st, float (&s)[NT][4], float scale_log2, int lane, int n_valid,
                                             uint32_t (&p0)[NT], uint32_t (&p1)[NT]) {
  bool move = false;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[t][i] *= scale_log2;
      if (n_valid < kStep && (lane >> 2) + (i >= 2 ? 8 : 0) >= n_valid) s[t][i] = -INFINITY;
    }
    move |= fmaxf(s[t][0], s[t][2]) > st.m[t][0] + kRescaleThreshold;
    move |= fmaxf(s[t][1], s[t][3]) > st.m[t][1] + kRescaleThreshold;
  }
  if (__any_sync(0xffffffffu, move)) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float x = fmaxf(s[t][r], s[t][2 + r]);
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
        if (x > st.m[t][r] + kRescaleThreshold) {
          const float alpha = ex2(st.m[t][r] - x);  // 0 the first time
          st.m[t][r] = x;
          st.l[t][r] *= alpha;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            st.o[t][j][r] *= alpha;
            st.o[t][j][2 + r] *= alpha;
          }
        }
      }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    // a row all of whose logits so far are -inf has no maximum yet: its weights are 0 (or NaN, where a logit is)
    const float m0 = st.m[t][0] == -INFINITY ? 0.f : st.m[t][0], m1 = st.m[t][1] == -INFINITY ? 0.f : st.m[t][1];
    const float e0 = ex2(s[t][0] - m0), e1 = ex2(s[t][1] - m1), e2 = ex2(s[t][2] - m0), e3 = ex2(s[t][3] - m1);
    st.l[t][0] += e0 + e2;
    st.l[t][1] += e1 + e3;
    p0[t] = transpose8x8(cvt_bf16x2(e0, e1));
    p1[t] = transpose8x8(cvt_bf16x2(e2, e3));
  }
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 4 : 3)
attention_kv4_rows_kernel(const __nv_bfloat16* __restrict__ Q, const __nv_bfloat16* __restrict__ K,
                          const __nv_bfloat16* __restrict__ V, __nv_bfloat16* __restrict__ O,
                          const __grid_constant__ fc::Kv4AttnGeom g) {
  constexpr int kRows = 8 * NT, kLaneDims = D / 4, kLaneCols = D / 8;
  __shared__ float o_s[kWarps][kRows][D + 4];
  __shared__ float2 ml_s[kWarps][kRows];
  const fc::AttnGeom& a = g.a;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, n = lane >> 2, q = lane & 3;
  const int part = blockIdx.x, hk = blockIdx.y;
  int v0 = 0;
  const int c = fc::tile_chunk<kRows>(a, blockIdx.z, v0);
  if (part == 0 && hk == 0 && blockIdx.z == 0 && tid == 0) fc::report_bad_ids(a);
  if (c < 0 || !fc::chunk_active(a, c)) return;
  const int rows_here = min(kRows, (a.q_row_off[c + 1] - a.q_row_off[c]) * a.group - v0);

  // keys of this part: of the clean region, or of the window
  const bool window = part >= g.cache_parts;
  int k0, k1;
  if (!window) {
    k0 = part * g.part_keys;
    k1 = (int)min((int64_t)k0 + g.part_keys, (int64_t)min(g.n_cache, a.vis[c]));
  } else {
    k0 = (part - g.cache_parts) * g.window_part_keys;
    k1 = (int)min((int64_t)k0 + g.window_part_keys, (int64_t)a.vis[c] - g.n_cache);
  }

  uint32_t qb[NT][kLaneDims / 2];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = 8 * t + n;
#pragma unroll
    for (int i = 0; i < kLaneDims / 8; ++i) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (r < rows_here) {
        const int v = v0 + r;
        const __nv_bfloat16* src = Q + (int64_t)(hk * a.group + v % a.group) * a.q_hs + (int64_t)(a.q_row_off[c] + v / a.group) * a.q_rs;
        x = *reinterpret_cast<const uint4*>(src + q * kLaneDims + 8 * i);
      }
      qb[t][4 * i] = x.x; qb[t][4 * i + 1] = x.y; qb[t][4 * i + 2] = x.z; qb[t][4 * i + 3] = x.w;
    }
  }
  State<D, NT> st;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) st.o[t][j][0] = st.o[t][j][1] = st.o[t][j][2] = st.o[t][j][3] = 0.f;
    st.m[t][0] = st.m[t][1] = -INFINITY;
    st.l[t][0] = st.l[t][1] = 0.f;
  }
  const float scale_log2 = a.scale * 1.4426950408889634f;

  if (!window) {
    const uint8_t* kc = g.cache.k_codes + hk * g.cache.code_hs + q * (kLaneDims / 2);
    const uint8_t* vc = g.cache.v_codes + hk * g.cache.code_hs + n * (kLaneCols / 2);
    const uint16_t* ks = g.cache.k_scales + hk * g.cache.scale_hs + q * kLaneDims / 32;
    const uint16_t* vs = g.cache.v_scales + hk * g.cache.scale_hs + n * kLaneCols / 32;
    // positions behind the last key repeat it: their weights are zero
    auto load = [&](int kb, Raw<D>& r) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int64_t j = min(kb + 8 * t + n, k1 - 1);
        load_words(kc + j * g.cache.code_rs, r.k[t]);
        r.ks[t] = __ldg(ks + j * g.cache.scale_rs);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t j = min(kb + 2 * q + (i & 1) + 8 * (i >> 1), k1 - 1);
        load_words(vc + j * g.cache.code_rs, r.v[i]);
        r.vs[i] = __ldg(vs + j * g.cache.scale_rs);
      }
    };
    Raw<D> next;
    int kb = k0 + kStep * warp;
    if (kb < k1) load(kb, next);
    for (; kb < k1; kb += kStep * kWarps) {
      const Raw<D> r = next;
      if (kb + kStep * kWarps < k1) load(kb + kStep * kWarps, next);
      float s[NT][4] = {};
      {
        const uint32_t s0 = fc::kv4_scale2(r.ks[0]), s1 = fc::kv4_scale2(r.ks[1]);
        const uint32_t b0 = fc::kv4_bias2(s0), b1 = fc::kv4_bias2(s1);
#pragma unroll
        for (int w = 0; w < Raw<D>::WK; ++w) {
          uint32_t x[4], y[4];
          fc::kv4_word(r.k[0][w], s0, b0, x);
          fc::kv4_word(r.k[1][w], s1, b1, y);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            mma(s[t], x[0], y[0], x[1], y[1], qb[t][4 * w], qb[t][4 * w + 1]);
            mma(s[t], x[2], y[2], x[3], y[3], qb[t][4 * w + 2], qb[t][4 * w + 3]);
          }
        }
      }
      uint32_t p0[NT], p1[NT];
      softmax_step<D, NT>(st, s, scale_log2, lane, k1 - kb, p0, p1);
      const uint32_t sl = r.vs[0] | (r.vs[1] << 16), sh = r.vs[2] | (r.vs[3] << 16);
      const uint32_t bl = fc::kv4_bias2(sl), bh = fc::kv4_bias2(sh);
#pragma unroll
      for (int w = 0; w < Raw<D>::WV; ++w) {
        uint32_t el[4], ol[4], eh[4], oh[4];  // even and odd elements, low and high keys
        fc::kv4_word(prmt(r.v[0][w], r.v[1][w], 0x5410), sl, bl, el);
        fc::kv4_word(prmt(r.v[0][w], r.v[1][w], 0x7632), sl, bl, ol);
        fc::kv4_word(prmt(r.v[2][w], r.v[3][w], 0x5410), sh, bh, eh);
        fc::kv4_word(prmt(r.v[2][w], r.v[3][w], 0x7632), sh, bh, oh);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int t = 0; t < NT; ++t) mma(st.o[t][4 * w + i], el[i], ol[i], eh[i], oh[i], p0[t], p1[t]);
      }
    }
  } else {
    const __nv_bfloat16* kp = K + hk * a.k_hs + q * kLaneDims;
    const __nv_bfloat16* vp = V + hk * a.v_hs + n * kLaneCols;
    for (int kb = k0 + kStep * warp; kb < k1; kb += kStep * kWarps) {
      float s[NT][4] = {};
      {
        const __nv_bfloat16* r0 = kp + fc::window_row(a, min(kb + n, k1 - 1)) * a.k_rs;
        const __nv_bfloat16* r1 = kp + fc::window_row(a, min(kb + 8 + n, k1 - 1)) * a.k_rs;
#pragma unroll
        for (int i = 0; i < kLaneDims / 8; ++i) {
          const uint4 x = *reinterpret_cast<const uint4*>(r0 + 8 * i), y = *reinterpret_cast<const uint4*>(r1 + 8 * i);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            mma(s[t], x.x, y.x, x.y, y.y, qb[t][4 * i], qb[t][4 * i + 1]);
            mma(s[t], x.z, y.z, x.w, y.w, qb[t][4 * i + 2], qb[t][4 * i + 3]);
          }
        }
      }
      uint32_t p0[NT], p1[NT];
      softmax_step<D, NT>(st, s, scale_log2, lane, k1 - kb, p0, p1);
      const __nv_bfloat16* r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = vp + fc::window_row(a, min(kb + 2 * q + (i & 1) + 8 * (i >> 1), k1 - 1)) * a.v_rs;
#pragma unroll
      for (int w = 0; w < kLaneCols / 8; ++w) {
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const uint4*>(r[i] + 8 * w);
        const uint32_t* y[4] = {&x[0].x, &x[1].x, &x[2].x, &x[3].x};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int t = 0; t < NT; ++t)
            mma(st.o[t][4 * w + i], prmt(y[0][i], y[1][i], 0x5410), prmt(y[0][i], y[1][i], 0x7632), prmt(y[2][i], y[3][i], 0x5410),
                prmt(y[2][i], y[3][i], 0x7632), p0[t], p1[t]);
      }
    }
  }

  // join the four warps
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float l = st.l[t][r];
      l += __shfl_xor_sync(0xffffffffu, l, 4);
      l += __shfl_xor_sync(0xffffffffu, l, 8);
      l += __shfl_xor_sync(0xffffffffu, l, 16);
      const int row = 8 * t + 2 * q + r;
      if (n == 0) ml_s[warp][row] = make_float2(st.m[t][r], l);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        o_s[warp][row][n * kLaneCols + 2 * j] = st.o[t][j][r];
        o_s[warp][row][n * kLaneCols + 2 * j + 1] = st.o[t][j][2 + r];
      }
    }
  __syncthreads();
  const bool last = g.n_splits == 1;
  for (int x = tid; x < rows_here * (D / 4); x += kThreads) {
    const int row = x / (D / 4), d4 = x % (D / 4) * 4;
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, ml_s[w][row].x);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float2 ml = ml_s[w][row];
      if (!(ml.y != 0.f)) continue;
      const float f = ex2(ml.x - m);
      const float4 y = *reinterpret_cast<const float4*>(&o_s[w][row][d4]);
      l = fmaf(f, ml.y, l);
      o.x = fmaf(f, y.x, o.x); o.y = fmaf(f, y.y, o.y); o.z = fmaf(f, y.z, o.z); o.w = fmaf(f, y.w, o.w);
    }
    const int v = v0 + row;
    if (!last) {
      const int64_t vr = (int64_t)(a.q_row_off[c] - a.q_row_off[0]) * a.group + v;
      const int64_t at = (hk * g.n_vrows + vr) * g.n_splits + part;
      *reinterpret_cast<float4*>(g.part_o + at * D + d4) = o;
      if (d4 == 0) g.part_ml[at] = make_float2(m, l);
    } else {
      const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
      const int h = hk * a.group + v % a.group;
      const int64_t rowg = a.q_row_off[c] + v / a.group;
      *reinterpret_cast<uint2*>(O + h * a.o_hs + rowg * a.o_rs + d4) =
          make_uint2(cvt_bf16x2(o.x * inv, o.y * inv), cvt_bf16x2(o.z * inv, o.w * inv));
      if (a.lse && d4 == 0) a.lse[h * a.lse_hs + rowg] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : (l == l ? -INFINITY : l);
    }
  }
}

// Rows per tile: eight where no chunk has more, else sixteen.
int tiles_of(const fc::Kv4AttnGeom& g) {
  for (int c = 0; c < g.a.W; ++c)
    if ((int64_t)(g.a.q_row_off[c + 1] - g.a.q_row_off[c]) * g.a.group > 8) return 2;
  return 1;
}

}  // namespace

namespace fc {

size_t kv4_rows_workspace(const fc_ctx* ctx, Kv4AttnGeom& g) {
  int vis = 0;
  for (int c = 0; c < g.a.W; ++c) vis = std::max(vis, g.a.vis[c]);
  const int nt = tiles_of(g);
  const int64_t tiles = tile_count(g.a, 8 * nt) * g.a.H_kv;
  const int64_t cache = std::min(vis, g.n_cache), window = std::max(vis - g.n_cache, 0);
  // One set of resident blocks, shared out by what a key costs: a window key has 3.6 times the bytes of a packed one.  At least
  // two steps of every warp in a part.
  constexpr int64_t kWindowCost = 3, kLeast = 2 * kStep * kWarps;
  const int64_t work = cache + kWindowCost * window;
  const int64_t slots = std::max<int64_t>(1, (int64_t)ctx->sm_count * (nt == 1 ? 4 : 3) / std::max<int64_t>(1, tiles));
  int64_t per = std::max(kLeast, (work + slots - 1) / slots);
  per = (per + kStep * kWarps - 1) / (kStep * kWarps) * (kStep * kWarps);
  const int64_t wper = std::max<int64_t>(kStep * kWarps, per / kWindowCost / (kStep * kWarps) * (kStep * kWarps));
  g.part_keys = (int32_t)std::min<int64_t>(per, INT32_MAX / 2);
  g.window_part_keys = (int32_t)std::min<int64_t>(wper, INT32_MAX / 2);
  g.cache_parts = (int32_t)((cache + g.part_keys - 1) / g.part_keys);
  g.n_splits = (int32_t)std::max<int64_t>(1, g.cache_parts + (window + g.window_part_keys - 1) / g.window_part_keys);
  if (g.n_splits == 1) return 0;
  const int64_t parts = g.a.H_kv * g.n_vrows * g.n_splits;
  return align_up(parts * g.a.d * sizeof(float), 256) + align_up(parts * sizeof(float2), 256);
}

int kv4_rows(cudaStream_t st, const Kv4AttnGeom& g, const void* Q, const void* K, const void* V, void* O) {
  const int nt = tiles_of(g);
  const int64_t tiles = tile_count(g.a, 8 * nt);
  if (tiles == 0) return FC_OK;
  if (tiles > 65535) return FC_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)g.n_splits, (unsigned)g.a.H_kv, (unsigned)tiles);
#define FC_KV4_ROWS(D, NT)                                                                                              \
  attention_kv4_rows_kernel<D, NT><<<grid, kThreads, 0, st>>>((const __nv_bfloat16*)Q, (const __nv_bfloat16*)K,         \
                                                              (const __nv_bfloat16*)V, (__nv_bfloat16*)O, g)
  if (g.a.d == 128) { if (nt == 1) FC_KV4_ROWS(128, 1); else FC_KV4_ROWS(128, 2); }
  else { if (nt == 1) FC_KV4_ROWS(64, 1); else FC_KV4_ROWS(64, 2); }
#undef FC_KV4_ROWS
  FC_LAUNCH_CHECK("attention_kv4_rows_kernel");
  return g.n_splits > 1 ? kv4_combine(st, g, FC_BF16, O, true) : FC_OK;
}

}  // namespace fc
