// Attention of few query rows over [4-bit clean region | window]: one pass over the keys, cut into parts that a second kernel
// joins; also the path of fp32 tensors whatever their rows.
//
// Bound by the bytes of the clean region and, next to it, by the issue slots that unpacking takes: 4.5 bits an element leave an
// SM about 46 elements per clock to unpack at the copy rate.  So a warp takes the codes of 16 keys from its own ring in shared
// memory (cp.async, three steps ahead) straight into the registers of its tensor-core operands, at about 1.6 instructions an element.
//   S^T = K Q^T   m16n8k16, keys as rows, up to 8 NT query rows as columns.  The order of the head's elements along the
//                 contraction is free as long as K and Q agree: lane (key, q) takes elements [q D/4, (q+1) D/4) of its key, which
//                 is one access and one scale.
//   O^T = V^T P^T dims as rows.  Again the order of the rows is free: lane (n, q) takes dims [n D/8, (n+1) D/8) of keys 2q,
//                 2q+1, 2q+8, 2q+9; the codes of two keys are brought into one register before they are unpacked, so that
//                 the pair along the contraction is a pair of 16-bit halves.
// P^T goes from the accumulator layout of the first product to the operand layout of the second by movmatrix.
// The maximum is lazy (it moves when a logit passes it by 2^8), so that the usual step has no shuffles and no rescaling.
// The four warps of a block take 16-key steps in turn and join their sums through shared memory at the end.
//
// fp32.  A 24-bit number is exactly the sum of three bf16 numbers, and an unpacked key is exactly one.  So Q K^T over the clean
// region is three products of bf16 numbers, each exact before it is added in fp32, and so is P V.  Over an fp32 window six
// of the nine products of parts are taken.  The parts are rounded to nearest, so that the second is at most 2^-8 of the number and the third 2^-17,
// and what is left out, 2^-24 of the product at most and of either sign (parts that are cut off leave out up to 2^-21, always of the product's
// sign, and save 0 to 2 % of the time: 600 rows of 8 heads of 128 over 1900 keys and the window 121.2 us, rounded 123.2).
// The tensor core cuts, rather than rounds, what it adds up; so the small parts have accumulators of their own, and O is added up
// outside, step by step.
#include <algorithm>
#include <cmath>

#include "fc_attention_kv4.cuh"
#include "fc_mma_sync.cuh"

namespace {

using namespace fc::sm100;  // mma and its operands, ex2, cvt_bf16x2, max3

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStep = 16;  // keys per warp and step
constexpr float kRescaleThreshold = 8.f;
constexpr int kWindowCost = 3;  // a window key has 3.6 times the bytes of a packed one in bf16, 7.1 times in fp32; nothing is unpacked
// Resident blocks, by the registers the kernel is given (measured: three and two are as fast as four and three at one token, and
// faster at 64 rows of 24 heads over 28064 keys, 110 us against 125 before a step's products were moved up).
constexpr int blocks_per_sm(int nt) { return nt == 1 ? 3 : 2; }

template <typename T> constexpr int kParts = sizeof(T) == 4 ? 3 : 1;  // of Q, and of a window's K and V
// Of P.  bf16 rounds a weight by up to 2^-8, which is as much again as the output's own rounding: of up to eight rows, bound by
// the unpacking, the rest of the weight is taken along (one token over 28080 keys: 32.5 us against 31.0, error 1.7e-3 against 2.4e-3);
// of sixteen it would cost 20 to 25 %.
template <typename T, int NT> constexpr int kWeightParts = sizeof(T) == 4 ? 3 : (NT == 1 ? 2 : 1);

// A warp's ring of 16-key steps in shared memory, filled by cp.async: the codes of K and V, then their scales.
template <int D> struct Ring {
  static constexpr int kCodes = kStep * D / 2, kScales = kStep * D / 16;  // bytes of one tensor's step
  static constexpr int kBytes = 2 * (kCodes + kScales);
  static constexpr int kStages = 4;
};

// The window's keys in the place of the ring: 16 rows of K and 16 of V.  K of the next step is on its way while V of this one is
// worked on, and the other way round.
template <typename T, int D> struct Window {
  static constexpr int kRow = D * (int)sizeof(T), kBytes = kStep * kRow, kPieces = kRow / 16;
  // Where 16-byte piece p of row r lies in its row, so that the eight lanes that are served together read different banks.
  static __device__ __forceinline__ int k_piece(int r, int p) {
    return kPieces == 32 ? p ^ ((p >> 3) & 3) ^ ((r & 1) << 2) : p ^ ((p >> 3) & 1) ^ ((r & 1) << 1);
  }
  static __device__ __forceinline__ int v_piece(int r, int p) {
    return kPieces == 32 ? p ^ ((r >> 1) & 3) : p ^ (((r >> 1) & 3) << 1) ^ ((p >> 1) & 1);
  }
};
// Shared memory of a warp: the ring or the window's rows; of a block: also, after the last step, what the warps join.
template <typename T, int D> constexpr int kWarpBytes =
    Ring<D>::kStages * Ring<D>::kBytes > 2 * Window<T, D>::kBytes ? Ring<D>::kStages * Ring<D>::kBytes : 2 * Window<T, D>::kBytes;
template <typename T, int D, int NT> constexpr int kBlockBytes =
    kWarps * (kWarpBytes<T, D> > 8 * NT * (D + 4) * 4 ? kWarpBytes<T, D> : 8 * NT * (D + 4) * 4);

template <int N> __device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// N words of shared memory in one access
template <int N> __device__ __forceinline__ void lds_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x; w[1] = x.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// What a warp carries along its keys: O^T, this lane's share of the sums, and per row the reference of its exponents (log2
// units) with the logit (as the product gives it) above which the reference moves.  A row that has met no finite logit yet has
// move_at = -inf and the reference 0: weights of -inf are 0 then, and a NaN stays one.
template <int D, int NT> struct State {
  float o[NT][D / 16][4];
  float l[NT][2], ref[NT][2], move_at[NT][2];
};

// S^T -> P^T operands, in two halves: the maxima (n_valid: keys of the step that exist, kTail only), and the weights.
template <int D, int NT, bool kTail>
__device__ __forceinline__ void move_maximum(State<D, NT>& st, float (&s)[NT][4], float scale_log2, int lane, int n_valid) {
  bool move = false;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (kTail) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((lane >> 2) + (i >= 2 ? 8 : 0) >= n_valid) s[t][i] = -INFINITY;
    }
    move |= fmaxf(s[t][0], s[t][2]) > st.move_at[t][0];
    move |= fmaxf(s[t][1], s[t][3]) > st.move_at[t][1];
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
        if (x > st.move_at[t][r]) {
          const float ref = x * scale_log2;
          const float alpha = st.move_at[t][r] == -INFINITY ? 0.f : ex2(st.ref[t][r] - ref);
          st.ref[t][r] = ref;
          st.move_at[t][r] = x + kRescaleThreshold / scale_log2;
          st.l[t][r] *= alpha;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            st.o[t][j][r] *= alpha;
            st.o[t][j][2 + r] *= alpha;
          }
        }
      }
  }
}
template <typename T, int D, int NT>
__device__ __forceinline__ void weights(State<D, NT>& st, const float (&s)[NT][4], float scale_log2,
                                        uint32_t (&p0)[kWeightParts<T, NT>][NT], uint32_t (&p1)[kWeightParts<T, NT>][NT]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float e0 = ex2(fmaf(s[t][0], scale_log2, -st.ref[t][0])), e1 = ex2(fmaf(s[t][1], scale_log2, -st.ref[t][1]));
    const float e2 = ex2(fmaf(s[t][2], scale_log2, -st.ref[t][0])), e3 = ex2(fmaf(s[t][3], scale_log2, -st.ref[t][1]));
    st.l[t][0] += e0 + e2;
    st.l[t][1] += e1 + e3;
    if constexpr (kParts<T> == 1) {
      const uint32_t a = cvt_bf16x2(e0, e1), b = cvt_bf16x2(e2, e3);
      p0[0][t] = transpose8x8(a);
      p1[0][t] = transpose8x8(b);
      if constexpr (kWeightParts<T, NT> == 2) {
        p0[1][t] = transpose8x8(cvt_bf16x2(e0 - fc::bf16_lo(a), e1 - fc::bf16_hi(a)));
        p1[1][t] = transpose8x8(cvt_bf16x2(e2 - fc::bf16_lo(b), e3 - fc::bf16_hi(b)));
      }
    } else {
      uint32_t a[3], b[3];
      parts_of(e0, e1, a);
      parts_of(e2, e3, b);
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        p0[i][t] = transpose8x8(a[i]);
        p1[i][t] = transpose8x8(b[i]);
      }
    }
  }
}

// S^T += K Q^T over 16 elements of the head, K as NK parts of operand registers: s the largest products, rest the others.
template <typename T, int D, int NT, int NK>
__device__ __forceinline__ void logits(float (&s)[NT][4], float (&rest)[NT][4], const uint32_t (&k)[NK][4],
                                       const uint32_t (&qb)[kParts<T>][NT][D / 8], int at) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int i = NK - 1; i >= 0; --i)
#pragma unroll
      for (int j = kParts<T> - 1; j >= 0; --j)
        if (i + j < 3) mma(i + j == 0 ? s[t] : rest[t], k[i][0], k[i][1], k[i][2], k[i][3], qb[j][t][at], qb[j][t][at + 1]);
  }
}
// O^T tile += V^T P^T, V as NV parts.
template <typename T, int NT, int NV>
__device__ __forceinline__ void weigh(float (&o)[4], const uint32_t (&v)[NV][4], const uint32_t (&p0)[kWeightParts<T, NT>][NT],
                                      const uint32_t (&p1)[kWeightParts<T, NT>][NT], int t) {
  if constexpr (kParts<T> == 1) {
#pragma unroll
    for (int i = kWeightParts<T, NT> - 1; i >= 0; --i) mma(o, v[0][0], v[0][1], v[0][2], v[0][3], p0[i][t], p1[i][t]);
  } else {
    float x[4] = {};
#pragma unroll
    for (int w = 2; w >= 0; --w)  // the smallest products first
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (w - i >= 0 && w - i < 3) mma(x, v[i][0], v[i][1], v[i][2], v[i][3], p0[w - i][t], p1[w - i][t]);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += x[i];
  }
}

// One step over 16 packed keys, which lie at `buf`, in two halves: S^T, and O^T += V^T P^T.
template <typename T, int D, int NT>
__device__ __forceinline__ void packed_logits(float (&s)[NT][4], const uint8_t* buf, const uint32_t (&qb)[kParts<T>][NT][D / 8], int lane) {
  using R = Ring<D>;
  const int n = lane >> 2, q = lane & 3;
  const uint8_t* kc = buf + n * (D / 2) + q * (D / 8);
  const uint16_t* ks = reinterpret_cast<const uint16_t*>(buf + 2 * R::kCodes) + n * (D / 32) + q * D / 128;
  float rest[NT][4] = {};
  uint32_t k0[D / 32], k1[D / 32];
  lds_words(kc, k0);
  lds_words(kc + 8 * (D / 2), k1);
  const uint32_t s0 = fc::kv4_scale2(ks[0]), s1 = fc::kv4_scale2(ks[8 * (D / 32)]);
  const uint32_t b0 = fc::kv4_bias2(s0), b1 = fc::kv4_bias2(s1);
#pragma unroll
  for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
  for (int w = 0; w < D / 32; ++w) {
    uint32_t x[4], y[4];
    fc::kv4_word(k0[w], s0, b0, x);
    fc::kv4_word(k1[w], s1, b1, y);
    const uint32_t lo[1][4] = {{x[0], y[0], x[1], y[1]}}, hi[1][4] = {{x[2], y[2], x[3], y[3]}};
    logits<T, D>(s, rest, lo, qb, 4 * w);
    logits<T, D>(s, rest, hi, qb, 4 * w + 2);
  }
  if constexpr (kParts<T> > 1) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] += rest[t][i];
  }
}
template <typename T, int D, int NT>
__device__ __forceinline__ void packed_weigh(State<D, NT>& st, const uint8_t* buf, const float (&s)[NT][4], float scale_log2, int lane) {
  using R = Ring<D>;
  const int n = lane >> 2, q = lane & 3;
  const uint8_t* vc = buf + R::kCodes + 2 * q * (D / 2) + n * (D / 16);
  const uint16_t* vs = reinterpret_cast<const uint16_t*>(buf + 2 * R::kCodes + R::kScales) + 2 * q * (D / 32) + n * D / 256;
  uint32_t v[4][D / 64], p0[kWeightParts<T, NT>][NT], p1[kWeightParts<T, NT>][NT];
#pragma unroll
  for (int i = 0; i < 4; ++i) lds_words(vc + ((i & 1) + 8 * (i >> 1)) * (D / 2), v[i]);
  const uint32_t sl = vs[0] | ((uint32_t)vs[D / 32] << 16), sh = vs[8 * (D / 32)] | ((uint32_t)vs[9 * (D / 32)] << 16);
  const uint32_t bl = fc::kv4_bias2(sl), bh = fc::kv4_bias2(sh);
  weights<T, D, NT>(st, s, scale_log2, p0, p1);
#pragma unroll
  for (int w = 0; w < D / 64; ++w) {
    uint32_t el[4], ol[4], eh[4], oh[4];  // even and odd elements, low and high keys
    fc::kv4_word(prmt(v[0][w], v[1][w], 0x5410), sl, bl, el);
    fc::kv4_word(prmt(v[0][w], v[1][w], 0x7632), sl, bl, ol);
    fc::kv4_word(prmt(v[2][w], v[3][w], 0x5410), sh, bh, eh);
    fc::kv4_word(prmt(v[2][w], v[3][w], 0x7632), sh, bh, oh);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x[1][4] = {{el[i], ol[i], eh[i], oh[i]}};
#pragma unroll
      for (int t = 0; t < NT; ++t) weigh<T, NT>(st.o[t][4 * w + i], x, p0, p1, t);
    }
  }
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(NT))
attention_kv4_rows_kernel(const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, T* __restrict__ O,
                          const __grid_constant__ fc::Kv4AttnGeom g) {
  constexpr int kRows = 8 * NT, kLaneDims = D / 4, kLaneCols = D / 8, kPer = 16 / (int)sizeof(T);
  using R = Ring<D>;
  using Wn = Window<T, D>;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float2 ml_s[kWarps][kRows];
  fc::pdl_launch_dependents();  // the joining kernel may take its place; it waits for this grid to end
  const fc::AttnGeom& a = g.a;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, n = lane >> 2, q = lane & 3;
  const int part = blockIdx.z, hk = blockIdx.y;
  int v0 = 0;
  const int c = fc::tile_chunk<kRows>(a, gridDim.x - 1 - blockIdx.x, v0);  // the last chunks, which see most, start first
  if (c < 0) return;
  const int rows_here = min(kRows, (a.q_row_off[c + 1] - a.q_row_off[c]) * a.group - v0);

  // The parts cut an axis of costs: the clean region's keys, then the window's at kWindowCost each.  This part's packed
  // keys are [k0, k1), its window keys [w0, w1).
  const int64_t x0 = (int64_t)part * g.part_keys, x1 = x0 + g.part_keys;
  const int cache = min(g.n_cache, a.vis[c]), behind = max(a.vis[c] - g.n_cache, 0);
  const int k0 = (int)min(x0, (int64_t)g.n_cache), k1 = (int)min(x1, (int64_t)cache);
  const int w0 = (int)min((max(x0 - g.n_cache_ceil, (int64_t)0)) / kWindowCost, (int64_t)behind);
  const int w1 = (int)min((max(x1 - g.n_cache_ceil, (int64_t)0)) / kWindowCost, (int64_t)behind);

  // A packed step's copies: lane L brings 16 bytes of rows L/4 and L/4 + 8 of the codes (D = 128), and the scales of a row of K
  // or V.  The pointers stand at the warp's next step; positions behind the part's last key repeat it.
  constexpr int kLanesPerRow = D / 32, kRowsPerCopy = 32 / kLanesPerRow, kAll = kStep * kWarps;
  const uint32_t ring = smem_u32(smem) + warp * kWarpBytes<T, D>;
  const int kb0 = k0 + kStep * warp;
  const uint8_t* codes_p = g.cache.k_codes + hk * g.cache.code_hs + (int64_t)(kb0 + lane / kLanesPerRow) * g.cache.code_rs + lane % kLanesPerRow * 16;
  const uint16_t* scales_p = (lane < 16 ? g.cache.k_scales : g.cache.v_scales) + hk * g.cache.scale_hs + (int64_t)(kb0 + lane % 16) * g.cache.scale_rs;
  const int64_t to_v = (int64_t)g.cache.v_codes - (int64_t)g.cache.k_codes;
  const uint32_t codes_s = ring + lane * 16, scales_s = ring + 2 * R::kCodes + lane * (D / 16);
  auto copy = [&](int stage, int kb) {
    const uint32_t at = codes_s + stage * R::kBytes, at_s = scales_s + stage * R::kBytes;
    if (kb + kStep <= k1) {
#pragma unroll
      for (int i = 0; i < kStep / kRowsPerCopy; ++i) {
        cp_async<16>(at + i * 512, codes_p + i * kRowsPerCopy * g.cache.code_rs);
        cp_async<16>(at + R::kCodes + i * 512, codes_p + to_v + i * kRowsPerCopy * g.cache.code_rs);
      }
      cp_async<D / 16>(at_s, scales_p);
    } else if (kb < k1) {
      const int last = k1 - 1 - kb;
#pragma unroll
      for (int i = 0; i < kStep / kRowsPerCopy; ++i) {
        const int r = lane / kLanesPerRow;
        const int64_t off = (int64_t)(min(r + i * kRowsPerCopy, last) - r) * g.cache.code_rs;
        cp_async<16>(at + i * 512, codes_p + off);
        cp_async<16>(at + R::kCodes + i * 512, codes_p + to_v + off);
      }
      cp_async<D / 16>(at_s, scales_p + (int64_t)(min(lane % 16, last) - lane % 16) * g.cache.scale_rs);
    }
    codes_p += kAll * g.cache.code_rs;
    scales_p += kAll * g.cache.scale_rs;
    cp_async_commit();
  };
  // A window step's copies of one tensor: the lanes look one row each up and pass it on.
  auto copy_window = [&](const T* base, int64_t rs, uint32_t at, int kb, bool is_v) {
    if (kb < w1) {
      const uint32_t row = (uint32_t)fc::window_row(a, min(kb + lane % 16, w1 - 1));  // below 2^32
      constexpr int kPieces = Wn::kPieces, kRowsAtOnce = 32 / kPieces;
#pragma unroll
      for (int i = 0; i < kStep / kRowsAtOnce; ++i) {
        const int r = i * kRowsAtOnce + lane / kPieces, p = lane % kPieces;
        const int64_t phys = __shfl_sync(0xffffffffu, row, r);
        cp_async<16>(at + r * Wn::kRow + 16 * (is_v ? Wn::v_piece(r, p) : Wn::k_piece(r, p)), base + phys * rs + kPer * p);
      }
    }
    cp_async_commit();
  };
  const T* kw = K + hk * a.k_hs;
  const T* vw = V + hk * a.v_hs;
  if (k0 < k1) {
#pragma unroll
    for (int i = 0; i < R::kStages; ++i) copy(i, kb0 + i * kAll);
  }
  uint32_t qb[kParts<T>][NT][kLaneDims / 2];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = 8 * t + n;
#pragma unroll
    for (int i = 0; i < kLaneDims / kPer; ++i) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (r < rows_here) {
        const int v = v0 + r;
        const T* src = Q + (int64_t)(hk * a.group + v % a.group) * a.q_hs + (int64_t)(a.q_row_off[c] + v / a.group) * a.q_rs;
        x = *reinterpret_cast<const uint4*>(src + q * kLaneDims + kPer * i);
      }
      if constexpr (kParts<T> == 1) {
        qb[0][t][4 * i] = x.x; qb[0][t][4 * i + 1] = x.y; qb[0][t][4 * i + 2] = x.z; qb[0][t][4 * i + 3] = x.w;
      } else {
        uint32_t lo[3], hi[3];
        parts_of(__uint_as_float(x.x), __uint_as_float(x.y), lo);
        parts_of(__uint_as_float(x.z), __uint_as_float(x.w), hi);
#pragma unroll
        for (int j = 0; j < 3; ++j) qb[j][t][2 * i] = lo[j], qb[j][t][2 * i + 1] = hi[j];
      }
    }
  }
  // everything up to here reads only what the host knows; the list is on the device
  if (part == 0 && hk == 0 && blockIdx.x == 0 && tid == 0) fc::report_bad_ids(a);
  if (!fc::chunk_active(a, c)) {
    cp_async_wait<0>();
    return;
  }

  State<D, NT> st;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) st.o[t][j][0] = st.o[t][j][1] = st.o[t][j][2] = st.o[t][j][3] = 0.f;
    st.l[t][0] = st.l[t][1] = st.ref[t][0] = st.ref[t][1] = 0.f;
    st.move_at[t][0] = st.move_at[t][1] = -INFINITY;
  }
  const float scale_log2 = a.scale * 1.4426950408889634f;

  const uint8_t* buf = smem + warp * kWarpBytes<T, D>;
  if (k0 < k1) {
    // The products of one step with the keys come between the maxima of the step before and its weights, so that the two
    // steps' chains of instructions fill each other's gaps.
    int stage = 0, kb = kb0;
    float s[NT][4], s_next[NT][4];
    auto at = [&](int step) { return buf + (stage + step) % R::kStages * R::kBytes; };
    auto done = [&]() {  // the step's place has been read by every lane: another step is sent for
      __syncwarp();
      copy(stage, kb + R::kStages * kAll);
      stage = (stage + 1) % R::kStages;
      kb += kAll;
    };
    if (kb + kStep <= k1) {
      cp_async_wait<R::kStages - 1>();
      __syncwarp();
      packed_logits<T, D, NT>(s, at(0), qb, lane);
      for (; kb + kAll + kStep <= k1;) {
        move_maximum<D, NT, false>(st, s, scale_log2, lane, kStep);
        cp_async_wait<R::kStages - 2>();
        __syncwarp();
        packed_logits<T, D, NT>(s_next, at(1), qb, lane);
        packed_weigh<T, D, NT>(st, at(0), s, scale_log2, lane);
        done();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][i] = s_next[t][i];
      }
      move_maximum<D, NT, false>(st, s, scale_log2, lane, kStep);
      packed_weigh<T, D, NT>(st, at(0), s, scale_log2, lane);
      done();
    }
    cp_async_wait<0>();
    __syncwarp();
    if (kb < k1) {
      packed_logits<T, D, NT>(s, at(0), qb, lane);
      move_maximum<D, NT, true>(st, s, scale_log2, lane, k1 - kb);
      packed_weigh<T, D, NT>(st, at(0), s, scale_log2, lane);
      __syncwarp();
    }
  }
  if (w0 < w1) {
    const int wb0 = w0 + kStep * warp;
    copy_window(kw, a.k_rs, ring, wb0, false);
    copy_window(vw, a.v_rs, ring + Wn::kBytes, wb0, true);
    for (int kb = wb0; kb < w1; kb += kAll) {
      cp_async_wait<1>();
      __syncwarp();
      float s[NT][4] = {}, rest[NT][4] = {};
#pragma unroll
      for (int i = 0; i < kLaneDims / kPer; ++i) {
        const int p = q * (kLaneDims / kPer) + i;
        const uint4 x = *reinterpret_cast<const uint4*>(buf + n * Wn::kRow + 16 * Wn::k_piece(n, p));
        const uint4 y = *reinterpret_cast<const uint4*>(buf + (n + 8) * Wn::kRow + 16 * Wn::k_piece(n, p));
        if constexpr (kParts<T> == 1) {
          const uint32_t lo[1][4] = {{x.x, y.x, x.y, y.y}}, hi[1][4] = {{x.z, y.z, x.w, y.w}};
          logits<T, D>(s, rest, lo, qb, 4 * i);
          logits<T, D>(s, rest, hi, qb, 4 * i + 2);
        } else {
          uint32_t xl[3], xh[3], yl[3], yh[3];
          parts_of(__uint_as_float(x.x), __uint_as_float(x.y), xl);
          parts_of(__uint_as_float(x.z), __uint_as_float(x.w), xh);
          parts_of(__uint_as_float(y.x), __uint_as_float(y.y), yl);
          parts_of(__uint_as_float(y.z), __uint_as_float(y.w), yh);
          const uint32_t k[3][4] = {{xl[0], yl[0], xh[0], yh[0]}, {xl[1], yl[1], xh[1], yh[1]}, {xl[2], yl[2], xh[2], yh[2]}};
          logits<T, D>(s, rest, k, qb, 2 * i);
        }
      }
      if constexpr (kParts<T> > 1) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][i] += rest[t][i];
      }
      __syncwarp();
      copy_window(kw, a.k_rs, ring, kb + kAll, false);
      uint32_t p0[kWeightParts<T, NT>][NT], p1[kWeightParts<T, NT>][NT];
      move_maximum<D, NT, true>(st, s, scale_log2, lane, w1 - kb);
      weights<T, D, NT>(st, s, scale_log2, p0, p1);
      cp_async_wait<1>();
      __syncwarp();
#pragma unroll
      for (int w = 0; w < kLaneCols / kPer; ++w) {
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 2 * q + (i & 1) + 8 * (i >> 1);
          x[i] = *reinterpret_cast<const uint4*>(buf + Wn::kBytes + r * Wn::kRow + 16 * Wn::v_piece(r, n * (kLaneCols / kPer) + w));
        }
        const uint32_t* y[4] = {&x[0].x, &x[1].x, &x[2].x, &x[3].x};
        if constexpr (kParts<T> == 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t v[1][4] = {{prmt(y[0][i], y[1][i], 0x5410), prmt(y[0][i], y[1][i], 0x7632),
                                       prmt(y[2][i], y[3][i], 0x5410), prmt(y[2][i], y[3][i], 0x7632)}};
#pragma unroll
            for (int t = 0; t < NT; ++t) weigh<T, NT>(st.o[t][4 * w + i], v, p0, p1, t);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) {  // dims 2i and 2i + 1 of the four that were read
            uint32_t e[4][3];
            parts_of(__uint_as_float(y[0][2 * i]), __uint_as_float(y[1][2 * i]), e[0]);
            parts_of(__uint_as_float(y[0][2 * i + 1]), __uint_as_float(y[1][2 * i + 1]), e[1]);
            parts_of(__uint_as_float(y[2][2 * i]), __uint_as_float(y[3][2 * i]), e[2]);
            parts_of(__uint_as_float(y[2][2 * i + 1]), __uint_as_float(y[3][2 * i + 1]), e[3]);
            const uint32_t v[3][4] = {{e[0][0], e[1][0], e[2][0], e[3][0]}, {e[0][1], e[1][1], e[2][1], e[3][1]},
                                      {e[0][2], e[1][2], e[2][2], e[3][2]}};
#pragma unroll
            for (int t = 0; t < NT; ++t) weigh<T, NT>(st.o[t][2 * w + i], v, p0, p1, t);
          }
        }
      }
      __syncwarp();
      copy_window(vw, a.v_rs, ring + Wn::kBytes, kb + kAll, true);
    }
    cp_async_wait<0>();
  }

  // join the four warps
  auto o_s = reinterpret_cast<float(*)[kRows][D + 4]>(smem);
  __syncthreads();
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float l = st.l[t][r];
      l += __shfl_xor_sync(0xffffffffu, l, 4);
      l += __shfl_xor_sync(0xffffffffu, l, 8);
      l += __shfl_xor_sync(0xffffffffu, l, 16);
      const int row = 8 * t + 2 * q + r;
      if (n == 0) ml_s[warp][row] = make_float2(st.move_at[t][r] == -INFINITY ? -INFINITY : st.ref[t][r], l);
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
      store4(O + h * a.o_hs + rowg * a.o_rs + d4, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
      if (a.lse && d4 == 0) a.lse[h * a.lse_hs + rowg] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : (l == l ? -INFINITY : l);
    }
  }
}

// Measured on B200: what a step of a block's four warps takes for every block of the SM it runs on.  Sixteen bf16 rows take as long
// as eight; in fp32 a second set of eight costs two thirds of the first (the keys are unpacked or cut into parts once).
double step_us(const fc::Kv4AttnGeom& g, int nt) {
  if (!g.f32) return g.a.d == 128 ? 0.30 : 0.18;
  return (g.a.d == 128 ? 0.40 : 0.20) * (nt == 2 ? 1.65 : 1.0);
}

// The split of the keys for tiles of 8 nt rows: the number of parts is the one that should be fastest.  A part is at least two
// steps; joining the parts costs a kernel and their bytes.  Where all blocks are resident at once, the fullest SM counts (one or
// two blocks on an SM take 1.35 or 1.08 times their share of a full one); otherwise all the work does, half a part more for the
// blocks that end last (the chunk that sees least comes last), and 3 us for each set of blocks to start and end.  fp32 parts in several
// sets take 4 us more, measured (100 rows of 8 heads on 2 over 1100 keys: one part 36 us, two 42, three 41).
struct Split {
  double us;
  int64_t part_keys;
  int32_t n;
};
constexpr int64_t kUnit = kStep * kWarps;

Split split_of(const fc_ctx* ctx, const fc::Kv4AttnGeom& g, int nt, int vis) {
  const int64_t tiles = fc::tile_count(g.a, 8 * nt) * g.a.H_kv;
  auto units_of = [&](int v) {
    const int64_t window = std::max(v - g.n_cache, 0);
    return ((window > 0 ? ((int64_t)g.n_cache + kUnit - 1) / kUnit * kUnit : std::min(v, g.n_cache)) + kWindowCost * window + kUnit - 1) / kUnit;
  };
  const int64_t units = std::max<int64_t>(1, units_of(vis)), slots = (int64_t)ctx->sm_count * blocks_per_sm(nt);
  int64_t work = 0, least = units;
  for (int c = 0; c < g.a.W; ++c) {
    const int64_t rows = (int64_t)(g.a.q_row_off[c + 1] - g.a.q_row_off[c]) * g.a.group;
    if (rows == 0) continue;
    least = std::min(least, units_of(g.a.vis[c]));
    work += (rows + 8 * nt - 1) / (8 * nt) * g.a.H_kv * units_of(g.a.vis[c]);
  }
  const double join_us = 2.0 * 4 * g.a.d * g.a.H_kv * g.n_vrows / 4e6, u = step_us(g, nt);
  Split best = {};
  int64_t last = 0;
  for (int64_t k = 1; k <= std::min<int64_t>(fc::kKv4MaxSplits, std::max<int64_t>(1, units / 2)); ++k) {
    const int64_t steps = (units + k - 1) / k, n = (units + steps - 1) / steps, blocks = tiles * n;
    if (n == last) continue;
    if (k > 1 && blocks > 4 * slots) break;
    last = n;
    const int64_t on_sm = (blocks + ctx->sm_count - 1) / ctx->sm_count;
    const double us = (blocks <= slots ? u * steps * (on_sm == 1 ? 1.35 : on_sm == 2 ? 2.15 : (double)on_sm) + 3
                                       : u * ((double)work / ctx->sm_count + 0.5 * blocks_per_sm(nt) * std::min(steps, least)) + 3.0 * blocks / slots +
                                             (n > 1 && g.f32 ? 4 : 0)) +
                      (n > 1 ? 4 + n * join_us : 0);
    if (k == 1 || us < best.us) best = {us, steps * kUnit, (int32_t)n};
  }
  return best;
}

}  // namespace

namespace fc {

size_t kv4_rows_workspace(const fc_ctx* ctx, Kv4AttnGeom& g) {
  int vis = 0;
  for (int c = 0; c < g.a.W; ++c) vis = std::max(vis, g.a.vis[c]);
  // Sixteen rows to a tile where some chunk has more than eight.  In fp32 that leaves fewer blocks of fewer registers to spare; so
  // it has to promise 5 % (three chunks of 300 rows of 8 heads of 128 over 4000 keys and the window: 242 us against 283 with eight;
  // 160 rows of 2 heads of 64 over 1040 keys: 16.7 against 12.5).
  bool many = false;
  for (int c = 0; c < g.a.W; ++c) many |= (int64_t)(g.a.q_row_off[c + 1] - g.a.q_row_off[c]) * g.a.group > 8;
  g.row_tiles = many && !g.f32 ? 2 : 1;
  Split best = split_of(ctx, g, g.row_tiles, vis);
  if (many && g.f32) {
    const Split two = split_of(ctx, g, 2, vis);
    if (two.us < 0.95 * best.us) best = two, g.row_tiles = 2;
  }
  g.part_keys = best.part_keys;
  g.n_splits = best.n;
  const int64_t cache = vis > g.n_cache ? ((int64_t)g.n_cache + kUnit - 1) / kUnit * kUnit : vis;
  g.n_cache_ceil = cache;
  g.rows_us = best.us + 4;
  if (g.n_splits == 1) return 0;
  const int64_t parts = g.a.H_kv * g.n_vrows * g.n_splits;
  return align_up(parts * g.a.d * sizeof(float), 256) + align_up(parts * sizeof(float2), 256);
}

int kv4_rows(cudaStream_t st, const Kv4AttnGeom& g, const void* Q, const void* K, const void* V, void* O) {
  const int nt = g.row_tiles;
  const int64_t tiles = tile_count(g.a, 8 * nt);
  if (tiles == 0) return FC_OK;
  if (tiles > INT32_MAX) return FC_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)tiles, (unsigned)g.a.H_kv, (unsigned)g.n_splits);
#define FC_KV4_ROWS(T, D, NT)                                                                                           \
  do {                                                                                                                  \
    constexpr int smem = kBlockBytes<T, D, NT>;                                                                         \
    if (smem > 48 * 1024)                                                                                               \
      FC_CUDA_CHECK(cudaFuncSetAttribute(attention_kv4_rows_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)); \
    attention_kv4_rows_kernel<T, D, NT><<<grid, kThreads, smem, st>>>((const T*)Q, (const T*)K, (const T*)V, (T*)O, g);  \
  } while (0)
#define FC_KV4_ROWS_PICK(T)                                                                        \
  do {                                                                                             \
    if (g.a.d == 128) { if (nt == 1) FC_KV4_ROWS(T, 128, 1); else FC_KV4_ROWS(T, 128, 2); }        \
    else { if (nt == 1) FC_KV4_ROWS(T, 64, 1); else FC_KV4_ROWS(T, 64, 2); }                       \
  } while (0)
  if (g.f32) FC_KV4_ROWS_PICK(float);
  else FC_KV4_ROWS_PICK(__nv_bfloat16);
#undef FC_KV4_ROWS_PICK
#undef FC_KV4_ROWS
  FC_LAUNCH_CHECK("attention_kv4_rows_kernel");
  return g.n_splits > 1 ? kv4_combine(st, g, g.f32 ? FC_F32 : FC_BF16, O, true) : FC_OK;
}

}  // namespace fc
