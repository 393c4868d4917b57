// Attention over [4-bit clean region | window] on CUDA cores with fp32 arithmetic throughout, softmax weights included: a second opinion
// for the tensor-core kernels, taken where impl = 1 asks for it.  The joining kernels at the end of the file serve the row kernel
// (fc_attention_kv4_rows.cu) as well.
//
// A block of 128 threads owns 32 virtual rows of one active chunk and one key head, and one part of the keys; four threads
// share a row, each holding every fourth 4-element piece of q and of the output.  Tiles of 32 keys are staged in shared
// memory as fp32, unpacked on the way in.  Where the rows alone do not fill the device the keys are cut into parts,
// and a second kernel joins the parts' outputs by their maxima and sums.
#include <algorithm>
#include <cmath>

#include "fc_attention_kv4.cuh"

namespace {

constexpr int kRows = 32, kKeys = 32, kThreads = 128;
constexpr int kMinPart = 128, kMaxSplits = 64;
constexpr int kCombineThreads = 256;

template <typename T> __device__ __forceinline__ float4 load4(const T* p);
template <> __device__ __forceinline__ float4 load4<float>(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <> __device__ __forceinline__ float4 load4<__nv_bfloat16>(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(fc::bf16_lo(w.x), fc::bf16_hi(w.x), fc::bf16_lo(w.y), fc::bf16_hi(w.y));
}
__device__ __forceinline__ void store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// Eight elements of a packed row as fp32.
__device__ __forceinline__ void unpack8(const uint8_t* codes, const uint16_t* scales, int w, float (&x)[8]) {
  const uint32_t s2 = fc::kv4_scale2(__ldg(scales + w / 4));
  uint32_t v[4];
  fc::kv4_word(__ldg(reinterpret_cast<const uint32_t*>(codes) + w), s2, fc::kv4_bias2(s2), v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = fc::bf16_lo(v[i]);
    x[2 * i + 1] = fc::bf16_hi(v[i]);
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
attention_kv4_simt_kernel(const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, T* __restrict__ O,
                          const __grid_constant__ fc::Kv4AttnGeom g) {
  constexpr int P = D / 16;  // 4-element pieces per thread
  __shared__ __align__(16) float k_s[kKeys * D];
  __shared__ __align__(16) float v_s[kKeys * D];
  __shared__ int sh_chunk, sh_v0;

  const fc::AttnGeom& a = g.a;
  const int tid = threadIdx.x, hk = blockIdx.y, part = blockIdx.z;
  if (tid < 32) {
    int v0 = 0;
    const int c = fc::tile_chunk<kRows>(a, blockIdx.x, v0);
    const bool on = fc::chunk_active(a, c);
    if (tid == 0) {
      sh_chunk = c >= 0 && on ? c : -1;
      sh_v0 = v0;
      if (blockIdx.x == 0 && hk == 0 && part == 0) fc::report_bad_ids(a);
    }
  }
  __syncthreads();
  const int c = sh_chunk;
  if (c < 0) return;
  const int r_in = tid >> 2, t = tid & 3;
  const int v = sh_v0 + r_in, row = a.q_row_off[c] + v / a.group, h = hk * a.group + v % a.group;
  const bool row_ok = row < a.q_row_off[c + 1];
  const int n_vis = min(a.vis[c], (int)min((int64_t)(part + 1) * g.part_keys, (int64_t)INT32_MAX));

  float q[P * 4], o[P * 4];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row_ok) x = load4<T>(Q + (int64_t)h * a.q_hs + (int64_t)row * a.q_rs + (i * 4 + t) * 4);
    q[4 * i] = x.x * a.scale; q[4 * i + 1] = x.y * a.scale; q[4 * i + 2] = x.z * a.scale; q[4 * i + 3] = x.w * a.scale;
    o[4 * i] = o[4 * i + 1] = o[4 * i + 2] = o[4 * i + 3] = 0.f;
  }
  float m = -INFINITY, l = 0.f;

  for (int64_t j0 = (int64_t)part * g.part_keys; j0 < n_vis; j0 += kKeys) {
    __syncthreads();  // previous tile fully consumed
    for (int x = tid; x < kKeys * (D / 8); x += kThreads) {
      const int jj = x / (D / 8), w = x % (D / 8);
      const int64_t j = j0 + jj;
      float kx[8] = {}, vx[8] = {};
      if (j < n_vis) {
        if (j < g.n_cache) {
          const int64_t co = hk * g.cache.code_hs + j * g.cache.code_rs, so = hk * g.cache.scale_hs + j * g.cache.scale_rs;
          unpack8(g.cache.k_codes + co, g.cache.k_scales + so, w, kx);
          unpack8(g.cache.v_codes + co, g.cache.v_scales + so, w, vx);
        } else {
          const int64_t p = fc::window_row(a, (int)(j - g.n_cache));
          const T* kp = K + hk * a.k_hs + p * a.k_rs + 8 * w;
          const T* vp = V + hk * a.v_hs + p * a.v_rs + 8 * w;
          *reinterpret_cast<float4*>(kx) = load4<T>(kp);
          *reinterpret_cast<float4*>(kx + 4) = load4<T>(kp + 4);
          *reinterpret_cast<float4*>(vx) = load4<T>(vp);
          *reinterpret_cast<float4*>(vx + 4) = load4<T>(vp + 4);
        }
      }
      float* ks = k_s + jj * D + 8 * w;
      float* vs = v_s + jj * D + 8 * w;
      *reinterpret_cast<float4*>(ks) = make_float4(kx[0], kx[1], kx[2], kx[3]);
      *reinterpret_cast<float4*>(ks + 4) = make_float4(kx[4], kx[5], kx[6], kx[7]);
      *reinterpret_cast<float4*>(vs) = make_float4(vx[0], vx[1], vx[2], vx[3]);
      *reinterpret_cast<float4*>(vs + 4) = make_float4(vx[4], vx[5], vx[6], vx[7]);
    }
    __syncthreads();

    float s[kKeys];
    float tile_max = -INFINITY;
#pragma unroll
    for (int jj = 0; jj < kKeys; ++jj) {
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float4 kk = *reinterpret_cast<const float4*>(k_s + jj * D + (i * 4 + t) * 4);
        dot = fmaf(q[4 * i], kk.x, dot);
        dot = fmaf(q[4 * i + 1], kk.y, dot);
        dot = fmaf(q[4 * i + 2], kk.z, dot);
        dot = fmaf(q[4 * i + 3], kk.w, dot);
      }
      dot += __shfl_xor_sync(0xffffffffu, dot, 1);
      dot += __shfl_xor_sync(0xffffffffu, dot, 2);
      s[jj] = j0 + jj < n_vis ? dot : -INFINITY;
      tile_max = fmaxf(tile_max, s[jj]);
    }
    const float m_new = fmaxf(m, tile_max);
    const float ref = m_new == -INFINITY ? 0.f : m_new;  // every logit so far is -inf (weight 0), or NaN (which stays)
    const float corr = expf(m - ref);  // exp(-inf) = 0 on the first tile
    l *= corr;
#pragma unroll
    for (int e = 0; e < P * 4; ++e) o[e] *= corr;
#pragma unroll
    for (int jj = 0; jj < kKeys; ++jj) {
      const float p = expf(s[jj] - ref);
      l += p;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float4 vv = *reinterpret_cast<const float4*>(v_s + jj * D + (i * 4 + t) * 4);
        o[4 * i] = fmaf(p, vv.x, o[4 * i]);
        o[4 * i + 1] = fmaf(p, vv.y, o[4 * i + 1]);
        o[4 * i + 2] = fmaf(p, vv.z, o[4 * i + 2]);
        o[4 * i + 3] = fmaf(p, vv.w, o[4 * i + 3]);
      }
    }
    m = m_new;
  }
  if (!row_ok) return;
  if (g.n_splits > 1) {
    const int64_t vr = (int64_t)(a.q_row_off[c] - a.q_row_off[0]) * a.group + v;
    const int64_t at = (hk * g.n_vrows + vr) * g.n_splits + part;
#pragma unroll
    for (int i = 0; i < P; ++i)
      *reinterpret_cast<float4*>(g.part_o + at * D + (i * 4 + t) * 4) = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    if (t == 0) g.part_ml[at] = make_float2(m, l);
    return;
  }
  const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
  T* out = O + (int64_t)h * a.o_hs + (int64_t)row * a.o_rs;
#pragma unroll
  for (int i = 0; i < P; ++i)
    store4(out + (i * 4 + t) * 4, make_float4(o[4 * i] * inv, o[4 * i + 1] * inv, o[4 * i + 2] * inv, o[4 * i + 3] * inv));
  if (a.lse && t == 0) a.lse[(int64_t)h * a.lse_hs + row] = l > 0.f ? m + logf(l) : (l == l ? -INFINITY : l);
}

// One block joins the parts of one virtual row: O = sum_p e^(m_p - m) o_p / sum_p e^(m_p - m) l_p.  The weights first, one part per
// thread; then groups of D/4 threads add up every so-many-th part, four elements a thread, and join through shared memory.
// A lone token has hundreds of parts at most and a few rows: what counts is that no load waits for another.
template <typename T, int D, bool kLog2>
__global__ void __launch_bounds__(kCombineThreads)
kv4_combine_kernel(T* __restrict__ O, const __grid_constant__ fc::Kv4AttnGeom g) {
  constexpr int kLanes = D / 4, kGroups = kCombineThreads / kLanes, kWarps = kCombineThreads / 32;
  __shared__ float w_s[fc::kKv4MaxSplits];
  __shared__ float4 o_s[kGroups][kLanes];
  __shared__ float m_s[kWarps], l_s[kWarps];
  const fc::AttnGeom& a = g.a;
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, hk = blockIdx.y;
  const int64_t vr = blockIdx.x;
  const int row = a.q_row_off[0] + (int)(vr / a.group), h = hk * a.group + (int)(vr % a.group);
  int c = 0;
  while (c + 1 < a.W && row >= a.q_row_off[c + 1]) ++c;
  const bool on = fc::chunk_active(a, c);
  fc::pdl_wait();  // the list was there before the kernel that wrote the parts began; the parts are there now
  if (!on) return;
  const int64_t at = (hk * g.n_vrows + vr) * g.n_splits;
  auto power = [](float x) { return kLog2 ? exp2f(x) : expf(x); };

  // the first parts are sent for before their weights are worked out
  const int grp = tid / kLanes, d4 = tid % kLanes;
  constexpr int kAhead = 4;
  float4 y[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (grp + i * kGroups < g.n_splits) y[i] = *reinterpret_cast<const float4*>(g.part_o + (at + grp + i * kGroups) * D + 4 * d4);

  float m = -INFINITY;
  float2 mine[(fc::kKv4MaxSplits + kCombineThreads - 1) / kCombineThreads];
#pragma unroll
  for (int i = 0; i < (int)(sizeof(mine) / sizeof(mine[0])); ++i) {
    const int p = tid + i * kCombineThreads;
    mine[i] = p < g.n_splits ? g.part_ml[at + p] : make_float2(-INFINITY, 0.f);
    m = fmaxf(m, mine[i].x);
  }
#pragma unroll
  for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
  if (lane == 0) m_s[warp] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) m = fmaxf(m, m_s[w]);
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(mine) / sizeof(mine[0])); ++i) {
    const int p = tid + i * kCombineThreads;
    const float w = mine[i].y != 0.f ? power(mine[i].x - m) : 0.f;  // an empty part: its maximum is -inf
    if (p < g.n_splits) w_s[p] = w;
    l += w == 0.f ? (mine[i].y == mine[i].y ? 0.f : mine[i].y) : w * mine[i].y;
  }
#pragma unroll
  for (int k = 16; k; k >>= 1) l += __shfl_xor_sync(0xffffffffu, l, k);
  if (lane == 0) l_s[warp] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) l += l_s[w];

  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (grp + i * kGroups < g.n_splits) {
      const float w = w_s[grp + i * kGroups];
      o.x = fmaf(w, y[i].x, o.x); o.y = fmaf(w, y[i].y, o.y); o.z = fmaf(w, y[i].z, o.z); o.w = fmaf(w, y[i].w, o.w);
    }
#pragma unroll 4
  for (int p = grp + kAhead * kGroups; p < g.n_splits; p += kGroups) {
    const float4 x = *reinterpret_cast<const float4*>(g.part_o + (at + p) * D + 4 * d4);
    const float w = w_s[p];
    o.x = fmaf(w, x.x, o.x); o.y = fmaf(w, x.y, o.y); o.z = fmaf(w, x.z, o.z); o.w = fmaf(w, x.w, o.w);
  }
  o_s[grp][d4] = o;
  __syncthreads();
  if (tid < kLanes) {
#pragma unroll
    for (int k = 1; k < kGroups; ++k) {
      const float4 x = o_s[k][tid];
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
    T* out = O + (int64_t)h * a.o_hs + (int64_t)row * a.o_rs + 4 * tid;
    store4(out, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (a.lse && tid == 0)
      a.lse[(int64_t)h * a.lse_hs + row] =
          l > 0.f ? (kLog2 ? (m + log2f(l)) * 0.6931471805599453f : m + logf(l)) : (l == l ? -INFINITY : l);
  }
}

// The same with one warp per row and no barrier, for many rows of few parts (at most 32): lane p holds part p's maximum and sum.
template <typename T, int D, bool kLog2>
__global__ void __launch_bounds__(kCombineThreads)
kv4_combine_warp_kernel(T* __restrict__ O, const __grid_constant__ fc::Kv4AttnGeom g) {
  constexpr int kLanes = D / 4, kGroups = 32 / kLanes;
  const fc::AttnGeom& a = g.a;
  const int lane = threadIdx.x % 32, hk = blockIdx.y;
  const int64_t vr = (int64_t)blockIdx.x * (kCombineThreads / 32) + threadIdx.x / 32;
  if (vr >= g.n_vrows) return;
  const int row = a.q_row_off[0] + (int)(vr / a.group), h = hk * a.group + (int)(vr % a.group);
  int c = 0;
  while (c + 1 < a.W && row >= a.q_row_off[c + 1]) ++c;
  const bool on = fc::chunk_active(a, c);
  fc::pdl_wait();
  if (!on) return;
  const int64_t at = (hk * g.n_vrows + vr) * g.n_splits;
  auto power = [](float x) { return kLog2 ? exp2f(x) : expf(x); };
  const float2 ml = lane < g.n_splits ? g.part_ml[at + lane] : make_float2(-INFINITY, 0.f);
  float m = ml.x;
#pragma unroll
  for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
  const float w = ml.y != 0.f ? power(ml.x - m) : 0.f;
  float l = w == 0.f ? (ml.y == ml.y ? 0.f : ml.y) : w * ml.y;
#pragma unroll
  for (int k = 16; k; k >>= 1) l += __shfl_xor_sync(0xffffffffu, l, k);
  const int grp = lane / kLanes, d4 = lane % kLanes;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int p0 = 0; p0 < g.n_splits; p0 += kGroups) {
    const int p = p0 + grp;
    const float wp = __shfl_sync(0xffffffffu, w, p & 31);
    if (p < g.n_splits) {
      const float4 x = *reinterpret_cast<const float4*>(g.part_o + (at + p) * D + 4 * d4);
      o.x = fmaf(wp, x.x, o.x); o.y = fmaf(wp, x.y, o.y); o.z = fmaf(wp, x.z, o.z); o.w = fmaf(wp, x.w, o.w);
    }
  }
  if (kGroups == 2) {
    o.x += __shfl_xor_sync(0xffffffffu, o.x, 16); o.y += __shfl_xor_sync(0xffffffffu, o.y, 16);
    o.z += __shfl_xor_sync(0xffffffffu, o.z, 16); o.w += __shfl_xor_sync(0xffffffffu, o.w, 16);
  }
  if (lane < kLanes) {
    const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
    T* out = O + (int64_t)h * a.o_hs + (int64_t)row * a.o_rs + 4 * d4;
    store4(out, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (a.lse && lane == 0)
      a.lse[(int64_t)h * a.lse_hs + row] =
          l > 0.f ? (kLog2 ? (m + log2f(l)) * 0.6931471805599453f : m + logf(l)) : (l == l ? -INFINITY : l);
  }
}

}  // namespace

namespace fc {

size_t kv4_simt_workspace(const fc_ctx* ctx, Kv4AttnGeom& g) {
  int vis = 0;
  for (int c = 0; c < g.a.W; ++c) vis = std::max(vis, g.a.vis[c]);
  const int64_t blocks = tile_count(g.a, kRows) * g.a.H_kv;
  const int64_t want = blocks > 0 ? (4ll * ctx->sm_count + blocks - 1) / blocks : 1;  // about four blocks an SM
  const int64_t most = std::min<int64_t>(kMaxSplits, (vis + kMinPart - 1) / kMinPart);
  const int64_t n = std::max<int64_t>(1, std::min(want, most));
  g.part_keys = std::max<int64_t>(kKeys, ((vis + n - 1) / n + kKeys - 1) / kKeys * kKeys);
  g.n_splits = (int32_t)std::max<int64_t>(1, ((int64_t)vis + g.part_keys - 1) / g.part_keys);
  if (g.n_splits == 1) return 0;
  const int64_t parts = g.a.H_kv * g.n_vrows * g.n_splits;
  return align_up(parts * g.a.d * sizeof(float), 256) + align_up(parts * sizeof(float2), 256);
}

int kv4_combine(cudaStream_t st, const Kv4AttnGeom& g, int dtype, void* O, bool log2_units) {
  // A block per row has all its loads in flight at once, a warp per row has no barriers: the first for a few rows, which
  // leave the device empty anyway, the second for many.
  const bool warps = g.n_splits <= 32 && g.n_vrows * g.a.H_kv >= 1024;
  const int per = warps ? kCombineThreads / 32 : 1;
  const dim3 grid((unsigned)((g.n_vrows + per - 1) / per), (unsigned)g.a.H_kv);
#define FC_COMBINE(T, D)                                                                    \
  do {                                                                                      \
    auto kernel = warps ? (log2_units ? kv4_combine_warp_kernel<T, D, true> : kv4_combine_warp_kernel<T, D, false>) \
                        : (log2_units ? kv4_combine_kernel<T, D, true> : kv4_combine_kernel<T, D, false>);          \
    FC_CUDA_CHECK(launch_pdl(kernel, grid, dim3(kCombineThreads), 0, st, (T*)O, g));               \
  } while (0)
  if (dtype == FC_F32) { if (g.a.d == 128) FC_COMBINE(float, 128); else FC_COMBINE(float, 64); }
  else { if (g.a.d == 128) FC_COMBINE(__nv_bfloat16, 128); else FC_COMBINE(__nv_bfloat16, 64); }
#undef FC_COMBINE
  FC_LAUNCH_CHECK("kv4_combine_kernel");
  return FC_OK;
}

int kv4_simt(cudaStream_t st, const Kv4AttnGeom& g, const void* Q, const void* K, const void* V, int dtype, void* O) {
  const int64_t tiles = tile_count(g.a, kRows);
  if (tiles == 0) return FC_OK;
  if (tiles > INT32_MAX) return FC_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)tiles, (unsigned)g.a.H_kv, (unsigned)g.n_splits);
#define FC_KV4_SIMT(T, D) \
  attention_kv4_simt_kernel<T, D><<<grid, kThreads, 0, st>>>((const T*)Q, (const T*)K, (const T*)V, (T*)O, g)
  if (dtype == FC_F32) { if (g.a.d == 128) FC_KV4_SIMT(float, 128); else FC_KV4_SIMT(float, 64); }
  else { if (g.a.d == 128) FC_KV4_SIMT(__nv_bfloat16, 128); else FC_KV4_SIMT(__nv_bfloat16, 64); }
#undef FC_KV4_SIMT
  FC_LAUNCH_CHECK("attention_kv4_simt_kernel");
  return g.n_splits > 1 ? kv4_combine(st, g, dtype, O, false) : FC_OK;
}

}  // namespace fc
