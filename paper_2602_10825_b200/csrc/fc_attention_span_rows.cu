// Attention of few query rows over [8-bit pages | plain rows], each chunk over its first tokens and its sliding window: one pass over the
// keys, cut into parts; also the path of fp32 tensors whatever their rows.  Up to sixteen parts of a tile of rows are the blocks of a thread block
// cluster, which join through its shared memory; a second kernel joins them where that is faster: a few tiles that see many keys, chunks that
// see far more than others, clusters that would leave much of the device empty.
//
// Bound by the bytes of the keys.  A warp takes 32 keys at a step (16 over plain rows) from its own ring in shared memory, which the copy
// engine fills (a box of the step's rows is one instruction of one lane, and lies swizzled so that the reads below meet no bank twice),
// and feeds them to mma.sync from registers:
//   S^T = K Q^T   m16n8k16, keys as rows, up to 8 NT query rows as columns.  The order of the head's elements along the
//                 contraction is free as long as K and Q agree: lane (n, q) takes, of keys n and n + 8, the bytes 32 q .. 32 q + 31 of
//                 every 128.
//   O^T = V^T P^T dims as rows.  Lane (n, q) takes dims 64 j + 8 n .. 64 j + 8 n + 7 of keys 2q, 2q+1, 2q+8, 2q+9; the elements
//                 of two keys are brought into one register, so that the pair along the contraction is a pair of 16-bit halves.
// P^T goes from the accumulator layout of the first product to the operand layout of the second by movmatrix.
//
// Pages.  A code is exactly an fp16 number, and one instruction makes two; so the products are of fp16.  Q, which is a
// bf16 number of any size, is brought into fp16 by a power of two of its row that puts the row's largest element at 2^14: all of its bits are
// kept down to 2^-29 of that.  The keys' scale goes into the logits, the values' scale multiplies a step's sum before it is
// added to O, which is in fp32.  Weights are taken 2^7 times larger than their reference asks for, so that fp16's smallest step,
// 2^-24, is 2^-31 of the largest weight; the values' scale, or over plain rows the weight, makes up for it.  A step is about 215 instructions for each 16 keys of one to eight rows, which is what a block alone on
// its SM is bound by (0.45 us for its four warps' 64 keys; with 16 keys a step, and a barrier, a look-up, a vote and a copy for each, 0.62); from
// one and a half blocks an SM on it is the bandwidth: one token over 28080 tokens of 24 heads 34.0 us, the same without the arithmetic 32, the
// bytes' own time 26.3.
// Plain rows go through the products of their own type (bf16, or for fp32 the six largest products of three bf16 parts each).
// fp32 over pages: two fp16 parts of Q, and of the weights, leave out at most 2^-23 of a number, or, where that is more, 2^-39 of the row's largest
// element of Q and 2^-43 of its largest weight.
// The maximum is lazy (it moves when a logit passes it by 2^8), so that the usual step has no shuffles and no rescaling.
#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "fc_attention_span.cuh"
#include "fc_mma_sync.cuh"

namespace {

using namespace fc::sm100;

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStep = 16;            // keys per warp and step over plain rows, and of a matrix instruction
constexpr int kPagedStep = 32;       // over pages
constexpr int kTable = 64 * 32;      // bytes of what a warp knows of its next steps over pages
constexpr int kRing = 16 * 1024;     // bytes of a warp's two rings
constexpr int kMaxCluster = 16;      // blocks of a cluster
constexpr int kSmem = kWarps * (kRing + kTable) + 1024;  // of a block, the rings on a 1024-byte boundary
constexpr float kSlack = 8.f;        // log2 units by which a logit may pass the maximum before that moves
constexpr float kLift = 7.f;         // weights are 2^kLift at the maximum
constexpr float kUnit = 32768.f;     // 2^(kLift + kSlack), the most that a weight can be: O is kept divided by it, so that it passes fp32's range no sooner than weights of 1 would
constexpr int blocks_per_sm(int nt) { return nt == 1 ? 3 : 2; }
constexpr int kPagedCost = 2;        // cost of a step over pages, and over plain rows
template <typename T> constexpr int kPlainCost = sizeof(T) == 4 ? 3 : 2;

template <typename T> constexpr int kParts = sizeof(T) == 4 ? 3 : 1;       // bf16 parts of Q, K and V over plain rows
template <typename T> constexpr int kHalves = sizeof(T) == 4 ? 2 : 1;      // fp16 parts of Q and of the weights over pages
constexpr float kRest = 2048.f;      // the weights' second part is taken 2^11 times larger: as large as the first at most, and fp16's smallest step is 2^-35 then
// Weights over plain rows: bf16 rounds one by up to 2^-8, as much again as the output's own rounding; for up to eight rows the rest is taken along.
template <typename T, int NT> constexpr int kWeightParts = sizeof(T) == 4 ? 3 : (NT == 1 ? 2 : 1);

template <typename T, int D> struct Ring {
  static constexpr int kPaged = kPagedStep * D, kPlain = kStep * D * (int)sizeof(T);  // bytes of one tensor's step
  static constexpr int kPagedStages = kRing / 2 / kPaged, kPlainStages = kRing / 2 / kPlain;
  static constexpr int kAtoms = D * (int)sizeof(T) / 128;  // boxes of 128 bytes x 16 rows of a plain step
  static_assert(kPlainStages >= 1 && kPagedStages <= 8, "stages");
};
constexpr int kBars = 8;  // barriers of a ring

__device__ __forceinline__ uint32_t cvt_f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127

// What a warp carries along its keys: O^T over kUnit, this lane's share of the sums, and per row the reference of its exponents (log2
// units) and the logit above which it moves.  A row that has met no finite logit yet has move_at = -inf and the reference 0:
// weights of -inf are 0 then, and a NaN stays one.
template <int D, int NT> struct State {
  float o[NT][D / 16][4];
  float l[NT][2], ref[NT][2], move_at[NT][2];
};

// Logits (log2 units) of N times 16 keys to weights, in place.  kMask: keys lo .. hi - 1 of them count.
template <int D, int NT, bool kMask, int N>
__device__ __forceinline__ void weigh_logits(State<D, NT>& st, float (&s)[N][NT][4], int lane, int lo, int hi) {
  bool move = false;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (kMask) {
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = 16 * k + (lane >> 2) + (i >= 2 ? 8 : 0);
          if (key < lo || key >= hi) s[k][t][i] = -INFINITY;
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x = fmaxf(s[0][t][r], s[0][t][2 + r]);
#pragma unroll
      for (int k = 1; k < N; ++k) x = max3(x, s[k][t][r], s[k][t][2 + r]);
      move |= x > st.move_at[t][r];
    }
  }
  if (__any_sync(0xffffffffu, move)) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float x = fmaxf(s[0][t][r], s[0][t][2 + r]);
#pragma unroll
        for (int k = 1; k < N; ++k) x = max3(x, s[k][t][r], s[k][t][2 + r]);
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
        if (x > st.move_at[t][r]) {
          const float ref = x - kLift;
          const float alpha = st.move_at[t][r] == -INFINITY ? 0.f : ex2(st.ref[t][r] - ref);
          st.ref[t][r] = ref;
          st.move_at[t][r] = x + kSlack;
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
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[k][t][i] = ex2(s[k][t][i] - st.ref[t][i & 1]);
      st.l[t][0] += s[k][t][0] + s[k][t][2];
      st.l[t][1] += s[k][t][1] + s[k][t][3];
    }
}

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Shared memory of block `rank` of the cluster, at this block's address `at`.
__device__ __forceinline__ uint32_t at_rank(uint32_t at, int rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at), "r"(rank));
  return a;
}
__device__ __forceinline__ float2 cluster_load2(uint32_t at, int rank) {
  float2 x;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(at_rank(at, rank)) : "memory");
  return x;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t at, int rank) {
  float4 x;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at_rank(at, rank)) : "memory");
  return x;
}

// What a row gets whose weights are all 0: nothing was seen (0, and a log-sum of -inf), or, in a chunk that sees tokens, every logit was -inf (NaN).
__device__ __noinline__ float without_weights(const fc::SpanGeom& g, int c) {
  bool sees = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) sees |= g.hi[i][c] > g.lo[i][c];
  return sees ? __uint_as_float(0x7fc00000u) : 0.f;
}

// Four elements of virtual row v of chunk c: a sum of weights times values over kUnit, its reference and the sum of the weights.
template <typename T>
__device__ __forceinline__ void write_row(T* O, const fc::SpanGeom& g, int c, int hk, int v, int d4, float4 o, float ref, float l) {
  const float inv = l > 0.f ? kUnit / l : (l == l ? without_weights(g, c) : l);
  const int h = hk * g.group + v % g.group;
  const int64_t row = g.q_row_off[c] + v / g.group;
  if (!fc::bounds_ok(row >= 0 && row < g.q_row_off[g.W] && h >= 0 && h < g.H_q, g.status)) return;
  store4(O + h * g.o_hs + row * g.o_rs + d4, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
  if (g.lse && d4 == 0) g.lse[h * g.lse_hs + row] = l > 0.f ? (ref + log2f(l)) * 0.6931471805599453f : (inv == 0.f ? -INFINITY : inv);
}

// What a warp knows of one of its next steps over pages: the pages of its two halves (the same one, but for pages of 16 tokens; -1: none is needed, or
// the entry names none); the first of its rows, and which of the 32 are seen, as row | lo << 8 | hi << 16, negative unless all are and
// one page has them; and the scales of K and V of the halves.
struct __align__(16) PagedStep {
  int page[2], place, pad;
  float ks[2], vs[2];  // vs / kUnit
};
static_assert(sizeof(PagedStep) * 64 == kTable, "two groups of 32 steps");

// The steps over plain rows, numbered run by run: a run is what a span and a segment share.
struct Walk {
  int run, first, steps, len, phys;  // steps first .. first + steps - 1 are this run's
};
__device__ __forceinline__ void walk_load(const fc::SpanGeom& g, int c, Walk& w) {
  w.len = 0;
  if (w.run < 2 * g.n_seg) {
    const int i = w.run < g.n_seg ? 2 : 3, s = w.run - (i - 2) * g.n_seg;
    const int lo = max(g.lo[i][c], g.seg_log[s]), hi = min(g.hi[i][c], g.seg_log[s + 1]);
    w.len = max(hi - lo, 0);
    w.phys = g.seg_phys[s] + lo - g.seg_log[s];
  }
  w.steps = (w.len + kStep - 1) / kStep;
}
__device__ __forceinline__ void walk_to(const fc::SpanGeom& g, int c, Walk& w, int step) {
  while (step >= w.first + w.steps && w.run < 2 * g.n_seg) {
    w.first += w.steps;
    ++w.run;
    walk_load(g, c, w);
  }
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(NT))
attention_span_rows_kernel(const __grid_constant__ CUtensorMap map_k8, const __grid_constant__ CUtensorMap map_v8,
                           const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                           const T* __restrict__ Q, T* __restrict__ O, const __grid_constant__ fc::SpanGeom g) {
  constexpr int kRows = 8 * NT;
  using R = Ring<T, D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars[kWarps][2][2][kBars];  // warp; pages (K and V) or plain rows; K or V; stage
  __shared__ float2 ml_s[kWarps][kRows];
  __shared__ uint32_t abort_s;
  fc::pdl_launch_dependents();  // the joining kernel may take its place; it waits for this grid to end
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, n = lane >> 2, q = lane & 3;
  const int hk = blockIdx.y;
  int c = 0;
  while (c + 1 < g.W && (int)blockIdx.x >= g.block_end[c]) ++c;
  const int local = (int)blockIdx.x - (c > 0 ? g.block_end[c - 1] : 0), n_parts = g.parts[c];
  const int part = local % n_parts, v0 = local / n_parts * kRows;
  const int rows_here = min(kRows, (g.q_row_off[c + 1] - g.q_row_off[c]) * g.group - v0);

  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const uint32_t ring_s = smem_u32(smem) + warp * kRing;
  volatile uint32_t* abort = &abort_s;
  auto bar = [&](int plain, int v, int stage) { return smem_u32(&bars[warp][plain][v][stage]); };
  if (lane < 4 * kBars) mbar_init(smem_u32(&bars[warp][0][0][0] + lane), 1);
  if (tid == 0) {
    abort_s = 0;
    if (g.pool.n_pages > 0) {
      tma_prefetch_desc(&map_k8);
      tma_prefetch_desc(&map_v8);
    }
    if (g.n_seg > 0) {
      tma_prefetch_desc(&map_k);
      tma_prefetch_desc(&map_v);
    }
  }
  mbar_fence_init();
  __syncthreads();

  // This part's steps: the axis has kPagedCost units for each step over pages, then kPlainCost for each over plain rows.
  const int log2 = g.pool.page_log2;
  auto steps_of = [&](int i) { return g.hi[i][c] > g.lo[i][c] ? (g.hi[i][c] + kPagedStep - 1) / kPagedStep - g.lo[i][c] / kPagedStep : 0; };
  const int n_first = steps_of(0), n_paged = n_first + steps_of(1);
  const int64_t x0 = (int64_t)part * g.part_units[c], x1 = x0 + g.part_units[c];
  auto paged_at = [&](int64_t x) { return (int)min((x + kPagedCost - 1) / kPagedCost, (int64_t)n_paged); };
  const int p0 = paged_at(x0), p1 = paged_at(x1);
  const bool last_part = part == n_parts - 1;  // takes what there is
  auto plain_at = [&](int64_t x) { return (int)((max(x - (int64_t)kPagedCost * n_paged, (int64_t)0) + kPlainCost<T> - 1) / kPlainCost<T>); };
  const int w0 = plain_at(x0), w1 = last_part ? INT_MAX - 64 : plain_at(x1);

  State<D, NT> st;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) st.o[t][j][0] = st.o[t][j][1] = st.o[t][j][2] = st.o[t][j][3] = 0.f;
    st.l[t][0] = st.l[t][1] = st.ref[t][0] = st.ref[t][1] = 0.f;
    st.move_at[t][0] = st.move_at[t][1] = -INFINITY;
  }
  const float scale_log2 = g.scale * 1.4426950408889634f;
  // query row 8 t + n of the tile, or NULL
  auto q_row = [&](int t) -> const T* {
    const int r = 8 * t + n;
    if (r >= rows_here) return nullptr;
    const int v = v0 + r;
    return Q + (int64_t)(hk * g.group + v % g.group) * g.q_hs + (int64_t)(g.q_row_off[c] + v / g.group) * g.q_rs;
  };

  if (hk == 0 && blockIdx.x == 0 && warp == 0) {
    const int n_ids = min(max(*g.n_active, 0), g.W);
    for (int i = lane; i < n_ids; i += 32)
      if ((g.active_ids[i] < 0 || g.active_ids[i] >= g.W) && g.status) atomicOr(g.status, (uint32_t)FC_DEV_BAD_INDEX);
  }

  // ------------------------------------------------------------------ pages
  const int m = max(0, (p1 - p0 - warp + kWarps - 1) / kWarps);  // this warp's steps: p0 + warp, + kWarps, ...
  constexpr int kPagedStages = R::kPagedStages;
  bool bad = false;  // an entry that names no page
  auto look_up = [&](int i) {  // all but the scales
    PagedStep x = {{-1, -1}, kPagedStep << 16, 0, {0.f, 0.f}, {0.f, 0.f}};
    if (i < m) {
      const int s = p0 + warp + i * kWarps, k = s < n_first ? 0 : 1;
      const int tok = (g.lo[k][c] / kPagedStep + (k ? s - n_first : s)) * kPagedStep;
      const int lo = max(g.lo[k][c] - tok, 0), hi = min(g.hi[k][c] - tok, kPagedStep);
      bool part = lo > 0 || hi < kPagedStep || log2 == 4;
      const int32_t* entry = g.table + c * g.table_cs + (tok >> log2);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (e == 1 && log2 > 4) {
          x.page[1] = x.page[0];
        } else if (log2 > 4 || (lo < 16 * (e + 1) && hi > 16 * e)) {
          x.page[e] = __ldg(entry + e);
          if (x.page[e] < 0 || x.page[e] >= g.pool.n_pages) {
            x.page[e] = -1;
            bad = part = true;
          }
        }
      }
      x.place = (tok & ((1 << log2) - 1)) | lo << 8 | hi << 16 | (part ? INT_MIN : 0);
    }
    return x;
  };
  auto look_up_scales = [&](PagedStep& x) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (x.page[e] >= 0) {
        x.ks[e] = __ldg(g.pool.k_scales + x.page[e] * g.pool.scale_ps + hk * g.pool.scale_hs);
        x.vs[e] = __ldg(g.pool.v_scales + x.page[e] * g.pool.scale_ps + hk * g.pool.scale_hs) * (1.f / kUnit);  // exact, below the normal numbers too
      }
  };
  const uint32_t bar_s = bar(0, 0, 0);
  auto send_paged = [&](int page0, int page1, int row, int stage) {
    const uint32_t b = bar_s + 8 * stage, dst = ring_s + stage * (2 * R::kPaged);
    if (page0 < 0 && page1 < 0) {  // nothing to bring
      mbar_arrive(b);
    } else if (log2 > 4) {
      mbar_expect_tx(b, 2 * R::kPaged);
      tma_load_4d(dst, &map_k8, b, 0, row, hk, page0);
      tma_load_4d(dst + R::kPaged, &map_v8, b, 0, row, hk, page0);
    } else {
      mbar_expect_tx(b, (page0 >= 0 && page1 >= 0 ? 2 : 1) * R::kPaged);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int page = e ? page1 : page0;
        if (page < 0) continue;
        tma_load_4d(dst + e * (16 * D), &map_k8, b, 0, 0, hk, page);
        tma_load_4d(dst + R::kPaged + e * (16 * D), &map_v8, b, 0, 0, hk, page);
      }
    }
  };
  // Lane L looks up steps L, 32 + L, ...: two groups of 32 are in the table.  The first steps are sent for before the scales are here.
  PagedStep* const table = reinterpret_cast<PagedStep*>(smem + kWarps * kRing + warp * kTable);
  const uint32_t table_s = smem_u32(table);
  if (m > 0) {
    PagedStep x = look_up(lane);
    if (lane < min(m, kPagedStages)) send_paged(x.page[0], x.page[1], x.place & 255, lane);
    look_up_scales(x);
    table[lane] = x;
    if (m > 32) {
      x = look_up(32 + lane);
      look_up_scales(x);
      table[32 + lane] = x;
    }
    __syncwarp();
  }
  // everything up to here asks only what the host knows; the list is on the device
  if (!fc::span_chunk_active(g, c)) {
    for (int i = 0; i < min(m, kPagedStages); ++i) mbar_wait_bounded(bar_s + 8 * i, 0, abort);  // what was sent for lands before its memory is given back
    return;
  }
  if (m > 0) {
    constexpr int kStages = kPagedStages;
    // Q as fp16 parts of rows brought to 2^14, and what undoes that
    uint32_t qb[kHalves<T>][NT][D / 8];
    float qs[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const T* row = q_row(t);
      float x[D / 4];
#pragma unroll
      for (int i = 0; i < D / 4; ++i) x[i] = 0.f;
      if (row) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int i = 0; i < D / 32; ++i) {
            const uint4 w = *reinterpret_cast<const uint4*>(row + q * (D / 4) + 8 * i);
            const uint32_t y[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) x[8 * i + 2 * k] = fc::bf16_lo(y[k]), x[8 * i + 2 * k + 1] = fc::bf16_hi(y[k]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            const float4 w = *reinterpret_cast<const float4*>(row + q * (D / 4) + 4 * i);
            x[4 * i] = w.x; x[4 * i + 1] = w.y; x[4 * i + 2] = w.z; x[4 * i + 3] = w.w;
          }
        }
      }
      uint32_t a = 0;
#pragma unroll
      for (int i = 0; i < D / 4; ++i) a = max(a, __float_as_uint(x[i]) & 0x7fffffffu);
      a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
      a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
      const int e = a == 0 ? 0 : min(max(14 - ((int)(a >> 23) - 127), -113), 126);
      const float f = pow2(e), back = pow2(-e) * scale_log2;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const float u = x[2 * i] * f, v = x[2 * i + 1] * f;
        qb[0][t][i] = cvt_f16x2(u, v);
        if constexpr (kHalves<T> == 2) qb[1][t][i] = cvt_f16x2(u - fc::half_lo(qb[0][t][i]), v - fc::half_hi(qb[0][t][i]));
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) qs[t][r] = __shfl_sync(0xffffffffu, back, (2 * q + r) * 4);
    }
    // where this lane reads: 32 (D = 128) or 16 bytes of keys n and n + 8; eight bytes of keys 2q, 2q+1, 2q+8, 2q+9.  A row is
    // 128 or 64 bytes, its 16-byte pieces exchanged by bits 7.. of the address.
    const int ka = D == 128 ? n * 128 + (((2 * q) ^ (n & 7)) << 4) : n * 64 + ((q ^ ((n >> 1) & 3)) << 4);
    // (rows r and r + 8 are 8 D bytes apart)
    auto v_at = [&](int r) {  // dims 8 n of row r; 64 + 8 n is 64 bytes from there, by exchange
      return D == 128 ? r * 128 + (((n >> 1) ^ (r & 7)) << 4) + 8 * (n & 1) : r * 64 + (((n >> 1) ^ ((r >> 1) & 3)) << 4) + 8 * (n & 1);
    };
    const uint32_t k_at = ring_s + ka, va[2] = {ring_s + R::kPaged + v_at(2 * q), ring_s + R::kPaged + v_at(2 * q + 1)};

    // A step: the products of its keys with Q, the weights, and O.  kPart: keys lo .. hi - 1 count, and the halves have pages and scales of
    // their own.
    auto step = [&](uint32_t off, float4 scales, int lo, int hi, bool none0, bool none1, auto parted) {
      constexpr bool kPart = decltype(parted)::value;
      float s[2][NT][4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint32_t k0[D / 16], k1[D / 16];
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          const uint32_t at = (k_at ^ (h << 4)) + off + e * (16 * D);
          const uint4 a = lds16(at), b = lds16(at + 8 * D);
          k0[4 * h] = a.x; k0[4 * h + 1] = a.y; k0[4 * h + 2] = a.z; k0[4 * h + 3] = a.w;
          k1[4 * h] = b.x; k1[4 * h + 1] = b.y; k1[4 * h + 2] = b.z; k1[4 * h + 3] = b.w;
        }
        float rest[NT][4];
#pragma unroll
        for (int w = 0; w < D / 16; ++w) {
          const uint32_t a0 = fc::e4m3_lo2(k0[w]), a1 = fc::e4m3_lo2(k1[w]), a2 = fc::e4m3_hi2(k0[w]), a3 = fc::e4m3_hi2(k1[w]);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            auto add = [&](float (&d)[4], const uint32_t (&b)[D / 8]) {
              if (w == 0) mma_f16_first(d, a0, a1, a2, a3, b[0], b[1]);
              else mma_f16(d, a0, a1, a2, a3, b[2 * w], b[2 * w + 1]);
            };
            add(s[e][t], qb[0][t]);
            if constexpr (kHalves<T> == 2) add(rest[t], qb[1][t]);
          }
        }
        const float ks = kPart && e == 1 ? scales.y : scales.x;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            s[e][t][k] = (kHalves<T> == 2 ? s[e][t][k] + rest[t][k] : s[e][t][k]) * (qs[t][k & 1] * ks);
            if (kPart && (e ? none1 : none0)) s[e][t][k] = 0.f;
          }
      }
      weigh_logits<D, NT, kPart, 2>(st, s, lane, lo, hi);
      uint32_t pa[2][kHalves<T>][NT][2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint32_t a = cvt_f16x2(s[e][t][0], s[e][t][1]), b = cvt_f16x2(s[e][t][2], s[e][t][3]);
          pa[e][0][t][0] = transpose8x8(a);
          pa[e][0][t][1] = transpose8x8(b);
          if constexpr (kHalves<T> == 2) {
            pa[e][1][t][0] = transpose8x8(cvt_f16x2((s[e][t][0] - fc::half_lo(a)) * kRest, (s[e][t][1] - fc::half_hi(a)) * kRest));
            pa[e][1][t][1] = transpose8x8(cvt_f16x2((s[e][t][2] - fc::half_lo(b)) * kRest, (s[e][t][3] - fc::half_hi(b)) * kRest));
          }
        }
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        uint2 v[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            v[e][k] = lds8((va[k & 1] ^ (j << 6)) + off + e * (16 * D) + (k >> 1) * (8 * D));
            if (kPart) {
              const int key = 16 * e + 2 * q + (k & 1) + 8 * (k >> 1);
              if ((e ? none1 : none0) || key < lo || key >= hi) v[e][k] = make_uint2(0u, 0u);  // whatever it is: 0 x NaN is NaN
            }
          }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 2; ++k) {  // dims 2 k and 2 k + 1 of the four that were read
            uint32_t a[2][4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t y[4] = {h ? v[e][0].y : v[e][0].x, h ? v[e][1].y : v[e][1].x, h ? v[e][2].y : v[e][2].x, h ? v[e][3].y : v[e][3].x};
              const uint32_t ab = prmt(y[0], y[1], k ? 0x7362 : 0x5140), cd = prmt(y[2], y[3], k ? 0x7362 : 0x5140);
              a[e][0] = fc::e4m3_lo2(ab); a[e][1] = fc::e4m3_hi2(ab); a[e][2] = fc::e4m3_lo2(cd); a[e][3] = fc::e4m3_hi2(cd);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              float(&o)[4] = st.o[t][4 * j + 2 * h + k];
#pragma unroll
              for (int w = kHalves<T> - 1; w >= 0; --w) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  if (kPart || e == 0) mma_f16_first(x, a[e][0], a[e][1], a[e][2], a[e][3], pa[e][w][t][0], pa[e][w][t][1]);
                  else mma_f16(x, a[e][0], a[e][1], a[e][2], a[e][3], pa[e][w][t][0], pa[e][w][t][1]);
                  if (kPart || e == 1) {
                    const float vs = (kPart && e == 0 ? scales.z : scales.w) * (w == 1 ? 1.f / kRest : 1.f);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = fmaf(vs, x[i], o[i]);
                  }
                }
              }
            }
          }
      }
    };
    int stage = 0;
    uint32_t parity = 0;
    PagedStep pending;
    for (int i = 0; i < m; ++i) {
      if (i >= 32 && (i & 15) == 0) {  // the group after this one: looked up as this one begins, in the table halfway through it
        if ((i & 16) == 0) {
          pending = look_up(i + 32 + lane);
          look_up_scales(pending);
        } else {
          table[((i & ~31) + 32 + lane) & 63] = pending;
        }
        __syncwarp();
      }
      const uint32_t entry = table_s + (i & 63) * (int)sizeof(PagedStep), off = stage * (2 * R::kPaged);
      const uint4 sc = lds16(entry + 16);
      const float4 scales = make_float4(__uint_as_float(sc.x), __uint_as_float(sc.y), __uint_as_float(sc.z), __uint_as_float(sc.w));
      const int place = (int)lds4(entry + 8);
      mbar_wait_bounded(bar_s + 8 * stage, parity, abort);
      __syncwarp();
      if (place >= 0) {
        step(off, scales, 0, kPagedStep, false, false, std::false_type());
      } else {
        const uint2 pages = lds8(entry);
        step(off, scales, place >> 8 & 255, place >> 16 & 255, (int)pages.x < 0, (int)pages.y < 0, std::true_type());
      }
      __syncwarp();  // the step's place has been read by every lane: another step is sent for
      if (i + kStages < m && elected()) {
        const uint4 x = lds16(table_s + ((i + kStages) & 63) * (int)sizeof(PagedStep));
        send_paged((int)x.x, (int)x.y, (int)x.z & 255, stage);
      }
      if (++stage == kStages) stage = 0, parity ^= 1;
    }
  }

  // ------------------------------------------------------------------ plain rows
  Walk now = {0, 0, 0, 0, 0};
  walk_load(g, c, now);
  walk_to(g, c, now, w0 + warp);
  if (w0 + warp < w1 && now.run < 2 * g.n_seg) {
    constexpr int kStages = R::kPlainStages, kPer = 16 / (int)sizeof(T);
    Walk ahead_k = now, ahead_v = now;
    auto send = [&](int i, Walk& w, int v) {
      const int s = w0 + warp + i * kWarps;
      if (s >= w1) return;
      walk_to(g, c, w, s);
      if (w.run >= 2 * g.n_seg || lane != 0) return;
      const int stage = i % kStages, row = w.phys + (s - w.first) * kStep;
      mbar_expect_tx(bar(1, v, stage), R::kPlain);
#pragma unroll
      for (int a = 0; a < R::kAtoms; ++a)
        tma_load_3d(ring_s + (v ? kRing / 2 : 0) + stage * R::kPlain + a * (kStep * 128), v ? &map_v : &map_k, bar(1, v, stage), a * (128 / (int)sizeof(T)), row, hk);
    };
    for (int i = 0; i < kStages; ++i) {
      send(i, ahead_k, 0);
      send(i, ahead_v, 1);
    }
    uint32_t qb[kParts<T>][NT][D / 8];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const T* row = q_row(t);
#pragma unroll
      for (int a = 0; a < R::kAtoms; ++a)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 x = row ? *reinterpret_cast<const uint4*>(row + a * (8 * kPer) + (2 * q + h) * kPer) : make_uint4(0u, 0u, 0u, 0u);
          if constexpr (kParts<T> == 1) {
            uint32_t* y = &qb[0][t][8 * a + 4 * h];
            y[0] = x.x; y[1] = x.y; y[2] = x.z; y[3] = x.w;
          } else {
            uint32_t lo[3], hi[3];
            parts_of(__uint_as_float(x.x), __uint_as_float(x.y), lo);
            parts_of(__uint_as_float(x.z), __uint_as_float(x.w), hi);
#pragma unroll
            for (int j = 0; j < 3; ++j) qb[j][t][4 * a + 2 * h] = lo[j], qb[j][t][4 * a + 2 * h + 1] = hi[j];
          }
        }
    }
    for (int i = 0;; ++i) {
      const int sidx = w0 + warp + i * kWarps;
      if (sidx >= w1) break;
      walk_to(g, c, now, sidx);
      if (now.run >= 2 * g.n_seg) break;
      const int hi = min(kStep, now.len - (sidx - now.first) * kStep), stage = i % kStages, parity = (i / kStages) & 1;
      mbar_wait_bounded(bar(1, 0, stage), parity, abort);
      __syncwarp();
      const uint32_t kp = ring_s + stage * R::kPlain;
      float s1[1][NT][4] = {}, rest[NT][4] = {};
      auto& s = s1[0];
      auto products = [&](const auto& k, int at) {  // K as NK parts of operand registers; `at`: first register of Q
        constexpr int NK = kParts<T>;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int a = NK - 1; a >= 0; --a)
#pragma unroll
            for (int b = NK - 1; b >= 0; --b)
              if (a + b < 3) mma(a + b == 0 ? s[t] : rest[t], k[a][0], k[a][1], k[a][2], k[a][3], qb[b][t][at], qb[b][t][at + 1]);
      };
#pragma unroll
      for (int a = 0; a < R::kAtoms; ++a)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = a * (kStep * 128) + n * 128 + (((2 * q + h) ^ (n & 7)) << 4);
          const uint4 x = lds16(kp + at), y = lds16(kp + at + 8 * 128);
          if constexpr (kParts<T> == 1) {
            const uint32_t lo[1][4] = {{x.x, y.x, x.y, y.y}}, hi4[1][4] = {{x.z, y.z, x.w, y.w}};
            products(lo, 8 * a + 4 * h);
            products(hi4, 8 * a + 4 * h + 2);
          } else {
            uint32_t xl[3], xh[3], yl[3], yh[3];
            parts_of(__uint_as_float(x.x), __uint_as_float(x.y), xl);
            parts_of(__uint_as_float(x.z), __uint_as_float(x.w), xh);
            parts_of(__uint_as_float(y.x), __uint_as_float(y.y), yl);
            parts_of(__uint_as_float(y.z), __uint_as_float(y.w), yh);
            const uint32_t k[3][4] = {{xl[0], yl[0], xh[0], yh[0]}, {xl[1], yl[1], xh[1], yh[1]}, {xl[2], yl[2], xh[2], yh[2]}};
            products(k, 4 * a + 2 * h);
          }
        }
      __syncwarp();
      send(i + kStages, ahead_k, 0);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[t][k] = (kParts<T> > 1 ? s[t][k] + rest[t][k] : s[t][k]) * scale_log2;
      if (hi == kStep) weigh_logits<D, NT, false, 1>(st, s1, lane, 0, kStep);
      else weigh_logits<D, NT, true, 1>(st, s1, lane, 0, hi);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[t][k] *= 1.f / kUnit;
      uint32_t pa[kWeightParts<T, NT>][NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if constexpr (kParts<T> == 1) {
          const uint32_t a = cvt_bf16x2(s[t][0], s[t][1]), b = cvt_bf16x2(s[t][2], s[t][3]);
          pa[0][t][0] = transpose8x8(a);
          pa[0][t][1] = transpose8x8(b);
          if constexpr (kWeightParts<T, NT> == 2) {
            pa[1][t][0] = transpose8x8(cvt_bf16x2(s[t][0] - fc::bf16_lo(a), s[t][1] - fc::bf16_hi(a)));
            pa[1][t][1] = transpose8x8(cvt_bf16x2(s[t][2] - fc::bf16_lo(b), s[t][3] - fc::bf16_hi(b)));
          }
        } else {
          uint32_t a[3], b[3];
          parts_of(s[t][0], s[t][1], a);
          parts_of(s[t][2], s[t][3], b);
#pragma unroll
          for (int j = 0; j < 3; ++j) pa[j][t][0] = transpose8x8(a[j]), pa[j][t][1] = transpose8x8(b[j]);
        }
      }
      mbar_wait_bounded(bar(1, 1, stage), parity, abort);
      __syncwarp();
      const uint32_t vp = ring_s + kRing / 2 + stage * R::kPlain;
      auto piece = [&](int k, int a, int p) {  // 16-byte piece p of atom a of the lane's k-th key; zeros behind the run's end
        const int r = 2 * q + (k & 1) + 8 * (k >> 1);
        uint4 x = lds16(vp + a * (kStep * 128) + r * 128 + ((p ^ (r & 7)) << 4));
        if (r >= hi) x = make_uint4(0u, 0u, 0u, 0u);
        return x;
      };
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        if constexpr (kParts<T> == 1) {
          uint4 x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = piece(k, j, n);
          const uint32_t* y[4] = {&x[0].x, &x[1].x, &x[2].x, &x[3].x};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t a0 = prmt(y[0][w], y[1][w], 0x5410), a1 = prmt(y[0][w], y[1][w], 0x7632);
            const uint32_t a2 = prmt(y[2][w], y[3][w], 0x5410), a3 = prmt(y[2][w], y[3][w], 0x7632);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int b = kWeightParts<T, NT> - 1; b >= 0; --b) mma(st.o[t][4 * j + w], a0, a1, a2, a3, pa[b][t][0], pa[b][t][1]);
          }
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = piece(k, 2 * j + (n >> 2), (n & 3) * 2 + h);
            const uint32_t* y[4] = {&x[0].x, &x[1].x, &x[2].x, &x[3].x};
#pragma unroll
            for (int w = 0; w < 2; ++w) {  // dims 2w and 2w + 1 of the four that were read
              uint32_t e[4][3];
              parts_of(__uint_as_float(y[0][2 * w]), __uint_as_float(y[1][2 * w]), e[0]);
              parts_of(__uint_as_float(y[0][2 * w + 1]), __uint_as_float(y[1][2 * w + 1]), e[1]);
              parts_of(__uint_as_float(y[2][2 * w]), __uint_as_float(y[3][2 * w]), e[2]);
              parts_of(__uint_as_float(y[2][2 * w + 1]), __uint_as_float(y[3][2 * w + 1]), e[3]);
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                float x4[4] = {};
#pragma unroll
                for (int sum = 2; sum >= 0; --sum)  // the smallest products first
#pragma unroll
                  for (int a = 0; a <= sum; ++a) mma(x4, e[0][a], e[1][a], e[2][a], e[3][a], pa[sum - a][t][0], pa[sum - a][t][1]);
#pragma unroll
                for (int k = 0; k < 4; ++k) st.o[t][4 * j + 2 * h + w][k] += x4[k];
              }
            }
          }
        }
      }
      __syncwarp();
      send(i + kStages, ahead_v, 1);
    }
  }

  if (bad && g.status) atomicOr(g.status, (uint32_t)FC_DEV_BAD_INDEX);

  // ------------------------------------------------------------------ join the four warps
  if (*abort) {  // something never arrived: copies still in flight get time to land before their memory is used again
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  __syncthreads();
  if (tid == 0 && *abort && g.status) atomicOr(g.status, (uint32_t)FC_DEV_TIMEOUT);
  auto o_s = reinterpret_cast<float(*)[kRows][D + 4]>(smem);
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
      for (int j = 0; j < D / 64; ++j)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          o_s[warp][row][64 * j + 8 * n + 2 * w] = st.o[t][4 * j + w][r];
          o_s[warp][row][64 * j + 8 * n + 2 * w + 1] = st.o[t][4 * j + w][2 + r];
        }
    }
  __syncthreads();
  auto block_o = reinterpret_cast<float(*)[D + 4]>(smem + sizeof(float) * kWarps * kRows * (D + 4));
  auto block_ml = reinterpret_cast<float2*>(block_o + kRows);
  for (int x = tid; x < rows_here * (D / 4); x += kThreads) {
    const int row = x / (D / 4), d4 = x % (D / 4) * 4;
    float mx = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, ml_s[w][row].x);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float2 ml = ml_s[w][row];
      if (!(ml.y != 0.f)) continue;
      const float f = ex2(ml.x - mx);
      const float4 y = *reinterpret_cast<const float4*>(&o_s[w][row][d4]);
      l = fmaf(f, ml.y, l);
      o.x = fmaf(f, y.x, o.x); o.y = fmaf(f, y.y, o.y); o.z = fmaf(f, y.z, o.z); o.w = fmaf(f, y.w, o.w);
    }
    if (n_parts == 1) {
      write_row<T>(O, g, c, hk, v0 + row, d4, o, mx, l);
    } else if (g.cluster) {
      *reinterpret_cast<float4*>(&block_o[row][d4]) = o;
      if (d4 == 0) block_ml[row] = make_float2(mx, l);
    } else {
      const int64_t at = ((int64_t)hk * gridDim.x + blockIdx.x) * kRows + row;
      *reinterpret_cast<float4*>(g.part_o + at * D + d4) = o;
      if (d4 == 0) g.part_ml[at] = make_float2(mx, l);
    }
  }
  if (n_parts == 1 || !g.cluster) return;
  // the parts of the tile are the blocks of this cluster: each joins a share of the rows' pieces
  cluster_barrier();
  for (int x = part * kThreads + tid; x < rows_here * (D / 4); x += n_parts * kThreads) {
    const int row = x / (D / 4), d4 = x % (D / 4) * 4;
    const uint32_t at_o = smem_u32(&block_o[row][d4]), at_ml = smem_u32(&block_ml[row]);
    float2 ml[kMaxCluster];
    float4 y[kMaxCluster];
    float mx = -INFINITY, l = 0.f;
#pragma unroll
    for (int p = 0; p < kMaxCluster; ++p)
      if (p < n_parts) {
        ml[p] = cluster_load2(at_ml, p);
        y[p] = cluster_load4(at_o, p);
      }
#pragma unroll
    for (int p = 0; p < kMaxCluster; ++p)
      if (p < n_parts) mx = fmaxf(mx, ml[p].x);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int p = 0; p < kMaxCluster; ++p) {
      if (p >= n_parts || !(ml[p].y != 0.f)) continue;
      const float f = ex2(ml[p].x - mx);
      l = fmaf(f, ml[p].y, l);
      o.x = fmaf(f, y[p].x, o.x); o.y = fmaf(f, y[p].y, o.y); o.z = fmaf(f, y[p].z, o.z); o.w = fmaf(f, y[p].w, o.w);
    }
    write_row<T>(O, g, c, hk, v0 + row, d4, o, mx, l);
  }
  cluster_barrier();  // the others have read this block's memory
}

// Joins the parts of a tile's rows, a block a row; its four warps take the parts in turn.
template <typename T, int D>
__global__ void __launch_bounds__(128)
attention_span_join_kernel(T* __restrict__ O, const __grid_constant__ fc::SpanGeom g, int n_blocks) {
  constexpr int kLanes = D / 4, kSets = 128 / kLanes, kAhead = 8;  // lanes of a part's row; parts at once
  __shared__ float4 o_s[kSets][kLanes];
  __shared__ float l_s[kSets], m_s[4];
  const int tid = threadIdx.x, lane = tid % 32, hk = blockIdx.y, kRows = 8 * g.row_tiles;
  int c = 0, t0 = 0;  // chunk, and its first tile
  int tile = blockIdx.x / kRows;
  for (;; ++c) {
    const int tiles = ((g.q_row_off[c + 1] - g.q_row_off[c]) * g.group + kRows - 1) / kRows;
    if (tile < t0 + tiles) break;
    t0 += tiles;
  }
  tile -= t0;
  const int row = blockIdx.x % kRows, v = tile * kRows + row, n = g.parts[c];
  fc::pdl_wait();
  if (n == 1 || v >= (g.q_row_off[c + 1] - g.q_row_off[c]) * g.group || !fc::span_chunk_active(g, c)) return;
  const int64_t at = ((int64_t)hk * n_blocks + (c > 0 ? g.block_end[c - 1] : 0) + tile * n) * kRows + row;  // of the first part
  float m = -INFINITY;
  for (int p = tid; p < n; p += 128) m = fmaxf(m, g.part_ml[at + (int64_t)p * kRows].x);
#pragma unroll
  for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
  if (lane == 0) m_s[tid / 32] = m;
  __syncthreads();
  m = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3]));
  const int set = tid / kLanes, d4 = tid % kLanes;
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = set; p0 < n; p0 += kSets * kAhead) {
    float2 ml[kAhead];
    float4 y[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int p = p0 + i * kSets;
      if (p < n) {
        ml[i] = g.part_ml[at + (int64_t)p * kRows];
        y[i] = *reinterpret_cast<const float4*>(g.part_o + (at + (int64_t)p * kRows) * D + 4 * d4);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (p0 + i * kSets >= n || !(ml[i].y != 0.f)) continue;
      const float f = exp2f(ml[i].x - m);
      l = fmaf(f, ml[i].y, l);
      o.x = fmaf(f, y[i].x, o.x); o.y = fmaf(f, y[i].y, o.y); o.z = fmaf(f, y[i].z, o.z); o.w = fmaf(f, y[i].w, o.w);
    }
  }
  o_s[set][d4] = o;
  if (d4 == 0) l_s[set] = l;
  __syncthreads();
  if (set > 0) return;
#pragma unroll
  for (int i = 1; i < kSets; ++i) {
    const float4 y = o_s[i][d4];
    o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
    l += l_s[i];
  }
  write_row<T>(O, g, c, hk, v, 4 * d4, o, m, l);
}

constexpr int kMaxParts = 256;

// Units of cost of a chunk's keys (see the kernel), over pages and over plain rows.
struct Units {
  int64_t paged, plain;
  int64_t all() const { return std::max<int64_t>(1, paged + plain); }
};
Units units_of(const fc::SpanGeom& g, int c) {
  auto steps = [&](int i) { return g.hi[i][c] > g.lo[i][c] ? (g.hi[i][c] + kPagedStep - 1) / kPagedStep - g.lo[i][c] / kPagedStep : 0; };
  int64_t plain = 0;
  for (int i = 2; i < 4; ++i)
    for (int s = 0; s < g.n_seg; ++s) {
      const int n = std::min(g.hi[i][c], g.seg_log[s + 1]) - std::max(g.lo[i][c], g.seg_log[s]);
      if (n > 0) plain += (n + kStep - 1) / kStep;
    }
  return {(int64_t)kPagedCost * (steps(0) + steps(1)), plain * (g.f32 ? kPlainCost<float> : kPlainCost<__nv_bfloat16>)};
}

// Measured on B200, in microseconds a unit of cost (a step of a block's four warps, divided by four and by kPagedCost or kPlainCost): of a
// block alone on its SM, of one of two, and of an SM whose blocks keep it busy (D = 128: the bandwidth).
struct UnitUs {
  double alone, two, full;
};
UnitUs unit_us(const fc::SpanGeom& g, int nt, double plain) {  // plain: their share of all units
  static const UnitUs t[2][2][2][2] = {{{{{0.066, 0.098, 0.057}, {0.088, 0.099, 0.052}}, {{0.086, 0.123, 0.062}, {0.092, 0.103, 0.051}}},
                                        {{{0.112, 0.135, 0.100}, {0.109, 0.184, 0.095}}, {{0.124, 0.160, 0.100}, {0.111, 0.188, 0.094}}}},
                                       {{{{0.079, 0.116, 0.052}, {0.100, 0.126, 0.063}}, {{0.103, 0.160, 0.080}, {0.113, 0.145, 0.072}}},
                                        {{{0.140, 0.199, 0.095}, {0.178, 0.237, 0.122}}, {{0.166, 0.230, 0.115}, {0.210, 0.275, 0.138}}}}};
  const UnitUs &a = t[g.f32][g.d == 128][nt - 1][0], &b = t[g.f32][g.d == 128][nt - 1][1];
  return {a.alone + plain * (b.alone - a.alone), a.two + plain * (b.two - a.two), a.full + plain * (b.full - a.full)};
}

// How a call's keys are cut for tiles of 8 nt rows.
//   in clusters   every tile's keys into the same number of parts, at most 16, whose blocks are a cluster and join themselves
//   by size       every chunk's into parts of at most `size` units, which a second kernel joins (3.5 us and its bytes): where a few tiles see many keys,
//                 some chunks far more than others, or the clusters that fit leave much of the device empty (64 rows of 24 heads over 28000 tokens in
//                 pages: 100 us in three parts, 140 in clusters of two)
// of which the fastest is taken, by the times above; a call takes 4.8 us besides.
// Of 60 calls at random, of 5 to 60 us, the choice was within 1 % of the best of 32 cuts in the median, within 10 % for five in six, and at most 25 %
// above it; chunks that the device leaves out, which the host does not know, can cost more (41 and 63 % were seen where it left out five of six).
struct Cut {
  double us;
  int32_t cluster;
  int64_t size;
};
Cut cut_of(const fc_ctx* ctx, const fc::SpanGeom& g, int nt, const Units* units) {
  const double sm = ctx->sm_count, places = sm * blocks_per_sm(nt);
  int64_t tiles[FC_MAX_CHUNKS], all = 0, most = 1;
  double work = 0, plain = 0;
  for (int c = 0; c < g.W; ++c) {
    tiles[c] = (fc::span_rows(g, c) + 8 * nt - 1) / (8 * nt) * g.H_kv;
    all += tiles[c];
    work += (double)tiles[c] * units[c].all();
    plain += (double)tiles[c] * units[c].plain;
    if (tiles[c]) most = std::max(most, units[c].all());
  }
  const UnitUs u = unit_us(g, nt, work > 0 ? plain / work : 0);
  // Clusters lie unevenly: some SMs hold three blocks before every one holds two.
  auto time_of = [&](double blocks, double size, double room, bool clusters) {
    size = std::ceil(size / (kWarps * kPagedCost)) * (kWarps * kPagedCost);
    const double lone = blocks <= sm ? u.alone : blocks <= (clusters ? 1.75 : 2.0) * sm || nt == 2 ? u.two : 1.25 * u.two;
    if (blocks <= room) return size * std::max(lone, u.full * blocks / sm);
    return u.full * work / sm + 0.7 * size * u.alone + 3.5 * blocks / room;  // a set of blocks takes 3.5 us to start and end
  };
  Cut best = {0, 1, 0};
  for (int n = 1; n <= kMaxCluster && (n == 1 || most >= kWarps * n); ++n) {
    const int16_t* clusters = ctx->span_clusters[g.f32][g.d == 128][nt - 1];
    const int held = clusters[n];
    if (n > 1 && held == 0 && (n > 8 || clusters[2] > 0)) break;  // not a size that the device takes
    const double room = n == 1 ? places : held > 0 ? (double)held * n : 0.75 * places;
    const double us = 4.8 + (n > 1 ? 0.5 + 0.1 * n : 0) + time_of((double)all * n, (double)((most + n - 1) / n), room, n > 1);
    if (n == 1 || us < best.us) best = {us, n, 0};
  }
  if (0.95 * best.us <= 4.8 + 3.5 + u.full * work / sm) return best;  // no cut by size is below that
  for (int64_t n = 2; n <= kMaxParts && most >= 2 * kWarps * n; n += (n + 7) / 8) {
    const int64_t size = (most + n - 1) / n;
    double blocks = 0, rows = 0;
    for (int c = 0; c < g.W; ++c) {
      const double parts = (double)((units[c].all() + size - 1) / size);
      blocks += tiles[c] * parts;
      if (parts > 1) rows += tiles[c] * parts * 8 * nt;
    }
    const double us = 4.8 + 3.5 + 2.0 * 4 * g.d * rows / 4e6 + time_of(blocks, (double)size, places, false);
    if (us < best.us) best = {us, 0, size};
  }
  return best;
}

double split(const fc_ctx* ctx, fc::SpanGeom& g) {
  Units units[FC_MAX_CHUNKS];
  bool many = false;
  for (int c = 0; c < g.W; ++c) {
    units[c] = units_of(g, c);
    many |= fc::span_rows(g, c) > 8;
  }
  // sixteen rows to a tile where some chunk has more than eight, unless twice the tiles are faster
  int nt = 1;
  Cut cut = cut_of(ctx, g, 1, units);
  if (many) {
    const Cut two = cut_of(ctx, g, 2, units);
    if (two.us + 0.7 < cut.us) cut = two, nt = 2;
  }
  g.row_tiles = nt;
  g.cluster = cut.cluster;
  int64_t blocks = 0;
  for (int c = 0; c < g.W; ++c) {
    const int64_t n = units[c].all(), parts = cut.cluster ? cut.cluster : (n + cut.size - 1) / cut.size;
    g.parts[c] = (int32_t)parts;
    constexpr int kRound = kWarps * kPagedCost;
    g.part_units[c] = (int32_t)(((n + parts - 1) / parts + kRound - 1) / kRound * kRound);  // whole rounds of the warps
    blocks += (fc::span_rows(g, c) + 8 * nt - 1) / (8 * nt) * parts;
    g.block_end[c] = (int32_t)std::min<int64_t>(blocks, INT32_MAX);
  }
  return cut.us;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode(fc_ctx* ctx, CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims,
           const cuuint64_t* strides, const cuuint32_t* box, CUtensorMapSwizzle swizzle) {
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  if (((EncodeTiledFn)ctx->encode_tiled)(map, type, rank, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                         swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
    fc::set_cuda_error(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    return FC_ERR_CUDA;
  }
  return FC_OK;
}
// Pages of codes: a box is 32 rows of a block, or all 16.
int map_pages(fc_ctx* ctx, CUtensorMap* map, const void* base, const fc::SpanGeom& g) {
  const int page = 1 << g.pool.page_log2;
  const int64_t block = (int64_t)page * g.d;  // the stride of an axis of one entry is never used, but has to be a valid one
  const cuuint64_t dims[4] = {(cuuint64_t)g.d, (cuuint64_t)page, (cuuint64_t)g.H_kv, (cuuint64_t)g.pool.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)g.d, (cuuint64_t)(g.H_kv > 1 ? g.pool.code_hs : block), (cuuint64_t)(g.pool.n_pages > 1 ? g.pool.code_ps : block)};
  const cuuint32_t box[4] = {(cuuint32_t)g.d, (cuuint32_t)std::min(page, kPagedStep), 1, 1};
  return encode(ctx, map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, base, dims, strides, box, g.d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}
// Plain rows: a box is 128 bytes of 16 rows.
int map_rows(fc_ctx* ctx, CUtensorMap* map, const void* base, const fc::SpanGeom& g, int64_t hs, int64_t rs) {
  const int es = g.f32 ? 4 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)g.d, (cuuint64_t)g.kv_rows, (cuuint64_t)g.H_kv};
  const cuuint64_t strides[2] = {(cuuint64_t)rs * es, (cuuint64_t)(g.H_kv > 1 ? hs : rs) * es};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / es), kStep, 1};
  return encode(ctx, map, g.f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}


// Clusters of n blocks that the device holds at once.
template <typename T, int D, int NT>
void ask_clusters(int16_t (&held)[kMaxCluster + 1]) {
  auto kernel = attention_span_rows_kernel<T, D, NT>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
    return;
  for (int n = 2; n <= kMaxCluster; ++n) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)n;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int count = 0;
    if (cudaOccupancyMaxActiveClusters(&count, kernel, &cfg) == cudaSuccess) held[n] = (int16_t)std::min(count, 30000);
  }
}

}  // namespace

namespace fc {

void span_rows_setup(fc_ctx* ctx) {
  auto& h = ctx->span_clusters;
  for (auto& a : h)
    for (auto& b : a)
      for (auto& c : b)
        for (int16_t& x : c) x = 0;
  ask_clusters<__nv_bfloat16, 64, 1>(h[0][0][0]);
  ask_clusters<__nv_bfloat16, 64, 2>(h[0][0][1]);
  ask_clusters<__nv_bfloat16, 128, 1>(h[0][1][0]);
  ask_clusters<__nv_bfloat16, 128, 2>(h[0][1][1]);
  ask_clusters<float, 64, 1>(h[1][0][0]);
  ask_clusters<float, 64, 2>(h[1][0][1]);
  ask_clusters<float, 128, 1>(h[1][1][0]);
  ask_clusters<float, 128, 2>(h[1][1][1]);
  cudaGetLastError();  // a question that was refused is no error of a call
}

size_t span_rows_workspace(const fc_ctx* ctx, SpanGeom& g) {
  g.rows_us = split(ctx, g);
  bool joined = false;
  for (int c = 0; c < g.W; ++c) joined |= g.parts[c] > 1;
  if (!joined || g.cluster) return 0;
  const size_t rows = (size_t)g.H_kv * g.block_end[g.W - 1] * 8 * g.row_tiles;
  return align_up(rows * g.d * sizeof(float), 256) + align_up(rows * sizeof(float2), 256);
}

int span_rows_launch(fc_ctx* ctx, cudaStream_t st, const SpanGeom& g, const void* Q, const void* K, const void* V, void* O) {
  const int nt = g.row_tiles, blocks = g.block_end[g.W - 1];
  if (blocks == 0) return FC_OK;
  if (blocks == INT32_MAX) return FC_ERR_UNSUPPORTED;
  bool paged = false, plain = false, joined = false;
  int64_t rows = 0;
  for (int c = 0; c < g.W; ++c) {
    paged |= g.hi[0][c] > g.lo[0][c] || g.hi[1][c] > g.lo[1][c];
    plain |= g.hi[2][c] > g.lo[2][c] || g.hi[3][c] > g.lo[3][c];
    joined |= g.parts[c] > 1;
    rows += (span_rows(g, c) + 8 * nt - 1) / (8 * nt) * 8 * nt;
  }
  if (rows > INT32_MAX) return FC_ERR_UNSUPPORTED;
  CUtensorMap k8 = {}, v8 = {}, k = {}, v = {};
  int rc;
  if (paged && ((rc = map_pages(ctx, &k8, g.pool.k_codes, g)) != FC_OK || (rc = map_pages(ctx, &v8, g.pool.v_codes, g)) != FC_OK)) return rc;
  if (plain && ((rc = map_rows(ctx, &k, K, g, g.k_hs, g.k_rs)) != FC_OK || (rc = map_rows(ctx, &v, V, g, g.v_hs, g.v_rs)) != FC_OK)) return rc;
  const dim3 grid((unsigned)blocks, (unsigned)g.H_kv);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;  // which span_rows_setup allowed, and clusters of up to sixteen
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)std::max(g.cluster, 1);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = g.cluster > 1 ? 1 : 0;
#define FC_SPAN_ROWS(T, D, NT)                                                                                                        \
  do {                                                                                                                                \
    static_assert((kWarps + 1) * 8 * NT * (D + 4) * 4 + 8 * NT * 8 <= kWarps * kRing, "what is joined takes the rings' place");       \
    FC_CUDA_CHECK(cudaLaunchKernelEx(&cfg, attention_span_rows_kernel<T, D, NT>, k8, v8, k, v, (const T*)Q, (T*)O, g));                \
  } while (0)
#define FC_SPAN_ROWS_PICK(T)                                                                       \
  do {                                                                                             \
    if (g.d == 128) { if (nt == 1) FC_SPAN_ROWS(T, 128, 1); else FC_SPAN_ROWS(T, 128, 2); }        \
    else { if (nt == 1) FC_SPAN_ROWS(T, 64, 1); else FC_SPAN_ROWS(T, 64, 2); }                     \
  } while (0)
  if (g.f32) FC_SPAN_ROWS_PICK(float);
  else FC_SPAN_ROWS_PICK(__nv_bfloat16);
#undef FC_SPAN_ROWS_PICK
#undef FC_SPAN_ROWS
  FC_LAUNCH_CHECK("attention_span_rows_kernel");
  if (!joined || g.cluster) return FC_OK;
  const dim3 join((unsigned)rows, (unsigned)g.H_kv);
  cudaError_t e;
  if (g.f32) e = g.d == 128 ? launch_pdl(attention_span_join_kernel<float, 128>, join, dim3(128), 0, st, (float*)O, g, blocks)
                            : launch_pdl(attention_span_join_kernel<float, 64>, join, dim3(128), 0, st, (float*)O, g, blocks);
  else e = g.d == 128 ? launch_pdl(attention_span_join_kernel<__nv_bfloat16, 128>, join, dim3(128), 0, st, (__nv_bfloat16*)O, g, blocks)
                      : launch_pdl(attention_span_join_kernel<__nv_bfloat16, 64>, join, dim3(128), 0, st, (__nv_bfloat16*)O, g, blocks);
  FC_CUDA_CHECK(e);
  FC_LAUNCH_CHECK("attention_span_join_kernel");
  return FC_OK;
}

}  // namespace fc
