// fc_chunk_attention_kv8 and fc_chunk_attention_span: argument validation and the choice of the kernel.
#include <algorithm>
#include <climits>
#include <cmath>

#include "fc_attention_span.cuh"

namespace {

// The arguments that say which tokens a chunk sees.
struct Visible {
  const int32_t *cache_len, *vis, *begin, *window_first;  // any but vis may be NULL
  int32_t n_sink;
};

// The part of the arguments that the workspace depends on.
int check_geometry(const fc_attn_desc* desc, int dtype, int page, int64_t table_cs, const int32_t* q_chunk_row_off, const Visible& v,
                   const int32_t* seg_logical_off, int n_seg, fc::SpanGeom& g) {
  if (!desc || !q_chunk_row_off || !v.vis || n_seg < 0 || v.n_sink < 0) return FC_ERR_INVALID_ARG;
  if (dtype != FC_BF16 && dtype != FC_F32) return FC_ERR_UNSUPPORTED;
  if (desc->d != 64 && desc->d != 128) return FC_ERR_UNSUPPORTED;
  if (desc->H_q <= 0 || desc->H_kv <= 0 || desc->H_q % desc->H_kv || desc->W <= 0) return FC_ERR_INVALID_ARG;
  if (desc->W > FC_MAX_CHUNKS || desc->H_kv > 65535 || n_seg > FC_MAX_SEGMENTS - 2) return FC_ERR_UNSUPPORTED;
  if (desc->impl != 0 && desc->impl != 2 && desc->impl != 3) return FC_ERR_INVALID_ARG;
  if (!(desc->scale >= 0.f)) return FC_ERR_INVALID_ARG;
  if (desc->impl == 2 && dtype != FC_BF16) return FC_ERR_UNSUPPORTED;
  g.H_q = desc->H_q; g.H_kv = desc->H_kv; g.d = desc->d; g.W = desc->W;
  g.group = desc->H_q / desc->H_kv;
  g.scale = desc->scale != 0.f ? desc->scale : 1.f / sqrtf((float)desc->d);
  g.f32 = dtype == FC_F32;
  g.n_seg = n_seg;
  g.table_cs = table_cs;
  if (n_seg > 0) {
    if (!seg_logical_off) return FC_ERR_INVALID_ARG;
    for (int s = 0; s <= n_seg; ++s) {
      if (s == 0 ? seg_logical_off[0] != 0 : seg_logical_off[s] < seg_logical_off[s - 1]) return FC_ERR_INVALID_ARG;
      g.seg_log[s] = seg_logical_off[s];
    }
  }
  const int64_t plain = n_seg > 0 ? g.seg_log[n_seg] : 0;
  if (plain > INT32_MAX - 4096) return FC_ERR_UNSUPPORTED;
  for (int c = 0; c <= g.W; ++c) {
    if (q_chunk_row_off[c] < 0 || (c > 0 && q_chunk_row_off[c] < q_chunk_row_off[c - 1])) return FC_ERR_INVALID_ARG;
    g.q_row_off[c] = q_chunk_row_off[c];
  }
  if ((int64_t)(g.q_row_off[g.W] - g.q_row_off[0]) * g.group > INT32_MAX - 4096) return FC_ERR_UNSUPPORTED;
  bool paged = false;
  for (int c = 0; c < g.W; ++c) {
    const int64_t n = v.cache_len ? v.cache_len[c] : 0, vis = v.vis[c], first = v.window_first ? v.window_first[c] : 0;
    const int64_t begin = v.begin ? v.begin[c] : 0;
    if (n < 0 || vis < 0 || first < 0 || begin < 0) return FC_ERR_INVALID_ARG;
    if (n + plain > INT32_MAX - 4096) return FC_ERR_UNSUPPORTED;  // logical offsets are 32-bit, and counters may run past the end by a step
    if (vis > n && first + (vis - n) > plain) return FC_ERR_INVALID_ARG;
    // [0, sink) and [from, vis), one piece where they meet
    int64_t sink = std::min<int64_t>(v.n_sink, vis), from = std::max(std::min(begin, vis), sink);
    if (from == sink) sink = from = 0;
    const int64_t cut[4][2] = {{0, std::min(sink, n)}, {std::min(from, n), std::min(vis, n)},
                               {first, first + std::max<int64_t>(sink - n, 0)},
                               {first + std::max<int64_t>(from - n, 0), first + std::max<int64_t>(vis - n, 0)}};
    for (int i = 0; i < 4; ++i) {
      g.lo[i][c] = (int32_t)cut[i][0];
      g.hi[i][c] = (int32_t)std::max(cut[i][0], cut[i][1]);
      if (i < 2) paged |= g.hi[i][c] > g.lo[i][c];
    }
  }
  if (paged) {
    g.pool.page_log2 = fc::page_log2(page);
    if (g.pool.page_log2 < 0) return FC_ERR_UNSUPPORTED;
    if (table_cs < 0) return FC_ERR_INVALID_ARG;
  }
  return FC_OK;
}

bool sees_pages(const fc::SpanGeom& g) {
  for (int c = 0; c < g.W; ++c)
    if (g.hi[0][c] > g.lo[0][c] || g.hi[1][c] > g.lo[1][c]) return true;
  return false;
}
bool sees_rows(const fc::SpanGeom& g) {
  for (int c = 0; c < g.W; ++c)
    if (g.hi[2][c] > g.lo[2][c] || g.hi[3][c] > g.lo[3][c]) return true;
  return false;
}

// The tcgen05 path: what is seen of the pages is unpacked into the workspace first, [H_kv, rows, d] of K and of V, and the tokens'
// spans become rows of that.
struct TilePlan {
  fc::AttnSplit split;
  fc::AttnSpans spans;
  fc::Kv8Jobs jobs;
  int32_t vis[FC_MAX_CHUNKS];  // keys that each chunk sees
  int rows;                    // of the workspace, per head
  size_t k, v, plan, o, ml, bytes;  // offsets
  double us;                        // estimate of the whole path
};

constexpr double kTilesUs = 12;  // what the path takes besides its work, measured

// False if there are more rows to unpack than a tensor map's place can name.
bool plan_tiles(const fc_ctx* ctx, const fc::SpanGeom& g, TilePlan& p) {
  // the tokens to unpack: of the shared sequence those that some chunk sees, else each chunk's own
  p.jobs = {};
  const bool shared = g.table_cs == 0;
  for (int c = 0; c < g.W; ++c) {
    for (int i = 0; i < 4; ++i) p.spans.lo[i][c] = g.lo[i][c], p.spans.hi[i][c] = g.hi[i][c];
    p.vis[c] = 0;
    for (int i = 0; i < 4; ++i) p.vis[c] += g.hi[i][c] - g.lo[i][c];
  }
  p.rows = 0;
  p.jobs.W = g.W;
  for (int c0 = 0; c0 < g.W; c0 += shared ? g.W : 1) {
    const int c1 = shared ? g.W : c0 + 1;
    // What is seen, in order, cut wherever the set of chunks that see it changes: a job is brought only if one of its chunks is active, and
    // entries that nobody needs are nobody's concern.  Jobs that meet lie next to each other, so that a chunk's range stays one.
    struct End {
      int32_t at;
      uint64_t who;  // begins or ends to see
    } end[4 * FC_MAX_CHUNKS];
    int n = 0;
    for (int c = c0; c < c1; ++c)
      for (int i = 0; i < 2; ++i)
        if (g.hi[i][c] > g.lo[i][c] && fc::span_rows(g, c) > 0) end[n++] = {g.lo[i][c], 1ull << c}, end[n++] = {g.hi[i][c], 1ull << c};
    std::sort(end, end + n, [](const End& a, const End& b) { return a.at < b.at; });
    const int first_job = p.jobs.n;
    uint64_t who = 0;
    for (int k = 0; k + 1 < n; ++k) {
      who ^= end[k].who;
      const int64_t len = (int64_t)end[k + 1].at - end[k].at;
      if (who == 0 || len == 0) continue;
      if (p.rows + len > INT32_MAX - 4096) return false;
      p.jobs.needed[p.jobs.n] = who;
      p.jobs.job[p.jobs.n++] = {shared ? 0 : c0, end[k].at, (int32_t)len, p.rows};
      p.rows += (int)len;
    }
    for (int c = c0; c < c1; ++c)
      for (int i = 0; i < 2; ++i) {
        if (g.hi[i][c] <= g.lo[i][c] || fc::span_rows(g, c) == 0) {
          p.spans.lo[i][c] = p.spans.hi[i][c] = 0;
          continue;
        }
        const fc::Kv8Job* job = std::upper_bound(p.jobs.job + first_job, p.jobs.job + p.jobs.n, g.lo[i][c],
                                                 [](int32_t token, const fc::Kv8Job& x) { return token < x.first; }) - 1;
        p.spans.lo[i][c] += job->dst_row - job->first;
        p.spans.hi[i][c] += job->dst_row - job->first;
      }
  }
  // grouped heads share their key tiles where whole groups fill a tile of 128 rows
  p.split = fc::AttnSplit();
  if (128 % g.group == 0 && (int64_t)g.q_row_off[g.W] * g.group <= INT32_MAX - 4096) p.split.pack = g.group;
  int64_t items = 0, tiles = 0;  // work items of 256 rows, and the key tiles that they take together
  int most = 0;
  for (int c = 0; c < g.W; ++c) {
    const int64_t n = ((int64_t)(g.q_row_off[c + 1] - g.q_row_off[c]) * p.split.pack + 255) / 256;
    items += n;
    tiles += n * ((p.vis[c] + 127) / 128);
    if (n > 0) most = std::max(most, p.vis[c]);
  }
  items *= g.H_q / p.split.pack;
  tiles *= g.H_q / p.split.pack;
  const int most_tiles = (most + 127) / 128;
  if (most_tiles >= 6) p.split.slots = (int32_t)std::min<int64_t>(3 * ctx->sm_count, items * fc::kMaxParts);
  float last = 0.f;
  const int rest = (int)(items % ctx->sm_count);
  if (rest > 0) fc::split_parts(rest, ctx->sm_count, most_tiles, g.d, p.split.slots, &last);
  // the launches of the path, 1.8 us a key tile, the unpacking at 6.4 TB/s
  const double whole = items > 0 ? (double)tiles / items : 0;
  p.us = kTilesUs + 1.8 * ((double)(items / ctx->sm_count) * whole + last) + 2.0 * g.H_kv * p.rows * g.d * 3 / 6.4e6;
  const size_t bytes = (size_t)g.H_kv * p.rows * g.d * 2, parts = (size_t)p.split.slots * 256;
  p.k = fc::attention_tc_workspace_bytes();
  p.v = p.k + fc::align_up(bytes, 256);
  p.plan = p.v + fc::align_up(bytes, 256);
  p.o = p.plan + fc::align_up((4 + 4 * (size_t)ctx->sm_count) * sizeof(int32_t), 256);
  p.ml = p.o + parts * g.d * sizeof(float);
  p.bytes = p.ml + parts * sizeof(float2);
  return true;
}

// Strides of Q that a tensor map takes.  The kernel for few rows takes any.
bool maps_fit(const fc_attn_desc* d) { return d->q_rs < (1ll << 38) && (d->H_q == 1 || (d->q_hs > 0 && d->q_hs < (1ll << 31))); }

// What a call does, with the workspace it takes and the split of the keys in g.
struct Plan {
  bool tiles;  // the tcgen05 kernel
  TilePlan t;
  size_t bytes;
};
int plan(const fc_ctx* ctx, const fc_attn_desc* desc, fc::SpanGeom& g, Plan& p) {
  p.tiles = false;
  if (desc->impl != 2) {
    p.bytes = fc::span_rows_workspace(ctx, g);
    if (desc->impl == 3 || g.f32 || g.rows_us <= kTilesUs) return FC_OK;
  }
  const bool fits = maps_fit(desc) && plan_tiles(ctx, g, p.t);
  if (!fits && desc->impl == 2) return FC_ERR_UNSUPPORTED;
  if (fits && (desc->impl == 2 || p.t.us < g.rows_us)) {
    p.tiles = true;
    p.bytes = p.t.bytes;
  }
  return FC_OK;
}

int attend(fc_ctx* ctx, void* stream, const fc_attn_desc* desc, const void* Q, const fc_kv8_pool* pool, const int32_t* table,
           int64_t table_cs, const void* K, const void* V, int dtype, const int32_t* q_chunk_row_off, const Visible& visible,
           const int32_t* seg_logical_off, const int32_t* seg_phys_off, int n_seg, const int32_t* active_ids,
           const int32_t* n_active, void* O, float* lse, int64_t lse_hs, uint32_t* status, void* ws, size_t ws_bytes) {
  if (!ctx) return FC_ERR_INVALID_ARG;
  fc::SpanGeom g = {};
  int rc = check_geometry(desc, dtype, pool ? pool->page : 0, table_cs, q_chunk_row_off, visible, seg_logical_off, n_seg, g);
  if (rc != FC_OK) return rc;
  if (g.q_row_off[g.W] == g.q_row_off[0]) return FC_OK;
  if (!Q || !O || !active_ids || !n_active) return FC_ERR_INVALID_ARG;
  const int es = fc::elem_size(dtype);
  const bool rows = sees_rows(g), pages = sees_pages(g);
  const int64_t strides[8] = {desc->q_hs, desc->q_rs, desc->o_hs, desc->o_rs, desc->k_hs, desc->k_rs, desc->v_hs, desc->v_rs};
  for (int i = 0; i < (rows ? 8 : 4); ++i) {
    if (strides[i] < 0 || (strides[i] * es) % 16) return FC_ERR_MISALIGNED;
    if (i % 2 && strides[i] < desc->d) return FC_ERR_INVALID_ARG;
    if (i >= 4 && (strides[i] >= (1ll << 36) || (i % 2 == 0 && g.H_kv > 1 && strides[i] == 0))) return FC_ERR_UNSUPPORTED;  // what a tensor map takes
  }
  if (desc->H_q > 1 && desc->o_hs < desc->d) return FC_ERR_INVALID_ARG;  // heads of O would overlap
  if (!fc::aligned16(Q) || !fc::aligned16(O)) return FC_ERR_MISALIGNED;
  if (pages) {
    if (!pool || !table) return FC_ERR_INVALID_ARG;
    if ((rc = fc::kv8_check(pool, g.H_kv, g.d)) != FC_OK) return rc;
    g.pool = fc::kv8_view(*pool);
    g.table = table;
  }
  if (n_seg > 0) {
    if (!seg_phys_off) return FC_ERR_INVALID_ARG;
    if (rows && (!K || !V)) return FC_ERR_INVALID_ARG;
    if (rows && (!fc::aligned16(K) || !fc::aligned16(V))) return FC_ERR_MISALIGNED;
    for (int s = 0; s < n_seg; ++s) {
      const int64_t len = g.seg_log[s + 1] - g.seg_log[s];
      if (seg_phys_off[s] < 0 || seg_phys_off[s] + len > desc->kv_rows) return FC_ERR_INVALID_ARG;
      if (seg_phys_off[s] + len > INT32_MAX - 4096) return FC_ERR_UNSUPPORTED;  // a row's place in a tensor map is 32-bit
      g.seg_phys[s] = seg_phys_off[s];
    }
  }
  if (lse && lse_hs <= 0) return FC_ERR_INVALID_ARG;
  if (!rows) g.n_seg = 0;
  g.q_hs = desc->q_hs; g.q_rs = desc->q_rs; g.k_hs = desc->k_hs; g.k_rs = desc->k_rs;
  g.v_hs = desc->v_hs; g.v_rs = desc->v_rs; g.o_hs = desc->o_hs; g.o_rs = desc->o_rs;
  g.kv_rows = std::min<int64_t>(desc->kv_rows, INT32_MAX);
  g.lse_hs = lse_hs;
  g.active_ids = active_ids; g.n_active = n_active; g.lse = lse; g.status = status;

  Plan p;
  if ((rc = plan(ctx, desc, g, p)) != FC_OK) return rc;
  if (p.bytes > 0) {
    if (!ws || ws_bytes < p.bytes) return FC_ERR_WORKSPACE;
    if (!fc::aligned16(ws)) return FC_ERR_MISALIGNED;
  }
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
  char* base = (char*)ws;
  if (!p.tiles) {
    if (p.bytes > 0) {
      const size_t r = (size_t)g.H_kv * g.block_end[g.W - 1] * 8 * g.row_tiles;
      g.part_o = (float*)ws;
      g.part_ml = (float2*)(base + fc::align_up(r * g.d * sizeof(float), 256));
    }
    return fc::span_rows_launch(ctx, st, g, Q, K, V, O);
  }
  TilePlan& t = p.t;
  fc::AttnGeom a = {};
  a.H_q = g.H_q; a.H_kv = g.H_kv; a.d = g.d; a.W = g.W; a.group = g.group; a.n_seg = rows ? g.n_seg : 0;
  a.q_hs = g.q_hs; a.q_rs = g.q_rs; a.k_hs = g.k_hs; a.k_rs = g.k_rs; a.v_hs = g.v_hs; a.v_rs = g.v_rs; a.o_hs = g.o_hs; a.o_rs = g.o_rs;
  a.kv_rows = g.kv_rows; a.lse_hs = g.lse_hs; a.scale = g.scale;
  std::copy(g.q_row_off, g.q_row_off + g.W + 1, a.q_row_off);
  std::copy(t.vis, t.vis + g.W, a.vis);
  std::copy(g.seg_log, g.seg_log + g.n_seg + 1, a.seg_log);
  std::copy(g.seg_phys, g.seg_phys + g.n_seg, a.seg_phys);
  a.active_ids = active_ids; a.n_active = n_active; a.lse = lse; a.status = status;
  struct Unpack {
    cudaStream_t st;
    const fc::SpanGeom* g;
    const TilePlan* t;
    void *k, *v;
    uint32_t* counter;
  } unpack = {st, &g, &t, base + t.k, base + t.v, (uint32_t*)ws};
  auto before = [](void* arg) -> int {
    const Unpack& x = *(const Unpack*)arg;
    const int64_t hs = (int64_t)x.t->rows * x.g->d;
    return fc::kv8_unpack_launch(x.st, x.g->pool, x.g->H_kv, x.g->d, x.g->table, x.g->table_cs, x.t->jobs, x.k, x.v, x.t->rows, FC_BF16, hs, x.g->d, hs,
                                 x.g->d, x.g->status, x.counter);
  };
  t.jobs.active_ids = active_ids;
  t.jobs.n_active = n_active;
  t.split.follows = t.rows > 0;
  t.split.o = (float*)(base + t.o);
  t.split.ml = (float2*)(base + t.ml);
  t.split.plan = (int32_t*)(base + t.plan);
  return fc::attention_tc_two(ctx, st, a, Q, base + t.k, base + t.v, t.rows, K, V, t.split, O, ws, ws_bytes, before, &unpack, &t.spans);
}

size_t workspace(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype, int page, int64_t table_cs, const int32_t* q_chunk_row_off,
                 const Visible& visible, const int32_t* seg_logical_off, int n_seg) {
  fc::SpanGeom g = {};
  if (!ctx || check_geometry(desc, dtype, page, table_cs, q_chunk_row_off, visible, seg_logical_off, n_seg, g) != FC_OK) return 0;
  if (g.q_row_off[g.W] == g.q_row_off[0]) return 0;
  Plan p;
  return plan(ctx, desc, g, p) == FC_OK ? p.bytes : 0;
}

}  // namespace

extern "C" size_t fc_chunk_attention_kv8_workspace_bytes(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype, int page, int64_t table_cs,
                                                         const int32_t* cache_len, const int32_t* q_chunk_row_off,
                                                         const int32_t* kv_visible_len, int n_sink, const int32_t* kv_begin,
                                                         const int32_t* window_first, const int32_t* seg_logical_off, int n_seg) {
  return workspace(ctx, desc, dtype, page, table_cs, q_chunk_row_off, {cache_len, kv_visible_len, kv_begin, window_first, n_sink},
                   seg_logical_off, n_seg);
}

extern "C" int fc_chunk_attention_kv8(fc_ctx* ctx, void* stream, const fc_attn_desc* desc, const void* Q, const fc_kv8_pool* pool,
                                      const int32_t* table, int64_t table_cs, const int32_t* cache_len, const void* K, const void* V,
                                      int dtype, const int32_t* q_chunk_row_off, const int32_t* kv_visible_len, int n_sink,
                                      const int32_t* kv_begin, const int32_t* window_first, const int32_t* seg_logical_off,
                                      const int32_t* seg_phys_off, int n_seg, const int32_t* active_ids, const int32_t* n_active,
                                      void* O, float* lse, int64_t lse_hs, uint32_t* status, void* ws, size_t ws_bytes) {
  return attend(ctx, stream, desc, Q, pool, table, table_cs, K, V, dtype, q_chunk_row_off,
                {cache_len, kv_visible_len, kv_begin, window_first, n_sink}, seg_logical_off, seg_phys_off, n_seg, active_ids, n_active, O,
                lse, lse_hs, status, ws, ws_bytes);
}

extern "C" size_t fc_chunk_attention_span_workspace_bytes(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype,
                                                          const int32_t* q_chunk_row_off, const int32_t* kv_visible_len, int n_sink,
                                                          const int32_t* kv_begin, const int32_t* seg_logical_off, int n_seg) {
  return workspace(ctx, desc, dtype, 0, 0, q_chunk_row_off, {nullptr, kv_visible_len, kv_begin, nullptr, n_sink}, seg_logical_off, n_seg);
}

extern "C" int fc_chunk_attention_span(fc_ctx* ctx, void* stream, const fc_attn_desc* desc, const void* Q, const void* K, const void* V,
                                       int dtype, const int32_t* q_chunk_row_off, const int32_t* kv_visible_len, int n_sink,
                                       const int32_t* kv_begin, const int32_t* seg_logical_off, const int32_t* seg_phys_off, int n_seg,
                                       const int32_t* active_ids, const int32_t* n_active, void* O, float* lse, int64_t lse_hs,
                                       uint32_t* status, void* ws, size_t ws_bytes) {
  return attend(ctx, stream, desc, Q, nullptr, nullptr, 0, K, V, dtype, q_chunk_row_off, {nullptr, kv_visible_len, kv_begin, nullptr, n_sink},
                seg_logical_off, seg_phys_off, n_seg, active_ids, n_active, O, lse, lse_hs, status, ws, ws_bytes);
}
