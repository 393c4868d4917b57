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

struct Plan {
  bool tiles;  // the tcgen05 kernel
  size_t bytes;
};
Plan plan(const fc_ctx* ctx, const fc_attn_desc* desc, fc::SpanGeom& g) {
  (void)desc;
  Plan p = {};
  p.bytes = fc::span_rows_workspace(ctx, g);
  return p;
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
  g.q_hs = desc->q_hs; g.q_rs = desc->q_rs; g.k_hs = desc->k_hs; g.k_rs = desc->k_rs;
  g.v_hs = desc->v_hs; g.v_rs = desc->v_rs; g.o_hs = desc->o_hs; g.o_rs = desc->o_rs;
  g.kv_rows = std::min<int64_t>(desc->kv_rows, INT32_MAX);
  g.lse_hs = lse_hs;
  g.active_ids = active_ids; g.n_active = n_active; g.lse = lse; g.status = status;

  const Plan p = plan(ctx, desc, g);
  if (p.bytes > 0) {
    if (!ws || ws_bytes < p.bytes) return FC_ERR_WORKSPACE;
    if (!fc::aligned16(ws)) return FC_ERR_MISALIGNED;
  }
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
  if (p.bytes > 0) {
    const size_t r = (size_t)g.H_kv * g.block_end[g.W - 1] * 8 * g.row_tiles;
    g.part_o = (float*)ws;
    g.part_ml = (float2*)((char*)ws + fc::align_up(r * g.d * sizeof(float), 256));
  }
  return fc::span_rows_launch(ctx, st, g, Q, K, V, O);
}

size_t workspace(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype, int page, int64_t table_cs, const int32_t* q_chunk_row_off,
                 const Visible& visible, const int32_t* seg_logical_off, int n_seg) {
  fc::SpanGeom g = {};
  if (!ctx || check_geometry(desc, dtype, page, table_cs, q_chunk_row_off, visible, seg_logical_off, n_seg, g) != FC_OK) return 0;
  if (g.q_row_off[g.W] == g.q_row_off[0]) return 0;
  return plan(ctx, desc, g).bytes;
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
