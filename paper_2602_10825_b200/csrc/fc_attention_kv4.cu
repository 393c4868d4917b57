// fc_chunk_attention_kv4: argument validation and the choice of the kernel.
#include <algorithm>
#include <climits>
#include <cmath>

#include "fc_attention_kv4.cuh"

namespace {

// The part of the arguments that the workspace depends on.
int check_geometry(const fc_attn_desc* desc, int dtype, const int32_t* q_chunk_row_off, const int32_t* kv_visible_len,
                   int n_cache, fc::Kv4AttnGeom& g) {
  if (!desc || !q_chunk_row_off || !kv_visible_len) return FC_ERR_INVALID_ARG;
  if (dtype != FC_BF16 && dtype != FC_F32) return FC_ERR_UNSUPPORTED;
  if (desc->d != 64 && desc->d != 128) return FC_ERR_UNSUPPORTED;
  if (desc->H_q <= 0 || desc->H_kv <= 0 || desc->H_q % desc->H_kv || desc->W <= 0 || n_cache < 0) return FC_ERR_INVALID_ARG;
  if (desc->W > FC_MAX_CHUNKS || desc->H_kv > 65535) return FC_ERR_UNSUPPORTED;
  if (desc->impl < 0 || desc->impl > 3) return FC_ERR_INVALID_ARG;
  if (!(desc->scale >= 0.f)) return FC_ERR_INVALID_ARG;
  if (desc->impl == 2 && dtype != FC_BF16) return FC_ERR_UNSUPPORTED;
  fc::AttnGeom& a = g.a;
  a.H_q = desc->H_q; a.H_kv = desc->H_kv; a.d = desc->d; a.W = desc->W;
  a.group = desc->H_q / desc->H_kv;
  a.scale = desc->scale != 0.f ? desc->scale : 1.f / sqrtf((float)desc->d);
  for (int c = 0; c <= a.W; ++c) {
    if (q_chunk_row_off[c] < 0 || (c > 0 && q_chunk_row_off[c] < q_chunk_row_off[c - 1])) return FC_ERR_INVALID_ARG;
    a.q_row_off[c] = q_chunk_row_off[c];
  }
  for (int c = 0; c < a.W; ++c) {
    if (kv_visible_len[c] < 0) return FC_ERR_INVALID_ARG;
    if (kv_visible_len[c] > INT32_MAX - 4096) return FC_ERR_UNSUPPORTED;  // key counters may run past the end by a step
    a.vis[c] = kv_visible_len[c];
  }
  g.n_cache = n_cache;
  g.f32 = dtype == FC_F32;
  g.n_vrows = (int64_t)(a.q_row_off[a.W] - a.q_row_off[0]) * a.group;
  if (g.n_vrows > INT32_MAX) return FC_ERR_UNSUPPORTED;
  return FC_OK;
}

enum Path { kSimt, kRows, kUnpacked };

// Rows of the clean region that some chunk sees.
int cache_rows(const fc::Kv4AttnGeom& g) {
  int n = 0;
  for (int c = 0; c < g.a.W; ++c) n = std::max(n, g.a.vis[c]);
  return std::min(n, g.n_cache);
}

// Workspace of the unpacked path: the tcgen05 kernel's own, K, V, and room for parts of the keys.
struct UnpackedPlan {
  fc::AttnSplit split;
  size_t k, v, plan, o, ml, bytes;  // offsets
  double us;                        // estimate of the whole path
};

UnpackedPlan plan_unpacked(const fc_ctx* ctx, const fc::Kv4AttnGeom& g) {
  const fc::AttnGeom& a = g.a;
  UnpackedPlan p;
  // grouped heads share their key tiles where whole groups fill a tile of 128 rows
  if (128 % a.group == 0 && (int64_t)a.q_row_off[a.W] * a.group <= INT32_MAX - 4096) p.split.pack = a.group;
  int64_t items = 0;
  int vis = 0;
  for (int c = 0; c < a.W; ++c) {
    items += ((int64_t)(a.q_row_off[c + 1] - a.q_row_off[c]) * p.split.pack + 255) / 256;  // rows of a work item
    vis = std::max(vis, a.vis[c]);
  }
  items *= a.H_q / p.split.pack;
  // Room for three parts a block: the cut items fill one round or two and some.
  const int tiles = (int)(((int64_t)vis + 127) / 128);
  if (tiles >= 6) p.split.slots = (int32_t)std::min<int64_t>(3 * ctx->sm_count, items * fc::kMaxParts);
  float last = 0.f;
  const int rest = (int)(items % ctx->sm_count);
  if (rest > 0) fc::split_parts(rest, ctx->sm_count, tiles, a.d, p.split.slots, &last);
  // 8 us for the launches of the path, 1.8 us a key tile, the unpacking at 6 TB/s
  p.us = 8 + 1.8 * ((double)(items / ctx->sm_count) * tiles + last) + 2.0 * a.H_kv * cache_rows(g) * a.d * 2.56 / 6e6;
  const size_t rows = (size_t)a.H_kv * cache_rows(g) * a.d * 2, parts = (size_t)p.split.slots * 256;
  p.k = fc::attention_tc_workspace_bytes();
  p.v = p.k + fc::align_up(rows, 256);
  p.plan = p.v + fc::align_up(rows, 256);
  p.o = p.plan + fc::align_up((4 + 4 * (size_t)ctx->sm_count) * sizeof(int32_t), 256);
  p.ml = p.o + parts * a.d * sizeof(float);
  p.bytes = p.ml + parts * sizeof(float2);
  return p;
}

// Strides that a tensor map takes: not 0 where there is more than one head, below 2^40 bytes.  The few-row kernel takes any.
bool maps_fit(const fc_attn_desc* d) {
  auto fits = [](int heads, int64_t hs, int64_t rs) { return rs < (1ll << 38) && (heads == 1 || (hs > 0 && hs < (1ll << 31))); };
  const bool window = d->kv_rows > 0;
  return fits(d->H_q, d->q_hs, d->q_rs) && (!window || (fits(d->H_kv, d->k_hs, d->k_rs) && fits(d->H_kv, d->v_hs, d->v_rs)));
}

// What a call does, with the workspace it takes and the split of the keys in g.
//
// Few rows read the packed keys in one pass but spend a tensor instruction on eight of them; many rows pay for unpacking once.  The
// line between the two moves with the heads and the keys, so that the estimates are compared.  Measured, row kernel against
// unpacking: 24 heads of 128 over 28000 keys, 64 rows 111 us and 140, 128 rows 223 and 142; over 1500 keys, 64 rows 17 and 20, 256 rows 44
// and 27; 16 heads on 4 over 28000 keys, 16 rows 26 and 37, 64 rows 86 and 45; 8 heads of 64 over 6000 keys, 128 rows 16 and
// 20, 256 rows 25 and 23.  Of 72 such sizes the estimates took the slower one by more than 8 % once (16 heads on 4, 32 rows, 28000
// keys: 43.4 against 38.5).
struct Plan {
  Path path;
  UnpackedPlan unpacked;  // kUnpacked
  size_t bytes;
};

Plan plan(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype, fc::Kv4AttnGeom& g) {
  Plan p = {};
  if (desc->impl == 1) {
    p.path = kSimt;
    p.bytes = fc::kv4_simt_workspace(ctx, g);
    return p;
  }
  if (desc->impl != 2) {
    p.path = kRows;
    p.bytes = fc::kv4_rows_workspace(ctx, g);
    if (desc->impl == 3 || dtype == FC_F32) return p;
  }
  p.unpacked = plan_unpacked(ctx, g);
  if (desc->impl == 2 || (p.unpacked.us < g.rows_us && maps_fit(desc))) {
    p.path = kUnpacked;
    p.bytes = p.unpacked.bytes;
  }
  return p;
}

}  // namespace

extern "C" size_t fc_chunk_attention_kv4_workspace_bytes(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype,
                                                         const int32_t* q_chunk_row_off, const int32_t* kv_visible_len,
                                                         int n_cache) {
  fc::Kv4AttnGeom g = {};
  if (!ctx || check_geometry(desc, dtype, q_chunk_row_off, kv_visible_len, n_cache, g) != FC_OK) return 0;
  return plan(ctx, desc, dtype, g).bytes;
}

extern "C" int fc_chunk_attention_kv4(fc_ctx* ctx, void* stream, const fc_attn_desc* desc, const void* Q,
                                      const fc_kv4_cache* cache, int n_cache, const void* K, const void* V, int dtype,
                                      const int32_t* q_chunk_row_off, const int32_t* kv_visible_len,
                                      const int32_t* seg_logical_off, const int32_t* seg_phys_off, int n_seg,
                                      const int32_t* active_ids, const int32_t* n_active, void* O, float* lse, int64_t lse_hs,
                                      uint32_t* status, void* ws, size_t ws_bytes) {
  if (!ctx || !desc || n_seg < 0) return FC_ERR_INVALID_ARG;
  fc::Kv4AttnGeom g = {};
  int rc = check_geometry(desc, dtype, q_chunk_row_off, kv_visible_len, n_cache, g);
  if (rc != FC_OK) return rc;
  if (g.n_vrows == 0) return FC_OK;
  if (!Q || !O || !active_ids || !n_active) return FC_ERR_INVALID_ARG;
  fc::AttnGeom& a = g.a;
  const int es = fc::elem_size(dtype);
  const int64_t strides[8] = {desc->q_hs, desc->q_rs, desc->o_hs, desc->o_rs, desc->k_hs, desc->k_rs, desc->v_hs, desc->v_rs};
  for (int i = 0; i < (n_seg > 0 ? 8 : 4); ++i) {
    if (strides[i] < 0 || (strides[i] * es) % 16) return FC_ERR_MISALIGNED;
    if (i % 2 && strides[i] < desc->d) return FC_ERR_INVALID_ARG;
  }
  if (desc->H_q > 1 && desc->o_hs < desc->d) return FC_ERR_INVALID_ARG;  // heads of O would overlap
  if (!fc::aligned16(Q) || !fc::aligned16(O)) return FC_ERR_MISALIGNED;
  if (n_cache > 0 && (rc = fc::kv4_check(cache, desc->d, n_cache)) != FC_OK) return rc;
  if (n_seg > FC_MAX_SEGMENTS - 1) return FC_ERR_UNSUPPORTED;
  int64_t window = 0;
  if (n_seg > 0) {
    if (!K || !V || !seg_logical_off || !seg_phys_off || desc->kv_rows <= 0) return FC_ERR_INVALID_ARG;
    if (!fc::aligned16(K) || !fc::aligned16(V)) return FC_ERR_MISALIGNED;
    for (int s = 0; s <= n_seg; ++s) {
      if (s == 0 ? seg_logical_off[0] != 0 : seg_logical_off[s] < seg_logical_off[s - 1]) return FC_ERR_INVALID_ARG;
      a.seg_log[s] = seg_logical_off[s];
    }
    for (int s = 0; s < n_seg; ++s) {
      const int64_t len = seg_logical_off[s + 1] - seg_logical_off[s];
      if (seg_phys_off[s] < 0 || seg_phys_off[s] + len > desc->kv_rows) return FC_ERR_INVALID_ARG;
      a.seg_phys[s] = seg_phys_off[s];
    }
    window = seg_logical_off[n_seg];
  }
  if (n_cache + window > INT32_MAX - 4096) return FC_ERR_UNSUPPORTED;  // logical offsets of the two stores together are 32-bit
  for (int c = 0; c < a.W; ++c)
    if (a.vis[c] > n_cache + window) return FC_ERR_INVALID_ARG;
  if (lse && lse_hs <= 0) return FC_ERR_INVALID_ARG;
  a.n_seg = n_seg;
  a.q_hs = desc->q_hs; a.q_rs = desc->q_rs; a.k_hs = desc->k_hs; a.k_rs = desc->k_rs;
  a.v_hs = desc->v_hs; a.v_rs = desc->v_rs; a.o_hs = desc->o_hs; a.o_rs = desc->o_rs;
  a.kv_rows = desc->kv_rows; a.lse_hs = lse_hs;
  a.active_ids = active_ids; a.n_active = n_active; a.lse = lse; a.status = status;
  if (n_cache > 0) g.cache = fc::kv4_view(*cache);

  if (desc->impl == 2 && !maps_fit(desc)) return FC_ERR_UNSUPPORTED;
  Plan p = plan(ctx, desc, dtype, g);
  const size_t need = p.bytes;
  if (need > 0) {
    if (!ws || ws_bytes < need) return FC_ERR_WORKSPACE;
    if (!fc::aligned16(ws)) return FC_ERR_MISALIGNED;
    if (p.path != kUnpacked) {
      const int64_t parts = a.H_kv * g.n_vrows * g.n_splits;
      g.part_o = (float*)ws;
      g.part_ml = (float2*)((char*)ws + fc::align_up(parts * a.d * sizeof(float), 256));
    }
  }
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
  if (p.path == kSimt) return fc::kv4_simt(st, g, Q, K, V, dtype, O);
  if (p.path == kRows) return fc::kv4_rows(st, g, Q, K, V, O);
  UnpackedPlan& u = p.unpacked;
  const int n0 = cache_rows(g);
  char* base = (char*)ws;
  struct Unpack {
    cudaStream_t st;
    const fc::Kv4AttnGeom* g;
    int n0;
    void *k, *v;
    uint32_t* counter;
  } unpack = {st, &g, n0, base + u.k, base + u.v, (uint32_t*)ws};
  auto before = [](void* arg) -> int {
    const Unpack& x = *(const Unpack*)arg;
    const int64_t hs = (int64_t)x.n0 * x.g->a.d;
    return fc::kv4_unpack_launch(x.st, x.g->cache, x.g->a.H_kv, x.g->a.d, 0, x.n0, x.k, x.v, FC_BF16, hs, x.g->a.d, hs, x.g->a.d, x.counter);
  };
  u.split.follows = n0 > 0;
  u.split.o = (float*)(base + u.o);
  u.split.ml = (float2*)(base + u.ml);
  u.split.plan = (int32_t*)(base + u.plan);
  return fc::attention_tc_two(ctx, st, a, Q, base + u.k, base + u.v, n0, K, V, u.split, O, ws, ws_bytes, before, &unpack);
}
