// What the two kernels of fc_chunk_attention_kv8 and fc_chunk_attention_span share.
#pragma once

#include "fc_attention.cuh"
#include "fc_kv8.cuh"

namespace fc {

// Query rows are taken per key head, as in fc_attention_kv4.cuh: virtual row v of chunk c and key head hk is query head
// hk * group + v % group, row q_row_off[c] + v / group.
struct SpanGeom {
  int32_t H_q, H_kv, d, W, group, n_seg;
  int64_t q_hs, q_rs, k_hs, k_rs, v_hs, v_rs, o_hs, o_rs, kv_rows, lse_hs;
  float scale;
  bool f32;                       // type of Q, the plain tokens and O
  int32_t q_row_off[FC_MAX_CHUNKS + 1];
  // What chunk c sees: tokens [lo[i][c], hi[i][c]) of its pages (i = 0: first tokens, 1: the sliding window), and of the plain
  // tokens in the order of the segment table (i = 2, 3).  Where there is nothing, lo = hi.
  int32_t lo[4][FC_MAX_CHUNKS], hi[4][FC_MAX_CHUNKS];
  int32_t seg_log[FC_MAX_SEGMENTS + 1], seg_phys[FC_MAX_SEGMENTS];
  Kv8View pool;
  const int32_t* table;
  int64_t table_cs;
  const int32_t *active_ids, *n_active;
  float* lse;
  uint32_t* status;
  // Kernel for few rows: the keys of chunk c are cut into parts[c] parts of part_units[c] units of cost; blocks are numbered
  // chunk by chunk, tile by tile, part by part.
  int32_t row_tiles;                 // rows of a tile / 8
  int32_t cluster;                   // the parts of a tile are as many, one thread block cluster, and join themselves; 0: a second kernel joins
  int32_t parts[FC_MAX_CHUNKS], part_units[FC_MAX_CHUNKS], block_end[FC_MAX_CHUNKS];
  float* part_o;                     // [H_kv, blocks, rows of a tile, d] sums not divided by their weights
  float2* part_ml;                   // [H_kv, blocks, rows of a tile]: reference (log2 units) and sum of the weights
  double rows_us;                    // estimate of the whole call
};

// Whether chunk c is on the device-side list (at most 64 entries); called by whole warps.
__device__ __forceinline__ bool span_chunk_active(const SpanGeom& g, int c) {
  static_assert(FC_MAX_CHUNKS <= 64, "two entries a lane");
  const int lane = threadIdx.x % 32, n = min(max(*g.n_active, 0), g.W);
  const bool mine = (lane < n && g.active_ids[lane] == c) || (lane + 32 < n && g.active_ids[lane + 32] == c);
  return __any_sync(0xffffffffu, mine);
}

inline int64_t span_rows(const SpanGeom& g, int c) { return (int64_t)(g.q_row_off[c + 1] - g.q_row_off[c]) * g.group; }

// Few rows, and fp32: the plan (split and workspace), and the launches.
size_t span_rows_workspace(const fc_ctx* ctx, SpanGeom& g);
int span_rows_launch(fc_ctx* ctx, cudaStream_t st, const SpanGeom& g, const void* Q, const void* K, const void* V, void* O);

}  // namespace fc
