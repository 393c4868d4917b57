// What the kernels of fc_chunk_attention_kv4 share.
#pragma once

#include "fc_attention.cuh"
#include "fc_kv4.cuh"

namespace fc {

// Query rows are taken per key head: the `group` query heads that share it are rows of the same tile, so that a key is
// fetched and unpacked once for all of them.  Virtual row v of chunk c and key head hk is query head hk * group + v % group,
// row q_row_off[c] + v / group.
constexpr int kKv4MaxSplits = 512;

struct Kv4AttnGeom {
  AttnGeom a;        // segments and store fields describe the window; vis counts cache and window together
  Kv4View cache;
  int32_t n_cache;
  bool f32;             // type of Q, the window and O
  int32_t n_splits;  // parts the keys are cut into, at most kKv4MaxSplits
  int64_t part_keys;    // keys per part (few-row kernel: on its axis of costs)
  int64_t n_cache_ceil; // few-row kernel: where the window starts on that axis
  int32_t row_tiles;    // few-row kernel: rows of a tile / 8
  double rows_us;       // few-row kernel: estimate of the whole call
  int64_t n_vrows;   // virtual rows per key head, all chunks
  float* part_o;     // [H_kv, n_vrows, n_splits, d] unnormalised outputs, used if n_splits > 1
  float2* part_ml;   // [H_kv, n_vrows, n_splits] running maximum (log2 units for the tensor-core kernel) and sum
};

// Whether chunk c is on the device-side list (at most 64 entries); called by whole warps.
__device__ __forceinline__ bool chunk_active(const AttnGeom& a, int c) {
  static_assert(FC_MAX_CHUNKS <= 64, "two entries a lane");
  const int lane = threadIdx.x % 32, n = min(max(*a.n_active, 0), a.W);
  const bool mine = (lane < n && a.active_ids[lane] == c) || (lane + 32 < n && a.active_ids[lane + 32] == c);
  return __any_sync(0xffffffffu, mine);
}

// An id outside [0, W) is reported and otherwise ignored.
__device__ __forceinline__ void report_bad_ids(const AttnGeom& a) {
  const int n = min(max(*a.n_active, 0), a.W);
  for (int i = 0; i < n; ++i)
    if ((a.active_ids[i] < 0 || a.active_ids[i] >= a.W) && a.status) atomicOr(a.status, (uint32_t)FC_DEV_BAD_INDEX);
}

// Physical row of window token j, or -1 (an offset past the table's end cannot occur: the host checks visible lengths).
__device__ __forceinline__ int64_t window_row(const AttnGeom& a, int j) {
  for (int s = 0; s < a.n_seg; ++s)
    if (j < a.seg_log[s + 1]) return (int64_t)a.seg_phys[s] + (j - a.seg_log[s]);
  return -1;
}

// Chunk and first virtual row of tile t where each chunk's rows are cut into tiles of kRows; chunk -1 past the end.
template <int kRows>
__device__ __forceinline__ int tile_chunk(const AttnGeom& a, int t, int& v0) {
  for (int c = 0; c < a.W; ++c) {
    const int tiles = (int)(((int64_t)(a.q_row_off[c + 1] - a.q_row_off[c]) * a.group + kRows - 1) / kRows);
    if (t < tiles) {
      v0 = t * kRows;
      return c;
    }
    t -= tiles;
  }
  return -1;
}

inline int64_t tile_count(const AttnGeom& a, int rows_per_tile) {
  int64_t n = 0;
  for (int c = 0; c < a.W; ++c)
    n += ((int64_t)(a.q_row_off[c + 1] - a.q_row_off[c]) * a.group + rows_per_tile - 1) / rows_per_tile;
  return n;
}

size_t kv4_simt_workspace(const fc_ctx* ctx, Kv4AttnGeom& g);  // also sets the split
int kv4_simt(cudaStream_t st, const Kv4AttnGeom& g, const void* Q, const void* K, const void* V, int dtype, void* O);
// few rows, and fp32: tensor cores fed from registers
size_t kv4_rows_workspace(const fc_ctx* ctx, Kv4AttnGeom& g);
int kv4_rows(cudaStream_t st, const Kv4AttnGeom& g, const void* Q, const void* K, const void* V, void* O);
// Joins the parts of every active row and writes O and lse.
int kv4_combine(cudaStream_t st, const Kv4AttnGeom& g, int dtype, void* O, bool log2_units);

}  // namespace fc
