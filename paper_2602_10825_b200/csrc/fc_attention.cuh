// Geometry shared by the two attention kernels of libfc (CUDA-core and tcgen05).
#pragma once

#include <cuda.h>

#include "fc_common.cuh"

namespace fc {

struct AttnGeom {
  int32_t H_q, H_kv, d, W, group, n_seg;
  int32_t n_seg0;  // leading segments that lie in a second store (attention_tc_two), else 0
  int64_t q_hs, q_rs, k_hs, k_rs, v_hs, v_rs, o_hs, o_rs, kv_rows, lse_hs, tok_hs;
  float scale;
  int32_t q_row_off[FC_MAX_CHUNKS + 1];
  int32_t vis[FC_MAX_CHUNKS];
  int32_t seg_log[FC_MAX_SEGMENTS + 1];
  int32_t seg_phys[FC_MAX_SEGMENTS];
  const int32_t* tok_index;
  const int32_t* active_ids;
  const int32_t* n_active;
  float* lse;
  uint32_t* status;
};

// attention_tc_two only: how the work is cut up.  Parts of the keys have their results joined by another kernel (n_splits 1: no
// parts).
struct AttnSplit {
  int32_t pack = 1;     // query heads taken as rows of one tile: 1, or the group where it divides a tile's 128 rows
  bool follows = false; // the stream's last kernel writes K0 / V0, clears the counter and lets this one start early
  int32_t n_splits = 1, part_keys = 0;  // part p: logical keys [p part_keys, (p + 1) part_keys), the last one to the end
  int64_t n_vrows = 0;
  float* o = nullptr;   // [H_kv, n_vrows, n_splits, d]: sums not divided by their weights
  float2* ml = nullptr; // [H_kv, n_vrows, n_splits]: reference (log2 units) and sum of the weights
};

int attention_simt(cudaStream_t st, const AttnGeom& g, const void* Q, const void* K, const void* V,
                   int dtype, void* O);
// bf16 only: builds the tensor maps and launches the warp-specialised tcgen05 kernel.
int attention_tc(fc_ctx* ctx, cudaStream_t st, const AttnGeom& g, const void* Q, const void* K,
                 const void* V, void* O, void* ws, size_t ws_bytes);
size_t attention_tc_workspace_bytes();
// The same over two stores: logical tokens [0, n0) are the rows of K0 / V0 (dense [H_kv, n0, d]), the others are found
// in K / V through the segment table, whose offsets count from n0.  `before` is called once nothing but launches is left that
// could fail; it launches the kernel that writes K0 / V0.
int attention_tc_two(fc_ctx* ctx, cudaStream_t st, const AttnGeom& g, const void* Q, const void* K0, const void* V0, int n0,
                     const void* K, const void* V, const AttnSplit& split, void* O, void* ws, size_t ws_bytes,
                     int (*before)(void*), void* arg);
// warp-specialised kernel; tensor maps as built by attention_tc (tk0, tv0: those of the second store, or NULL),
// `counter` = 4 bytes of workspace
int attention_ws_launch(fc_ctx* ctx, cudaStream_t st, const AttnGeom& g, const CUtensorMap& tq,
                        const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap* tk0, const CUtensorMap* tv0,
                        const AttnSplit& split, void* O, uint32_t* counter);
bool attention_tc_supported(const AttnGeom& g, int dtype);
// Tensor map of a [heads, rows, d] bf16 tensor: box = 64 elements (128 bytes) x `box_rows` rows x 1 head, 128-byte
// swizzle; rows past `rows` read as zero.
int make_tmap(fc_ctx* ctx, CUtensorMap* map, const void* base, int d, int64_t rows, int heads, int64_t row_stride,
              int64_t head_stride, int box_rows = 128);

}  // namespace fc
