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

// attention_tc_two only: how the work is cut up.
//
// Work items (a chunk's 256 rows of one head or group of heads) are handed out to one block per SM.  As many as fill whole rounds of
// the blocks are worked through in one piece; the keys of the others, the shortest, are cut into parts, so that the last
// round is full too.  How many there are is known on the device only (the active list is there), so the kernel decides and leaves
// word for the one that joins the parts.
struct AttnSplit {
  int32_t pack = 1;     // query heads taken as rows of one tile: 1, or the group where it divides a tile's 128 rows
  bool follows = false; // the stream's last kernel writes K0 / V0, clears the counter and lets this one start early
  int32_t slots = 0;    // room for parts; 0: every item in one piece
  float* o = nullptr;   // [slots, 256, d]: sums not divided by their weights
  float2* ml = nullptr; // [slots, 256]: reference (log2 units) and sum of the weights
  int32_t* plan = nullptr; // [4 + 4 * blocks]: cut items, parts of each, -, -; then of each: chunk, head, first row, -
};
constexpr int kMaxParts = 32;

// What each chunk sees where that is more than a prefix: rows [lo[i][c], hi[i][c]) of the first store (i = 0, 1), and tokens of
// the segment table (i = 2, 3), in this order.
struct AttnSpans {
  int32_t lo[4][FC_MAX_CHUNKS], hi[4][FC_MAX_CHUNKS];
};

// Parts for each of `rest` items of `tiles` key tiles on `blocks` blocks.  The unit is the time of a key tile, 1.8 us; the
// joining kernel costs three of them, and the parts' bytes go at 4 TB/s.
__host__ __device__ inline int split_parts(int rest, int blocks, int tiles, int d, int slots, float* cost) {
  const float part = (float)rest * 256 * d * 8 / 7.2e6f;
  int best_n = 1;
  float best = (float)tiles * ((rest + blocks - 1) / blocks);
  for (int n = 2; n <= kMaxParts && rest * n <= slots && n * 3 <= tiles; ++n) {
    const float c = (float)((rest * n + blocks - 1) / blocks) * ((tiles + n - 1) / n) + 3.f + n * part;
    if (c < best) best = c, best_n = n;
  }
  if (cost) *cost = best;
  return best_n;
}

int attention_simt(cudaStream_t st, const AttnGeom& g, const void* Q, const void* K, const void* V,
                   int dtype, void* O);
// bf16 only: builds the tensor maps and launches the warp-specialised tcgen05 kernel.
int attention_tc(fc_ctx* ctx, cudaStream_t st, const AttnGeom& g, const void* Q, const void* K,
                 const void* V, void* O, void* ws, size_t ws_bytes);
size_t attention_tc_workspace_bytes();
// The same over two stores: logical tokens [0, n0) are the rows of K0 / V0 (dense [H_kv, n0, d]), the others are found
// in K / V through the segment table, whose offsets count from n0.  With `spans` these say what each chunk sees, g.vis counts the keys of
// a chunk, and the segment table's offsets count from 0.  `before` is called once nothing but launches is left that
// could fail; it launches the kernel that writes K0 / V0.
int attention_tc_two(fc_ctx* ctx, cudaStream_t st, const AttnGeom& g, const void* Q, const void* K0, const void* V0, int n0,
                     const void* K, const void* V, const AttnSplit& split, void* O, void* ws, size_t ws_bytes,
                     int (*before)(void*), void* arg, const AttnSpans* spans = nullptr);
// warp-specialised kernel; tensor maps as built by attention_tc (tk0, tv0: those of the second store, or NULL),
// `counter` = 4 bytes of workspace
int attention_ws_launch(fc_ctx* ctx, cudaStream_t st, const AttnGeom& g, const CUtensorMap& tq,
                        const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap* tk0, const CUtensorMap* tv0,
                        const AttnSplit& split, const AttnSpans* spans, void* O, uint32_t* counter);
bool attention_tc_supported(const AttnGeom& g, int dtype);
// Tensor map of a [heads, rows, d] bf16 tensor: box = 64 elements (128 bytes) x `box_rows` rows x 1 head, 128-byte
// swizzle; rows past `rows` read as zero.
int make_tmap(fc_ctx* ctx, CUtensorMap* map, const void* base, int d, int64_t rows, int heads, int64_t row_stride,
              int64_t head_stride, int box_rows = 128);

}  // namespace fc
