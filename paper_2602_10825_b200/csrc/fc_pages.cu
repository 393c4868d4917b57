// fc_pages_take, _drop, _fork and _compact: who holds which page of a pool, and the copying that follows.
//
// The counts are found and changed by one block, in a fixed order: the free pages are walked in tiles of 4096, each thread four
// neighbouring counts, and a scan over the block gives every free page its rank.  That is latency (a tile takes
// about a microsecond), not bandwidth; it ends with the last page that is wanted.  fork and compact leave a list of copies in the workspace, and
// a second kernel, started early, moves the blocks of the pages: bound by HBM, 2 (page d + 4) bytes of K and of V a head.
#include <algorithm>
#include <climits>

#include "fc_kv8.cuh"

namespace {

constexpr int kThreads = 1024, kTile = 4 * kThreads;
constexpr int kCopyThreads = 256;

// Ranges of table entries, one a sequence.
struct Ranges {
  int32_t W;
  int32_t first[FC_MAX_CHUNKS], end[FC_MAX_CHUNKS];  // first entry; running count of entries
  int64_t table_cs;
};
__device__ __forceinline__ int32_t* entry_of(int32_t* table, const Ranges& r, int k) {
  int c = 0;
  while (k >= r.end[c]) ++c;
  return table + c * r.table_cs + r.first[c] + (k - (c > 0 ? r.end[c - 1] : 0));
}

// Exclusive sums over the block of x (two counts of 16 bits); `total` is the sum of all.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t& total) {
  __shared__ uint32_t warp_s[2][kThreads / 32];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  uint32_t sum = x;
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, sum, k);
    if (lane >= k) sum += y;
  }
  __syncthreads();
  if (lane == 31) warp_s[0][warp] = sum;
  __syncthreads();
  if (warp == 0) {
    const uint32_t w = warp_s[0][lane];
    uint32_t s = w;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, s, k);
      if (lane >= k) s += y;
    }
    warp_s[1][lane] = s;
  }
  __syncthreads();
  total = warp_s[1][31];
  return sum - x + (warp > 0 ? warp_s[1][warp - 1] : 0);
}

__device__ __forceinline__ int4 counts_at(const int32_t* ref, int p, int n_pages, int behind) {
  if (p + 4 <= n_pages) return *reinterpret_cast<const int4*>(ref + p);
  return make_int4(p < n_pages ? ref[p] : behind, p + 1 < n_pages ? ref[p + 1] : behind, p + 2 < n_pages ? ref[p + 2] : behind, behind);
}

// Calls give(rank, page) for the `wanted` free pages of the lowest numbers; returns how many there were.  The whole block calls it.
template <typename Give>
__device__ __forceinline__ int lowest_free(const int32_t* ref, int n_pages, int wanted, Give give) {
  int found = 0;
  for (int p0 = 0; p0 < n_pages && found < wanted; p0 += kTile) {
    const int p = p0 + 4 * (int)threadIdx.x;
    const int4 x = counts_at(ref, p, n_pages, 1);
    const int free4[4] = {x.x == 0, x.y == 0, x.z == 0, x.w == 0};
    uint32_t total;
    int rank = found + (int)block_scan(free4[0] + free4[1] + free4[2] + free4[3], total);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (free4[i]) {
        if (rank < wanted) give(rank, p + i);
        ++rank;
      }
    found += (int)total;
  }
  return min(found, wanted);
}

__global__ void __launch_bounds__(kThreads)
pages_take_kernel(int32_t* __restrict__ ref, int n_pages, int32_t* __restrict__ table, const __grid_constant__ Ranges r,
                  uint32_t* __restrict__ status) {
  const int wanted = r.end[r.W - 1];
  const int found = lowest_free(ref, n_pages, wanted, [&](int rank, int p) {
    *entry_of(table, r, rank) = p;
    ref[p] = 1;  // the block is past this tile's counts
  });
  for (int k = found + (int)threadIdx.x; k < wanted; k += kThreads) *entry_of(table, r, k) = -1;
  if (found < wanted && threadIdx.x == 0 && status) atomicOr(status, (uint32_t)FC_DEV_NO_PAGES);
}

__global__ void __launch_bounds__(256)
pages_drop_kernel(int32_t* __restrict__ ref, int n_pages, int32_t* __restrict__ table, const __grid_constant__ Ranges r,
                  uint32_t* __restrict__ status) {
  const int k = blockIdx.x * 256 + threadIdx.x;
  if (k >= r.end[r.W - 1]) return;
  int32_t* entry = entry_of(table, r, k);
  const int p = *entry;
  *entry = -1;
  if (p == -1) return;
  bool bad = p < 0 || p >= n_pages;
  if (!bad && atomicSub(ref + p, 1) <= 0) {  // nobody held it
    atomicAdd(ref + p, 1);
    bad = true;
  }
  if (bad && status) atomicOr(status, (uint32_t)FC_DEV_BAD_INDEX);
}

// What the copying kernel finds in the workspace: the number of copies, the number of used pages, then pairs (from, to; from -1: none),
// and, for compact, the new place of each page.
struct Copies {
  int32_t* n;     // [2]
  int2* pair;
  int32_t* place; // [n_pages]
};
Copies copies_at(void* ws, int n_pages) {
  const size_t pairs = (size_t)std::max(n_pages / 2 + 1, (int)FC_MAX_CHUNKS);
  char* p = (char*)ws;
  return {(int32_t*)p, (int2*)(p + 16), (int32_t*)(p + 16 + pairs * sizeof(int2))};
}
size_t copies_bytes(int n_pages) {
  const size_t pairs = (size_t)std::max(n_pages / 2 + 1, (int)FC_MAX_CHUNKS);
  return fc::align_up(16 + pairs * sizeof(int2) + (size_t)n_pages * sizeof(int32_t), 256);
}

struct Forks {
  int32_t n, page;
  int32_t src[FC_MAX_CHUNKS], dst[FC_MAX_CHUNKS], tokens[FC_MAX_CHUNKS];
  int64_t table_cs;
};

__global__ void __launch_bounds__(kThreads)
pages_fork_kernel(int32_t* __restrict__ ref, int n_pages, int32_t* __restrict__ table, const __grid_constant__ Forks f, Copies copies,
                  uint32_t* __restrict__ status) {
  __shared__ int32_t look_s[FC_MAX_CHUNKS], part_s[FC_MAX_CHUNKS], from_s[FC_MAX_CHUNKS], n_part;  // forks that copy a page, and from which
  constexpr int32_t kNoCopy = -2;
  fc::pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  bool bad = false;
  // A page that is free is not counted, so that every fork finds it free.
  constexpr int kAtOnce = 4;
  for (int i = warp; i < f.n; i += kThreads / 32) {
    const int32_t* src = table + f.src[i] * f.table_cs;
    int32_t* dst = table + f.dst[i] * f.table_cs;
    const int full = f.tokens[i] / f.page;
    for (int e0 = lane; e0 < full; e0 += 32 * kAtOnce) {
      int p[kAtOnce];
      bool named[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) p[k] = e0 + 32 * k < full ? src[e0 + 32 * k] : -1;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) named[k] = p[k] >= 0 && p[k] < n_pages && __ldcg(ref + p[k]) != 0;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        if (e0 + 32 * k < full) dst[e0 + 32 * k] = named[k] ? p[k] : -1;
        if (named[k]) atomicAdd(ref + p[k], 1);
        bad |= !named[k] && p[k] != -1;
      }
    }
  }
  if (tid < f.n) {  // the page that fork `tid` fills in part
    int from = kNoCopy;
    if (f.tokens[tid] % f.page != 0) {
      const int e = f.tokens[tid] / f.page, p = table[f.src[tid] * f.table_cs + e];
      if (p >= 0 && p < n_pages) {
        from = p;
        if (__ldcg(ref + p) == 0) {  // a page of its own all the same, into which nothing is copied
          bad = true;
          from = -1;
        }
      } else {
        table[f.dst[tid] * f.table_cs + e] = -1;
        bad |= p != -1;
      }
    }
    look_s[tid] = from;
  }
  __threadfence_block();
  __syncthreads();
  if (tid == 0) {
    int n = 0;
    for (int i = 0; i < f.n; ++i) {
      if (look_s[i] == kNoCopy) continue;
      part_s[n] = i;
      from_s[n++] = look_s[i];
    }
    n_part = n;
  }
  __syncthreads();
  const int wanted = n_part;
  const int found = lowest_free(ref, n_pages, wanted, [&](int rank, int p) {
    const int i = part_s[rank];
    table[f.dst[i] * f.table_cs + f.tokens[i] / f.page] = p;
    ref[p] = 1;
    copies.pair[rank] = make_int2(from_s[rank], p);
  });
  for (int k = found + tid; k < wanted; k += kThreads) table[f.dst[part_s[k]] * f.table_cs + f.tokens[part_s[k]] / f.page] = -1;
  if (tid == 0) copies.n[0] = found;
  if (status) {
    if (bad) atomicOr(status, (uint32_t)FC_DEV_BAD_INDEX);
    if (found < wanted && tid == 0) atomicOr(status, (uint32_t)FC_DEV_NO_PAGES);
  }
}

__global__ void __launch_bounds__(kThreads)
pages_compact_kernel(int32_t* __restrict__ ref, int n_pages, Copies copies, int32_t* __restrict__ n_used) {
  fc::pdl_launch_dependents();
  const int tid = threadIdx.x;
  uint32_t total;
  int used = 0;
  for (int p0 = 0; p0 < n_pages; p0 += kTile) {
    const int4 x = counts_at(ref, p0 + 4 * tid, n_pages, 0);
    block_scan((x.x != 0) + (x.y != 0) + (x.z != 0) + (x.w != 0), total);
    used += (int)total;
  }
  // The free pages below `used`, and the used ones from there on: as many of one kind as of the other.
  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < n_pages; p0 += kTile) {
    const int p = p0 + 4 * tid;
    const int4 x = counts_at(ref, p, n_pages, 0);
    const int c[4] = {x.x, x.y, x.z, x.w};
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mine += p + i < used ? (c[i] == 0) : (uint32_t)(c[i] != 0) << 16;
    const uint32_t before = block_scan(mine, total);
    int hole = holes + (int)(before & 0xffffu), mover = movers + (int)(before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p + i >= n_pages) break;
      if (p + i < used) {
        if (c[i] == 0) copies.pair[hole++].y = p + i;
      } else {
        if (c[i] != 0) copies.pair[mover++].x = p + i;
        else copies.place[p + i] = -1;
      }
    }
    holes += (int)(total & 0xffffu);
    movers += (int)(total >> 16);
  }
  __syncthreads();
  for (int k = tid; k < movers; k += kThreads) {
    const int2 m = copies.pair[k];
    ref[m.y] = ref[m.x];
    ref[m.x] = 0;
    copies.place[m.x] = m.y;
  }
  if (tid == 0) {
    copies.n[0] = movers;
    copies.n[1] = used;
    if (n_used) *n_used = used;
  }
}

struct CopyGeom {
  fc::Kv8View pool;
  Copies copies;
  int32_t H, block_bytes;
  // compact: the table whose entries are rewritten (n_seq 0: none)
  int32_t* table;
  int64_t table_cs;
  int32_t n_seq, entries;
};

// A unit of work is a block of a page that moves (one head's codes of K or V, and their scale).
__global__ void __launch_bounds__(kCopyThreads)
pages_copy_kernel(const __grid_constant__ CopyGeom g, uint32_t* __restrict__ status) {
  fc::pdl_wait();
  const int tid = threadIdx.x;
  const int64_t units = (int64_t)g.copies.n[0] * g.H * 2;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const bool is_v = u & 1;
    const int64_t rest = u >> 1;
    const int h = (int)(rest % g.H);
    const int2 m = g.copies.pair[rest / g.H];
    if (m.x < 0) continue;  // nothing to copy
    if (!fc::bounds_ok((uint32_t)m.x < (uint32_t)g.pool.n_pages && (uint32_t)m.y < (uint32_t)g.pool.n_pages, status)) continue;
    uint8_t* base = (is_v ? g.pool.v_codes : g.pool.k_codes) + h * g.pool.code_hs;
    const uint8_t* from = base + m.x * g.pool.code_ps;
    uint8_t* to = base + m.y * g.pool.code_ps;
    constexpr int kAtOnce = 2;
    for (int i0 = 16 * tid; i0 < g.block_bytes; i0 += 16 * kCopyThreads * kAtOnce) {
      uint4 x[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
        if (i0 + k * 16 * kCopyThreads < g.block_bytes) x[k] = fc::ld_stream16(from + i0 + k * 16 * kCopyThreads);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
        if (i0 + k * 16 * kCopyThreads < g.block_bytes) fc::st_stream16(to + i0 + k * 16 * kCopyThreads, x[k]);
    }
    if (tid == 0) {
      float* scales = (is_v ? g.pool.v_scales : g.pool.k_scales) + h * g.pool.scale_hs;
      scales[m.y * g.pool.scale_ps] = scales[m.x * g.pool.scale_ps];
    }
  }
  if (g.n_seq > 0) {
    const int used = g.copies.n[1];
    const int64_t n = (int64_t)g.n_seq * g.entries;
    for (int64_t k = (int64_t)blockIdx.x * kCopyThreads + tid; k < n; k += (int64_t)gridDim.x * kCopyThreads) {
      int32_t* entry = g.table + k / g.entries * g.table_cs + k % g.entries;
      const int p = *entry;
      if (p == -1 || (p >= 0 && p < used)) continue;  // no page, or one that stays
      const int to = p < 0 || p >= g.pool.n_pages ? -1 : g.copies.place[p];
      if (to >= 0) *entry = to;
      else if (status) atomicOr(status, (uint32_t)FC_DEV_BAD_INDEX);
    }
  }
}

int ranges_of(const int32_t* ref, int n_pages, const int32_t* table, int64_t table_cs, int W, const int32_t* first, const int32_t* last,
              Ranges& r) {
  if (!first || !last || n_pages <= 0 || W <= 0 || table_cs < 0) return FC_ERR_INVALID_ARG;
  if (W > FC_MAX_CHUNKS || n_pages > fc::kMaxPages) return FC_ERR_UNSUPPORTED;
  int64_t n = 0;
  for (int c = 0; c < W; ++c) {
    if (first[c] < 0 || last[c] < first[c]) return FC_ERR_INVALID_ARG;
    if (W > 1 && last[c] > table_cs) return FC_ERR_INVALID_ARG;
    n += last[c] - first[c];
    if (n > INT32_MAX - 4096) return FC_ERR_UNSUPPORTED;
    r.first[c] = first[c];
    r.end[c] = (int32_t)n;
  }
  r.W = W;
  r.table_cs = table_cs;
  if (n == 0) return FC_OK;
  if (!ref || !table) return FC_ERR_INVALID_ARG;
  return fc::aligned16(ref) ? FC_OK : FC_ERR_MISALIGNED;
}

int check_pool(const fc_kv8_pool* pool, int H, int d) {
  if (H <= 0) return FC_ERR_INVALID_ARG;
  if (H > 65535 || (d != 64 && d != 128)) return FC_ERR_UNSUPPORTED;
  return fc::kv8_check(pool, H, d);
}

int launch_copies(fc_ctx* ctx, cudaStream_t st, const CopyGeom& g, int64_t most, uint32_t* status) {
  const int64_t units = std::max<int64_t>(most * g.H * 2, g.n_seq > 0 ? 1 : 0);
  const int grid = (int)std::min<int64_t>(units, 8ll * ctx->sm_count);
  if (grid == 0) return FC_OK;
  FC_CUDA_CHECK(fc::launch_pdl(pages_copy_kernel, dim3(grid), dim3(kCopyThreads), 0, st, g, status));
  FC_LAUNCH_CHECK("pages_copy_kernel");
  return FC_OK;
}

}  // namespace

extern "C" int fc_pages_take(fc_ctx* ctx, void* stream, int32_t* ref, int n_pages, int32_t* table, int64_t table_cs, int W,
                             const int32_t* first, const int32_t* last, uint32_t* status) {
  if (!ctx) return FC_ERR_INVALID_ARG;
  Ranges r = {};
  const int rc = ranges_of(ref, n_pages, table, table_cs, W, first, last, r);
  if (rc != FC_OK || r.end[W - 1] == 0) return rc;
  FC_DEVICE_GUARD(ctx);
  pages_take_kernel<<<1, kThreads, 0, (cudaStream_t)stream>>>(ref, n_pages, table, r, status);
  FC_LAUNCH_CHECK("pages_take_kernel");
  return FC_OK;
}

extern "C" int fc_pages_drop(fc_ctx* ctx, void* stream, int32_t* ref, int n_pages, int32_t* table, int64_t table_cs, int W,
                             const int32_t* first, const int32_t* last, uint32_t* status) {
  if (!ctx) return FC_ERR_INVALID_ARG;
  Ranges r = {};
  const int rc = ranges_of(ref, n_pages, table, table_cs, W, first, last, r);
  if (rc != FC_OK || r.end[W - 1] == 0) return rc;
  FC_DEVICE_GUARD(ctx);
  pages_drop_kernel<<<(r.end[W - 1] + 255) / 256, 256, 0, (cudaStream_t)stream>>>(ref, n_pages, table, r, status);
  FC_LAUNCH_CHECK("pages_drop_kernel");
  return FC_OK;
}

extern "C" size_t fc_pages_workspace_bytes(int n_pages) { return n_pages > 0 ? copies_bytes(n_pages) : 0; }

extern "C" int fc_pages_fork(fc_ctx* ctx, void* stream, const fc_kv8_pool* pool, int H, int d, int32_t* ref, int32_t* table,
                             int64_t table_cs, int n_seq, int n, const int32_t* src, const int32_t* dst, const int32_t* tokens,
                             uint32_t* status, void* ws, size_t ws_bytes) {
  if (!ctx || n < 0 || n_seq <= 0 || table_cs < 0) return FC_ERR_INVALID_ARG;
  if (n > FC_MAX_CHUNKS) return FC_ERR_UNSUPPORTED;
  if (n == 0) return FC_OK;
  if (!src || !dst || !tokens || !ref || !table) return FC_ERR_INVALID_ARG;
  int rc = check_pool(pool, H, d);
  if (rc != FC_OK) return rc;
  Forks f = {};
  f.n = n;
  f.page = pool->page;
  f.table_cs = table_cs;
  int most = 0;
  for (int i = 0; i < n; ++i) {
    if (src[i] < 0 || src[i] >= n_seq || dst[i] < 0 || dst[i] >= n_seq || tokens[i] < 0) return FC_ERR_INVALID_ARG;
    if (((int64_t)tokens[i] + pool->page - 1) / pool->page > table_cs) return FC_ERR_INVALID_ARG;
    for (int k = 0; k < n; ++k)
      if (dst[i] == src[k] || (k != i && dst[i] == dst[k])) return FC_ERR_INVALID_ARG;
    f.src[i] = src[i];
    f.dst[i] = dst[i];
    f.tokens[i] = tokens[i];
    most += tokens[i] % pool->page != 0;
  }
  if (!fc::aligned16(ref)) return FC_ERR_MISALIGNED;
  if (!ws || ws_bytes < copies_bytes(pool->n_pages)) return FC_ERR_WORKSPACE;
  if (!fc::aligned16(ws)) return FC_ERR_MISALIGNED;
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
  const Copies copies = copies_at(ws, pool->n_pages);
  pages_fork_kernel<<<1, kThreads, 0, st>>>(ref, pool->n_pages, table, f, copies, status);
  FC_LAUNCH_CHECK("pages_fork_kernel");
  if (most == 0) return FC_OK;
  return launch_copies(ctx, st, {fc::kv8_view(*pool), copies, H, pool->page * d, nullptr, 0, 0, 0}, most, status);
}

extern "C" int fc_pages_compact(fc_ctx* ctx, void* stream, const fc_kv8_pool* pool, int H, int d, int32_t* ref, int32_t* table,
                                int64_t table_cs, int n_seq, int entries, int32_t* n_used, uint32_t* status, void* ws,
                                size_t ws_bytes) {
  if (!ctx || !ref || n_seq < 0 || entries < 0 || table_cs < 0) return FC_ERR_INVALID_ARG;
  if (n_seq > 0 && entries > 0 && (!table || (n_seq > 1 && table_cs < entries))) return FC_ERR_INVALID_ARG;
  int rc = check_pool(pool, H, d);
  if (rc != FC_OK) return rc;
  if (!fc::aligned16(ref)) return FC_ERR_MISALIGNED;
  if (!ws || ws_bytes < copies_bytes(pool->n_pages)) return FC_ERR_WORKSPACE;
  if (!fc::aligned16(ws)) return FC_ERR_MISALIGNED;
  FC_DEVICE_GUARD(ctx);
  cudaStream_t st = (cudaStream_t)stream;
  const Copies copies = copies_at(ws, pool->n_pages);
  pages_compact_kernel<<<1, kThreads, 0, st>>>(ref, pool->n_pages, copies, n_used);
  FC_LAUNCH_CHECK("pages_compact_kernel");
  const bool tables = n_seq > 0 && entries > 0;
  return launch_copies(ctx, st, {fc::kv8_view(*pool), copies, H, pool->page * d, table, table_cs, tables ? n_seq : 0, tables ? entries : 0},
                       std::max(pool->n_pages / 2, tables ? 1 : 0), status);
}
