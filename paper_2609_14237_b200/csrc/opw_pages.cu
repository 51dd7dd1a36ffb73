// Sharing and returning pages of the paged cache (include/opw_pages.h): fork, release, list of free pages.
#include <cstdint>

#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "opw_pages.h"
#include "opw_stage.h"

namespace opw_pages {

constexpr int kPage = 16;
constexpr uint32_t kErrBadPage = 1u;      // bit of the stage's status word
constexpr int kLayersPerLaunch = 64;      // pool pointers travel as kernel parameters

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

struct ForkParams {
  void* pool[kLayersPerLaunch];
  const int32_t* src;
  const int32_t* dst;
  const int32_t* lens;
  const int32_t* fresh;       // new_pages
  int32_t* table;
  int32_t* refs;
  uint32_t* status;
  int32_t n, num_rows, max_pages, num_pages;
  int32_t tiles, row_vecs;    // K and V tiles per page (2 * Hkv); 16-byte words per cached row (D / 8)
  int32_t book;               // this launch also does the bookkeeping (the first of a group of many layers)
};

constexpr int kForkThreads = 256;

// grid (n, blocks per fork, layers of this launch [+ 1 in front for the bookkeeping]).  The copy moves, of each of the page's K and V tiles,
// the contiguous `rest` rows that hold a token -- half a page on average -- as 16-byte words, a warp a tile.  (With the tile of each word
// found by a division the kernel was bound by instructions: 256 forks x 8 layers 22.1 us, now 18.2.  Of that the
// 63 MB written and the 8 MB read, the page of a parent with many children once, would take a copy 10.8: most of the rest is each of the
// 4608 blocks finding out what it has to copy.)  Every block decides for itself whether its fork is refused: a scan of the n rows and
// page ids, which all blocks share in L2, against a second launch that a list of accepted forks would need.
__global__ void __launch_bounds__(kForkThreads) fork_kernel(const __grid_constant__ ForkParams p) {
  pdl_wait();
  const int f = blockIdx.x;
  const int32_t src = p.src[f], dst = p.dst[f], len = p.lens[f], fresh = p.fresh[f];
  const int rest = len % kPage, whole = len / kPage;
  bool bad = src < 0 || src >= p.num_rows || dst < 0 || dst >= p.num_rows || len < 0 ||
             (int64_t)len > (int64_t)p.max_pages * kPage;
  if (!bad && rest > 0) bad = fresh < 0 || fresh >= p.num_pages;
  if (!bad) {
    bool clash = false;
    for (int i = threadIdx.x; i < p.n; i += kForkThreads) {
      clash |= p.src[i] == dst;
      if (i != f) {
        clash |= p.dst[i] == dst || p.dst[i] == src;
        clash |= rest > 0 && p.fresh[i] == fresh && p.lens[i] % kPage > 0;
      }
    }
    bad = __syncthreads_or(clash);
  }
  int32_t from = -1;
  if (!bad && rest > 0) {
    from = p.table[(int64_t)src * p.max_pages + whole];
    bad = from < 0 || from >= p.num_pages;
  }
  const bool bookkeeper = p.book && blockIdx.z == 0;
  if (bad) {
    if (bookkeeper && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(p.status, kErrBadPage);
    return;
  }
  if (bookkeeper) {
    const int32_t* parent = p.table + (int64_t)src * p.max_pages;
    int32_t* child = p.table + (int64_t)dst * p.max_pages;
    for (int i = blockIdx.y * kForkThreads + threadIdx.x; i < p.max_pages; i += gridDim.y * kForkThreads) {
      int32_t id = -1;
      if (i < whole) {
        id = parent[i];
        if (id >= p.num_pages) {
          atomicOr(p.status, kErrBadPage);
          id = -1;
        }
        if (id >= 0) atomicAdd(p.refs + id, 1);
        else id = -1;
      } else if (i == whole && rest > 0) {
        id = fresh;
        p.refs[fresh] = 1;
      }
      child[i] = id;
    }
    return;
  }
  if (rest == 0) return;
  uint4* pool = static_cast<uint4*>(p.pool[blockIdx.z - p.book]);
  const int64_t tile_vecs = (int64_t)kPage * p.row_vecs;
  const uint4* a = pool + (int64_t)from * p.tiles * tile_vecs;
  uint4* b = pool + (int64_t)fresh * p.tiles * tile_vecs;
  const int used = rest * p.row_vecs, lane = threadIdx.x & 31;
  for (int t = blockIdx.y * (kForkThreads / 32) + (threadIdx.x >> 5); t < p.tiles; t += gridDim.y * (kForkThreads / 32)) {
    const uint4* from_tile = a + t * tile_vecs;
    uint4* to_tile = b + t * tile_vecs;
    for (int i0 = lane; i0 < used; i0 += 4 * 32) {
      uint4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i0 + 32 * u < used) v[u] = from_tile[i0 + 32 * u];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i0 + 32 * u < used) to_tile[i0 + 32 * u] = v[u];
    }
  }
}

// grid (blocks over the row's entries, n): an entry each.  The exchange makes a row that is named twice drop each
// page once.  Bound by the round trips of one thread (row, entry, exchange, count): 1.4 us for 8 rows, 1.9 for 128 rows of 512 entries.
constexpr int kReleaseThreads = 256;
__global__ void __launch_bounds__(kReleaseThreads) release_kernel(const int32_t* rows, const int32_t* keep_lens, int32_t* table,
                                                                  int32_t* refs, uint32_t* status, int32_t num_rows,
                                                                  int32_t max_pages, int64_t num_pages) {
  pdl_wait();
  const int32_t row = rows[blockIdx.y];
  const int i = blockIdx.x * kReleaseThreads + threadIdx.x;
  if (row < 0 || row >= num_rows) {
    if (i == 0) atomicOr(status, kErrBadPage);
    return;
  }
  const int32_t keep = keep_lens ? keep_lens[blockIdx.y] : 0;
  const int first = keep > 0 ? (int)(((int64_t)keep + kPage - 1) / kPage) : 0;
  if (i < first || i >= max_pages) return;
  const int32_t id = atomicExch(table + (int64_t)row * max_pages + i, -1);
  if (id < 0) return;
  if (id >= num_pages) {
    atomicOr(status, kErrBadPage);
    return;
  }
  if (atomicSub(refs + id, 1) <= 0) {
    atomicAdd(refs + id, 1);
    atomicOr(status, kErrBadPage);
  }
}

// One cluster: each block counts the free pages of its contiguous share, the counts meet through shared memory, and the ids are
// written behind those of the blocks before.  Ascending by construction, no scratch memory, one launch.  A thread takes four pages in
// a row; of up to eight such rounds it remembers the finding (256k pages in all), beyond that it reads the counts again.  1000 pages 3.3 us, 40000 4.6, 100000 6.4, 300000 13,
// 1000000 44 (most of the small ones: launch and two cluster barriers; the large ones: eight SMs).
constexpr int kListBlocks = 8;
constexpr int kListThreads = 1024;
constexpr int kListRound = 4 * kListThreads, kListKept = 8;
__global__ void __launch_bounds__(kListThreads) free_pages_kernel(const int32_t* refs, int64_t num_pages, int32_t* list,
                                                                  int64_t max_list, int32_t* count) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ int32_t warp_n[2][kListThreads / 32];
  __shared__ int32_t mine;
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = (int)cluster.block_rank();
  const int64_t lo = num_pages * rank / kListBlocks, hi = num_pages * (rank + 1) / kListBlocks;
  auto look = [&](int64_t base) -> uint32_t {                     // bit k: page base + 4 * thread + k is free
    const int64_t i = base + 4 * threadIdx.x;
    uint32_t f = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < hi && refs[i + k] == 0) f |= 1u << k;
    return f;
  };
  uint32_t kept = 0;
  int32_t n = 0;
  int round = 0;
  for (int64_t base = lo; base < hi; base += kListRound, ++round) {
    const uint32_t f = look(base);
    if (round < kListKept) kept |= f << (4 * round);
    n += __popc(f);
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if (lane == 0) warp_n[0][warp] = n;
  __syncthreads();
  if (warp == 0) {
    const int32_t t = __reduce_add_sync(0xffffffffu, warp_n[0][lane]);
    if (lane == 0) mine = t;
  }
  cluster.sync();
  int32_t at = 0, all = 0;
  for (int r = 0; r < kListBlocks; ++r) {
    const int32_t c = *cluster.map_shared_rank(&mine, r);
    if (r < rank) at += c;
    all += c;
  }
  if (rank == 0 && threadIdx.x == 0) *count = all;
  cluster.sync();                          // nobody leaves while its count is read
  round = 0;
  for (int64_t base = lo; base < hi; base += kListRound, ++round) {
    const uint32_t f = round < kListKept ? (kept >> (4 * round)) & 15u : look(base);
    const int own = __popc(f);
    int incl = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    int32_t* sums = warp_n[round & 1];     // (two in turn: one barrier a round)
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    const int32_t w = sums[lane];
    int64_t to = (int64_t)at + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0) + incl - own;
    at += __reduce_add_sync(0xffffffffu, w);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((f >> k) & 1u) {
        if (to < max_list) list[to] = (int32_t)(base + 4 * threadIdx.x + k);
        ++to;
      }
  }
}

// The layers of a table group: in range and named once.
bool layers_ok(const opw_stage_view& v, const int32_t* layers, int32_t n) {
  if (!layers || n < 1 || n > v.num_layers) return false;
  for (int i = 0; i < n; ++i) {
    if (layers[i] < 0 || layers[i] >= v.num_layers) return false;
    for (int j = 0; j < i; ++j)
      if (layers[j] == layers[i]) return false;
  }
  return true;
}

}  // namespace opw_pages

extern "C" opw_status_t opw_kv_fork(opw_attn_stage_t* stage, const int32_t* layers, int32_t num_layers, int32_t n,
                                    const int32_t* src_rows, const int32_t* dst_rows, const int32_t* lens,
                                    const int32_t* new_pages, int32_t num_rows, int32_t* page_table, int32_t* refcounts,
                                    void* cuda_stream) {
  if (!stage || n < 0 || num_rows < 1) return OPW_ERR_INVALID_ARG;
  const opw_stage_view v = opw_view_of(stage);
  if (!opw_pages::layers_ok(v, layers, num_layers)) return OPW_ERR_INVALID_ARG;
  if (n == 0) return OPW_OK;
  if (!src_rows || !dst_rows || !lens || !new_pages || !page_table || !refcounts) return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)src_rows | (uintptr_t)dst_rows | (uintptr_t)lens | (uintptr_t)new_pages | (uintptr_t)page_table |
       (uintptr_t)refcounts) % 4)
    return OPW_ERR_INVALID_ARG;
  if (n > 65535) return OPW_ERR_CAPACITY;
  opw_pages::ForkParams p;
  p.src = src_rows;
  p.dst = dst_rows;
  p.lens = lens;
  p.fresh = new_pages;
  p.table = page_table;
  p.refs = refcounts;
  p.status = v.status;
  p.n = n;
  p.num_rows = num_rows;
  p.max_pages = v.max_pages;
  int64_t pages = INT32_MAX;
  for (int i = 0; i < num_layers; ++i)
    if (v.num_pages[layers[i]] < pages) pages = v.num_pages[layers[i]];
  p.num_pages = (int32_t)pages;
  p.tiles = 2 * v.Hkv;
  p.row_vecs = v.D / 8;
  opw_device_guard guard(v.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  // A block of eight warps for each eight tiles of a page
  int splits = (p.tiles + opw_pages::kForkThreads / 32 - 1) / (opw_pages::kForkThreads / 32);
  const int entries = (v.max_pages + 2 * opw_pages::kForkThreads - 1) / (2 * opw_pages::kForkThreads);   // of the bookkeeping
  if (splits < entries) splits = entries;
  if (splits > 64) splits = 64;
  // The bookkeeping goes with the LAST launch: the copies of the others read the parents' rows, which it leaves alone, but
  // a later launch must still see the same table when it decides what is refused.
  for (int l0 = 0; l0 < num_layers; l0 += opw_pages::kLayersPerLaunch) {
    const int here = num_layers - l0 < opw_pages::kLayersPerLaunch ? num_layers - l0 : opw_pages::kLayersPerLaunch;
    for (int i = 0; i < here; ++i) p.pool[i] = v.pool[layers[l0 + i]];
    p.book = l0 + here == num_layers;
    if (opw_launch(opw_pages::fork_kernel, dim3(n, splits, here + p.book), dim3(opw_pages::kForkThreads), 0,
                   static_cast<cudaStream_t>(cuda_stream), v.pdl, 1, p) != cudaSuccess) {
      (void)cudaGetLastError();
      return OPW_ERR_CUDA;
    }
    *v.launches += 1;
  }
  return OPW_OK;
}

extern "C" opw_status_t opw_kv_release(opw_attn_stage_t* stage, int32_t n, const int32_t* rows, const int32_t* keep_lens,
                                       int32_t num_rows, int32_t* page_table, int32_t* refcounts, int64_t num_pages,
                                       void* cuda_stream) {
  if (!stage || n < 0 || num_rows < 1 || num_pages < 1 || num_pages > INT32_MAX) return OPW_ERR_INVALID_ARG;
  if (n == 0) return OPW_OK;
  if (!rows || !page_table || !refcounts) return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)rows | (uintptr_t)keep_lens | (uintptr_t)page_table | (uintptr_t)refcounts) % 4) return OPW_ERR_INVALID_ARG;
  if (n > 65535) return OPW_ERR_CAPACITY;
  const opw_stage_view v = opw_view_of(stage);
  opw_device_guard guard(v.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  const int blocks = (v.max_pages + opw_pages::kReleaseThreads - 1) / opw_pages::kReleaseThreads;
  if (opw_launch(opw_pages::release_kernel, dim3(blocks, n), dim3(opw_pages::kReleaseThreads), 0,
                 static_cast<cudaStream_t>(cuda_stream), v.pdl, 1, rows, keep_lens, page_table, refcounts, v.status, num_rows,
                 v.max_pages, num_pages) != cudaSuccess) {
    (void)cudaGetLastError();
    return OPW_ERR_CUDA;
  }
  *v.launches += 1;
  return OPW_OK;
}

extern "C" opw_status_t opw_kv_free_pages(opw_attn_stage_t* stage, const int32_t* refcounts, int64_t num_pages,
                                          int32_t* free_list, int64_t max_list, int32_t* count, void* cuda_stream) {
  if (!stage || num_pages < 1 || num_pages > INT32_MAX || max_list < 0) return OPW_ERR_INVALID_ARG;
  if (!refcounts || !count || (max_list > 0 && !free_list)) return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)refcounts | (uintptr_t)free_list | (uintptr_t)count) % 4) return OPW_ERR_INVALID_ARG;
  const opw_stage_view v = opw_view_of(stage);
  opw_device_guard guard(v.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  if (opw_launch(opw_pages::free_pages_kernel, dim3(opw_pages::kListBlocks), dim3(opw_pages::kListThreads), 0,
                 static_cast<cudaStream_t>(cuda_stream), v.pdl, opw_pages::kListBlocks, refcounts, num_pages, free_list, max_list,
                 count) != cudaSuccess) {
    (void)cudaGetLastError();
    return OPW_ERR_CUDA;
  }
  *v.launches += 1;
  return OPW_OK;
}
