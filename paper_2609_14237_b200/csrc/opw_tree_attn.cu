// Host side of tree attention (include/opw_draft.h): argument checks, choice of kernel, launches.
#include <cstdint>
#include <new>
#include <vector>

#include "opw_draft.h"
#include "opw_pool_map.h"
#include "opw_stage.h"
#include "opw_tree_kernels.cuh"
#include "opw_tree_mma.cuh"

namespace {

constexpr size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct TreeLayout {
  size_t cum, partials, total;
};

struct Variant {              // a kernel, and how it cuts rows and keys
  int row_block, keys, workers;
  bool mma, wide;
};

// Keys are numbered in 32 bits, and the last tile reaches past the last key: the table has to leave it that room.
bool keys_fit(const opw_stage_view& v) {
  return (int64_t)v.max_pages * opw_tree::kPage <= INT32_MAX - 2 * opw_tree::kMmaKeys;
}

constexpr int kMmaMaxBatch = 2048;   // what the prefix sums may take of the shared memory beside the tiles

// Which kernel.  The tensor-core kernel reads a key tile once for 128 or 256 rows, a CTA at a time; the warp kernel once for 16 rows, a page
// and a warp at a time.  Measured at 32/8 heads of 128, us:
//   up to 16 rows, many sequences (64 of 1k to 4k keys, trees of 2 and 4)    warp 116 and 121, tensor core 132 and 135
//   up to 16 rows, fewer heads than twice the SMs (1 sequence of 1000 keys)  warp 14.7, tensor core 12.5 (now 11.5): a partial per CTA, not per warp
//   17 to 32 rows (64 sequences, trees of 8)   warp, with two row tiles a warp, 139; tensor core 130
//   beyond, the warp kernel would read the cache once per 16 rows (16 x 32k keys, 256 rows: 3133; tensor core 560)
// Both sides at other shapes (warp, tensor core; 64 sequences of 1k to 4k keys unless said): 64/8 heads of 128, 8 and 16 rows 114 and 126, 32 rows
// 183 and 129.  32/8 of 64, 8 and 16 rows 62 and 105, 32 rows 98 and 106; 40 sequences, 16 rows 43 and 69.  One sequence of 1000 keys, a
// chain of 4: 64/8 of 128 13.6 and 12.2, 16/1 of 128 11.8 and 11.0, 8/2 of 64 11.0 and 8.9.  16/1 of 128, 16 and 32 rows 33 and 27, 34 and 28.
// Known misses, where the rule of few heads takes the tensor cores and the warp kernel is faster: head_dim 64, 32 sequences of 8 kv heads 38 and
// 57; one kv head of 128, 16 sequences of 16 rows 15 and 22.
// The wide instance (two query tiles in shared memory) from 129 rows on; for up to 128 rows the narrow one with its deeper ring (130 against
// 138 us for the trees of 8).  At head_dim 256 two slots' accumulators alone would take all 512 columns of TMEM; those heads go through the
// warp kernel at every number of rows.
Variant pick(const opw_stage_view& v, int nodes, int batch) {
  const int rows = nodes * (v.Hq / v.Hkv);
  Variant k;
  k.wide = rows > 128;
  const bool few = batch * v.Hkv < 2 * v.sms;
  k.mma = (rows > 16 || few) && v.D != 256 && batch <= kMmaMaxBatch;
  k.keys = k.mma ? opw_tree::kMmaKeys : 16;
  k.row_block = k.mma ? (k.wide ? 256 : 128) : 16;
  k.workers = k.mma ? v.sms : v.sms * (v.D == 64 ? 12 : v.D == 128 ? 8 : 6);
  return k;
}

TreeLayout carve(const opw_stage_view& v, int max_nodes) {
  TreeLayout L;
  L.cum = 0;
  L.partials = align_up((size_t)(opw_tree::kMaxTreeBatch + 1) * 8);
  size_t most = 0;            // over every number of nodes a call may have
  for (int n = 1; n <= max_nodes; ++n) {
    for (int b : {1, kMmaMaxBatch, kMmaMaxBatch + 1}) {
      const Variant k = pick(v, n, b);
      const size_t need = (size_t)k.workers * 2 * k.row_block * (v.D + 2) * 4;
      if (need > most) most = need;
    }
  }
  L.total = L.partials + align_up(most);
  return L;
}

template <int D>
cudaError_t raise_smem() {
  return cudaFuncSetAttribute(opw_tree::tree_warp_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)opw_tree::WarpTree<D>::smem(opw_tree::kMaxTreeBatch));
}
template <int D, bool kWide>
cudaError_t raise_smem_mma() {
  return cudaFuncSetAttribute(opw_tree::tree_mma_kernel<D, kWide>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)opw_tree::MmaTree<D, kWide>::smem(kMmaMaxBatch));
}

template <int D>
cudaError_t launch_warp(const opw_stage_view& v, const opw_tree::TreeParams& p, cudaStream_t stream) {
  using C = opw_tree::WarpTree<D>;
  return opw_launch(opw_tree::tree_warp_kernel<D>, dim3(v.sms), dim3(C::kWarps * 32), C::smem(p.batch), stream, v.pdl, 1, p);
}

template <int D>
cudaError_t launch_combine(const opw_stage_view& v, const opw_tree::TreeCombineParams& c, int64_t blocks, bool deal,
                           cudaStream_t stream) {
  const int all = c.t.nodes * c.t.G, rows = all < c.row_block ? all : c.row_block, per = deal ? 4 : 32;
  const dim3 grid((unsigned)blocks, (rows + per - 1) / per, deal ? D / 32 : 1), block(opw_tree::kTreeCombineThreads);
  return deal ? opw_launch(opw_tree::tree_combine_kernel<D, 8, 1>, grid, block, 0, stream, v.pdl, 1, c)
              : opw_launch(opw_tree::tree_combine_kernel<D, 1, D / 32>, grid, block, 0, stream, v.pdl, 1, c);
}

template <int D, bool kWide>
cudaError_t launch_mma(const opw_stage_view& v, const CUtensorMap& map, const opw_tree::TreeParams& p, cudaStream_t stream) {
  return opw_launch(opw_tree::tree_mma_kernel<D, kWide>, dim3(v.sms), dim3(opw_tree::kMmaThreads),
                    opw_tree::MmaTree<D, kWide>::smem(p.batch), stream, v.pdl, 1, map, p);
}

}  // namespace

struct opw_tree_attn {
  opw_attn_stage_t* stage;
  int32_t max_nodes;
  TreeLayout lay;
  unsigned char* ws;
  std::vector<CUtensorMap> maps;   // of the layers' pools; empty at head_dim 256
};

extern "C" opw_status_t opw_tree_mask(int32_t nodes, const int32_t* parents, uint64_t* mask, int32_t* depth) {
  if (nodes < 1 || nodes > OPW_TREE_MAX_NODES || !parents || !mask) return OPW_ERR_INVALID_ARG;
  for (int i = 0; i < nodes; ++i)
    if (parents[i] < -1 || parents[i] >= i) return OPW_ERR_INVALID_ARG;
  for (int i = 0; i < nodes; ++i) {
    const int up = parents[i];
    mask[i] = (up >= 0 ? mask[up] : 0ull) | 1ull << i;
    if (depth) depth[i] = up >= 0 ? depth[up] + 1 : 0;
  }
  return OPW_OK;
}

extern "C" size_t opw_tree_attn_workspace_bytes(const opw_attn_stage_t* stage, int32_t max_nodes) {
  if (!stage || max_nodes < 1 || max_nodes > OPW_TREE_MAX_NODES) return 0;
  const opw_stage_view v = opw_view_of(const_cast<opw_attn_stage_t*>(stage));
  return keys_fit(v) ? carve(v, max_nodes).total : 0;
}

extern "C" opw_status_t opw_tree_attn_create(opw_attn_stage_t* stage, int32_t max_nodes, uint32_t flags, void* workspace,
                                             size_t workspace_bytes, opw_tree_attn_t** out) {
  if (!stage || !out || !workspace || flags != 0) return OPW_ERR_INVALID_ARG;
  if (max_nodes < 1 || max_nodes > OPW_TREE_MAX_NODES || (uintptr_t)workspace % 256) return OPW_ERR_INVALID_ARG;
  const opw_stage_view v = opw_view_of(stage);
  if (!keys_fit(v)) return OPW_ERR_UNSUPPORTED;
  const TreeLayout lay = carve(v, max_nodes);
  if (workspace_bytes < lay.total) return OPW_ERR_CAPACITY;
  opw_device_guard guard(v.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  cudaError_t e;
  if (v.D == 64) {
    e = raise_smem<64>();
    if (e == cudaSuccess) e = raise_smem_mma<64, false>();
    if (e == cudaSuccess) e = raise_smem_mma<64, true>();
  } else if (v.D == 128) {
    e = raise_smem<128>();
    if (e == cudaSuccess) e = raise_smem_mma<128, false>();
    if (e == cudaSuccess) e = raise_smem_mma<128, true>();
  } else {
    e = raise_smem<256>();
  }
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  opw_tree_attn* t = new (std::nothrow) opw_tree_attn();
  if (!t) return OPW_ERR_INVALID_ARG;
  const opw_status_t mapped = v.D == 256 ? OPW_OK : opw_map_pools(v, &t->maps);
  if (mapped != OPW_OK) {
    delete t;
    return mapped;
  }
  t->stage = stage;
  t->max_nodes = max_nodes;
  t->lay = lay;
  t->ws = static_cast<unsigned char*>(workspace);
  *out = t;
  return OPW_OK;
}

extern "C" opw_status_t opw_tree_attn_destroy(opw_tree_attn_t* tree) {
  delete tree;
  return OPW_OK;
}

extern "C" opw_status_t opw_tree_attention(opw_tree_attn_t* tree, int32_t layer, int32_t batch, int32_t nodes, const void* q,
                                           const uint64_t* tree_mask, const int32_t* positions, const int32_t* ctx_lens,
                                           const int32_t* tree_lens, const int32_t* page_table, void* out, float* lse,
                                           void* cuda_stream) {
  if (!tree || batch < 0 || nodes < 1) return OPW_ERR_INVALID_ARG;
  const opw_stage_view v = opw_view_of(tree->stage);
  if (layer < 0 || layer >= v.num_layers) return OPW_ERR_INVALID_ARG;
  if (batch == 0) return OPW_OK;
  if (!q || !tree_mask || !positions || !ctx_lens || !tree_lens || !page_table || !out) return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)out) % 16 || (uintptr_t)tree_mask % 8 ||
      ((uintptr_t)positions | (uintptr_t)ctx_lens | (uintptr_t)tree_lens | (uintptr_t)page_table | (uintptr_t)lse) % 4)
    return OPW_ERR_INVALID_ARG;
  if (nodes > tree->max_nodes || batch > v.max_batch || batch > opw_tree::kMaxTreeBatch) return OPW_ERR_CAPACITY;
  // what is written must not meet what other blocks still read
  const size_t rows = (size_t)batch * nodes, lse_bytes = lse ? rows * v.Hq * 4 : 0, out_bytes = rows * v.Hq * v.D * 2;
  auto meets = [&](const void* in, size_t bytes) {
    return opw_overlap(out, out_bytes, in, bytes) || (lse && opw_overlap(lse, lse_bytes, in, bytes));
  };
  if (meets(q, out_bytes) || meets(tree_mask, rows * 8) || meets(positions, rows * 4) || meets(ctx_lens, (size_t)batch * 4) ||
      meets(tree_lens, (size_t)batch * 4) || meets(page_table, (size_t)batch * v.max_pages * 4) ||
      (lse && opw_overlap(lse, lse_bytes, out, out_bytes)))
    return OPW_ERR_INVALID_ARG;
  const Variant k = pick(v, nodes, batch);
  opw_tree::TreeCombineParams c;
  opw_tree::TreeParams& p = c.t;
  p.pool = static_cast<const __nv_bfloat16*>(v.pool[layer]);
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.mask = tree_mask;
  p.positions = positions;
  p.ctx_lens = ctx_lens;
  p.tree_lens = tree_lens;
  p.page_table = page_table;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.partials = reinterpret_cast<float*>(tree->ws + tree->lay.partials);
  p.cum = reinterpret_cast<int64_t*>(tree->ws + tree->lay.cum);
  p.status = v.status;
  p.num_pages = v.num_pages[layer];
  p.batch = batch;
  p.nodes = nodes;
  p.Hq = v.Hq;
  p.Hkv = v.Hkv;
  p.G = v.Hq / v.Hkv;
  p.max_pages = v.max_pages;
  p.window = v.window[layer];
  p.scale_log2e = v.scale_log2e;
  c.D = v.D;
  c.row_block = k.row_block;
  c.keys = k.keys;
  c.max_blocks = (nodes * p.G + k.row_block - 1) / k.row_block;
  c.workers = k.workers;
  opw_device_guard guard(v.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (k.mma) {
    const CUtensorMap& map = tree->maps[layer];
    if (v.D == 64) e = k.wide ? launch_mma<64, true>(v, map, p, stream) : launch_mma<64, false>(v, map, p, stream);
    else e = k.wide ? launch_mma<128, true>(v, map, p, stream) : launch_mma<128, false>(v, map, p, stream);
  } else {
    e = v.D == 64 ? launch_warp<64>(v, p, stream) : v.D == 128 ? launch_warp<128>(v, p, stream) : launch_warp<256>(v, p, stream);
  }
  if (e == cudaSuccess) {
    *v.launches += 1;
    // Partials per row block, about: workers / blocks.  Above twelve they are dealt out to groups of threads: one chain of 4 at 1000
    // keys 12.5 us without, 12.2 with, at 8000 keys 21 and 19; where blocks are many it only adds blocks (64 trees of 8: 129 us
    // without, 208 with).  Without and with, chains of 4 at other shapes: 8/2 heads of 64, 8000 keys 28 and 12, 4 sequences 19 and 15.6;
    // 16/1 of 128 64 and 14, 4 sequences 35 and 15, 16 of them (not dealt out) 31 and 34; 16/2 of 256 64 and 18, 4 sequences 55 and 32, 16 (dealt out,
    // a miss) 66 and 75.
    const int64_t blocks = (int64_t)batch * v.Hkv * c.max_blocks;
    const bool deal = k.workers > 12 * blocks;
    e = v.D == 64 ? launch_combine<64>(v, c, blocks, deal, stream)
        : v.D == 128 ? launch_combine<128>(v, c, blocks, deal, stream) : launch_combine<256>(v, c, blocks, deal, stream);
  }
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  *v.launches += 1;
  return OPW_OK;
}
