// Host side of decode attention behind shared prefixes (include/opw_prefix.h): argument checks, choice of kernel, launches.
#include <cstdint>
#include <new>
#include <vector>

#include "opw_pool_map.h"
#include "opw_prefix.h"
#include "opw_prefix_kernels.cuh"
#include "opw_stage.h"

namespace {

using namespace opw_tree;

constexpr size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct PrefixLayout {
  size_t group_parts, row_parts, whole, group_cum, row_cum, info, split, total;
};

// Keys are numbered in 32 bits, and the last tile reaches past the last key: the table has to leave it that room.
bool keys_fit(const opw_stage_view& v) { return (int64_t)v.max_pages * kPage <= INT32_MAX - 2 * kMmaKeys; }

PrefixLayout carve(const opw_stage_view& v) {
  PrefixLayout L;
  const size_t batch = v.max_batch < kMaxPrefixBatch ? v.max_batch : kMaxPrefixBatch, row = (size_t)(v.D + 2) * 4;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes);
    return here;
  };
  L.group_parts = take(v.D == 256 ? 0 : (size_t)v.sms * 2 * 256 * row);
  L.row_parts = take((size_t)v.sms * 12 * 2 * 16 * row);
  L.whole = take(2 * batch * v.Hq * row);
  L.group_cum = take((size_t)(kMaxPrefixGroups + 1) * 8);
  L.row_cum = take((size_t)(kMaxPrefixGroups + kMaxPrefixBatch + 1) * 8);
  L.info = take((size_t)kMaxPrefixGroups * sizeof(GroupInfo));
  L.split = take(sizeof(PrefixSplit));
  L.total = at;
  return L;
}

// Who takes the groups: where one may have more than 16 rows (members x query heads of a kv head), the tensor cores, in blocks of up to 128 or, with
// 512 rows a group on average, of up to 256; else, and at head_dim 256 where two accumulators would fill TMEM, the warp kernel's 16 rows.
// How the batch is divided is known on the device only, and groups may be empty (a captured step has as many as it may ever need): the largest that
// there can be is the whole batch.  Measured, us, by the warp kernel, with 128 and with 256 rows; 32/8 heads of 128 unless said:
//   4 samples of 1000, 16 rows         14, 17, 18        64 behind 8k (256 rows)                  98, 45, 58
//   8 x 4 samples behind 4k, 16 rows   46, 47, 49        64 behind 8k, 64/8 heads (512 rows)     156, 61, 57
//   32 pairs behind 2k, 8 rows         78, 80, 88        256 behind 32k (1024 rows)             1053, 205, 182
// What this costs a batch that shares nothing, as many groups as rows: 64 rows of 1000 to 3000 keys 94, 100; 256 rows 220, 230; 5 rows of 500
// 14, 14; 8/2 heads of 64, 64 rows 25, 26.  Empty groups count in the average: 256 behind 32k among 255 of them is taken 128 rows at a time.
int mode_of(const opw_stage_view& v, int batch, int groups) {
  const int64_t rows = (int64_t)batch * (v.Hq / v.Hkv);
  if (v.D == 256 || rows <= 16) return kPrefixWarp;
  return rows < 512 * (int64_t)groups ? kPrefixNarrow : kPrefixWide;
}

template <int D, int kMode, bool kHigh>
cudaError_t raise_smem() {
  return cudaFuncSetAttribute(prefix_kernel<D, kMode, kHigh>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)PrefixSmem<D, kMode, kHigh>::kMost);
}
template <int D>
cudaError_t raise_all(bool high) {
  cudaError_t e = raise_smem<D, kPrefixWarp, true>();
  if constexpr (D != 256) {
    if (e == cudaSuccess) e = high ? raise_smem<D, kPrefixNarrow, true>() : raise_smem<D, kPrefixNarrow, false>();
    if (e == cudaSuccess) e = high ? raise_smem<D, kPrefixWide, true>() : raise_smem<D, kPrefixWide, false>();
  }
  return e;
}

template <int D, int kMode, bool kHigh>
cudaError_t launch(const opw_stage_view& v, const CUtensorMap& map, const PrefixParams& group_problem, const PrefixParams& p, cudaStream_t stream) {
  PrefixProblem<kGroupEnds> groups;
  PrefixProblem<kRowEnds> rows;
  static_cast<PrefixParams&>(groups) = group_problem;
  static_cast<PrefixParams&>(rows) = p;
  rows.lead = kMode == kPrefixWarp ? p.groups : 0;
  rows.all = rows.lead + p.batch;
  using S = PrefixSmem<D, kMode, kHigh>;
  rows.stages = S::stages(p.batch, p.groups);
  cudaError_t e = opw_launch(prefix_kernel<D, kMode, kHigh>, dim3(v.sms), dim3(S::kThreads), S::bytes(p.batch, p.groups, rows.stages), stream, v.pdl, 1, map, groups, rows);
  if (e != cudaSuccess) return e;
  *v.launches += 1;
  const int64_t n = (int64_t)p.batch * p.Hq, per = kPrefixCombineThreads / 32;
  const dim3 block(kPrefixCombineThreads);
  e = n < 4 * (int64_t)v.sms
          ? opw_launch(prefix_combine_kernel<D, kMode, kHigh, 4>, dim3((unsigned)n), block, 0, stream, v.pdl, 1, groups, rows)
          : opw_launch(prefix_combine_kernel<D, kMode, kHigh, 1>, dim3((unsigned)((n + per - 1) / per)), block, 0, stream, v.pdl, 1, groups, rows);
  if (e == cudaSuccess) *v.launches += 1;
  return e;
}
template <int D>
cudaError_t launch(const opw_stage_view& v, int mode, const CUtensorMap& map, const PrefixParams& g, const PrefixParams& p, cudaStream_t stream) {
  if constexpr (D != 256) {
    const bool high = p.G > 8;
    if (mode == kPrefixNarrow) return high ? launch<D, kPrefixNarrow, true>(v, map, g, p, stream) : launch<D, kPrefixNarrow, false>(v, map, g, p, stream);
    if (mode == kPrefixWide) return high ? launch<D, kPrefixWide, true>(v, map, g, p, stream) : launch<D, kPrefixWide, false>(v, map, g, p, stream);
  }
  return launch<D, kPrefixWarp, true>(v, map, g, p, stream);
}

}  // namespace

struct opw_prefix_attn {
  opw_attn_stage_t* stage;
  PrefixLayout lay;
  unsigned char* ws;
  std::vector<CUtensorMap> maps;   // of the layers' pools; empty at head_dim 256
};

extern "C" size_t opw_prefix_attn_workspace_bytes(const opw_attn_stage_t* stage) {
  if (!stage) return 0;
  const opw_stage_view v = opw_view_of(const_cast<opw_attn_stage_t*>(stage));
  return keys_fit(v) ? carve(v).total : 0;
}

extern "C" opw_status_t opw_prefix_attn_create(opw_attn_stage_t* stage, uint32_t flags, void* workspace, size_t workspace_bytes,
                                               opw_prefix_attn_t** out) {
  if (!stage || !out || !workspace || flags != 0 || (uintptr_t)workspace % 256) return OPW_ERR_INVALID_ARG;
  const opw_stage_view v = opw_view_of(stage);
  if (!keys_fit(v) || v.sms < 2) return OPW_ERR_UNSUPPORTED;      // (groups and rows have blocks of their own)
  const PrefixLayout lay = carve(v);
  if (workspace_bytes < lay.total) return OPW_ERR_CAPACITY;
  opw_device_guard guard(v.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  const cudaError_t e = v.D == 64 ? raise_all<64>(v.Hq / v.Hkv > 8) : v.D == 128 ? raise_all<128>(v.Hq / v.Hkv > 8) : raise_all<256>(false);
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  opw_prefix_attn* t = new (std::nothrow) opw_prefix_attn();
  if (!t) return OPW_ERR_INVALID_ARG;
  const opw_status_t mapped = v.D == 256 ? OPW_OK : opw_map_pools(v, &t->maps);
  if (mapped != OPW_OK) {
    delete t;
    return mapped;
  }
  t->stage = stage;
  t->lay = lay;
  t->ws = static_cast<unsigned char*>(workspace);
  *out = t;
  return OPW_OK;
}

extern "C" opw_status_t opw_prefix_attn_destroy(opw_prefix_attn_t* prefix) {
  delete prefix;
  return OPW_OK;
}

extern "C" opw_status_t opw_prefix_attention(opw_prefix_attn_t* prefix, int32_t layer, int32_t batch, int32_t groups, const void* q,
                                             const int32_t* kv_lens, const int32_t* group_starts, const int32_t* prefix_lens,
                                             const int32_t* page_table, void* out, float* lse, void* cuda_stream) {
  if (!prefix || batch < 0 || groups < 1) return OPW_ERR_INVALID_ARG;
  const opw_stage_view v = opw_view_of(prefix->stage);
  if (layer < 0 || layer >= v.num_layers) return OPW_ERR_INVALID_ARG;
  if (batch == 0) return OPW_OK;
  if (!q || !kv_lens || !group_starts || !prefix_lens || !page_table || !out) return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)out) % 16 ||
      ((uintptr_t)kv_lens | (uintptr_t)group_starts | (uintptr_t)prefix_lens | (uintptr_t)page_table | (uintptr_t)lse) % 4)
    return OPW_ERR_INVALID_ARG;
  if (batch > v.max_batch || batch > kMaxPrefixBatch || groups > kMaxPrefixGroups) return OPW_ERR_CAPACITY;
  // what is written must not meet what other blocks still read
  const size_t rows = (size_t)batch * v.Hq, lse_bytes = lse ? rows * 4 : 0, out_bytes = rows * v.D * 2;
  auto meets = [&](const void* in, size_t bytes) {
    return opw_overlap(out, out_bytes, in, bytes) || (lse && opw_overlap(lse, lse_bytes, in, bytes));
  };
  if (meets(q, out_bytes) || meets(kv_lens, (size_t)batch * 4) || meets(group_starts, (size_t)(groups + 1) * 4) ||
      meets(prefix_lens, (size_t)groups * 4) || meets(page_table, (size_t)batch * v.max_pages * 4) ||
      (lse && opw_overlap(lse, lse_bytes, out, out_bytes)))
    return OPW_ERR_INVALID_ARG;
  PrefixParams p;
  p.pool = static_cast<const __nv_bfloat16*>(v.pool[layer]);
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.lens = kv_lens;
  p.starts = group_starts;
  p.prefix_lens = prefix_lens;
  p.page_table = page_table;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  const PrefixLayout& lay = prefix->lay;
  p.partials = reinterpret_cast<float*>(prefix->ws + lay.row_parts);
  p.cum = reinterpret_cast<int64_t*>(prefix->ws + lay.row_cum);
  p.whole = reinterpret_cast<float*>(prefix->ws + lay.whole);
  p.info = reinterpret_cast<GroupInfo*>(prefix->ws + lay.info);
  p.split = reinterpret_cast<PrefixSplit*>(prefix->ws + lay.split);
  p.status = v.status;
  p.num_pages = v.num_pages[layer];
  p.batch = batch;
  p.groups = groups;
  p.Hq = v.Hq;
  p.Hkv = v.Hkv;
  p.G = v.Hq / v.Hkv;
  p.D = v.D;
  p.max_pages = v.max_pages;
  p.window = v.window[layer];
  p.scale_log2e = v.scale_log2e;
  p.lead = p.all = p.stages = 0;             // (with the launch)
  PrefixParams groups_problem = p;
  groups_problem.partials = reinterpret_cast<float*>(prefix->ws + lay.group_parts);
  groups_problem.cum = reinterpret_cast<int64_t*>(prefix->ws + lay.group_cum);
  groups_problem.lead = groups_problem.all = groups;
  opw_device_guard guard(v.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int mode = mode_of(v, batch, groups);
  static const CUtensorMap none = {};
  const CUtensorMap& map = prefix->maps.empty() ? none : prefix->maps[layer];
  const cudaError_t e = v.D == 64    ? launch<64>(v, mode, map, groups_problem, p, stream)
                        : v.D == 128 ? launch<128>(v, mode, map, groups_problem, p, stream)
                                     : launch<256>(v, mode, map, groups_problem, p, stream);
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  return OPW_OK;
}
