// Device code of decode attention behind shared prefixes (include/opw_prefix.h).
//
// The shared keys of a group are a problem of their own: its rows are the group's members x G query heads of a kv head, all of which see
// (almost) the same keys, so that a key tile that is read once serves up to 256 rows on the tensor cores.  The keys behind the prefix are
// the ordinary split-KV decode problem, G rows a sequence.  Both are the problems that the kernels of tree attention take
// (opw_tree_kernels.cuh), solved in ONE launch: some blocks run the tensor-core kernel over the groups, the others the warp kernel over the
// sequences, divided by what either costs.  The parts of a row's result -- one per worker that had keys of it -- are left in fp32
// and merged by a second kernel.
#pragma once

#include "opw_tree_mma.cuh"

namespace opw_tree {

constexpr int kMaxPrefixBatch = 2048, kMaxPrefixGroups = 1024;
constexpr int kRowWarps = 8;              // of a block with the sequences' own keys

// A group: keys that are shared (a multiple of the page, 0: none), the row of the page table to read them through, the shortest and
// the longest of its active members.
struct GroupInfo {
  int32_t shared, leader, shortest, longest;
};
struct PrefixSplit {                      // of a launch: blocks and units of either problem
  int64_t group_units, row_units;
  int32_t group_blocks, row_blocks;
};

struct PrefixParams {
  const __nv_bfloat16* pool;
  const __nv_bfloat16* q;
  const int32_t* lens;
  const int32_t* starts;
  const int32_t* prefix_lens;
  const int32_t* page_table;
  __nv_bfloat16* out;
  float* lse;
  float* group_parts;    // the partial slots of either problem
  float* row_parts;
  float* whole;          // [2][batch * Hq][D] outputs, [2][batch * Hq] maxima, sums: rows that one worker has seen all of
  int64_t* group_cum;    // units before each entity, for the merge
  int64_t* row_cum;
  GroupInfo* info;
  PrefixSplit* split;
  uint32_t* status;
  int64_t num_pages;
  int32_t batch, groups, Hq, Hkv, G, D, max_pages, window;
  float scale_log2e;
};

__device__ __forceinline__ int32_t length_of(const PrefixParams& p, int b) {   // 0: inactive
  const int64_t cap = min((int64_t)p.max_pages * kPage, (int64_t)INT32_MAX);
  return (int32_t)min((int64_t)max(p.lens[b], 0), cap);
}
__device__ __forceinline__ int32_t window_start(const PrefixParams& p, int32_t n) { return p.window > 0 ? max(n - p.window, 0) : 0; }
// the group of row b
__device__ __forceinline__ int group_of(const int32_t* starts, int groups, int b) {
  int lo = 0, hi = groups;                   // starts[lo] <= b < starts[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid] <= b) lo = mid; else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ Span no_span() { return {0, 0, 0, 0, 1, 0, 0, false}; }
// The rows of a group and its shared keys.  ctx: the first key that some row does not see.
__device__ __forceinline__ Span group_span(const PrefixParams& p, const GroupInfo& i, int32_t start, int32_t end, int row_block) {
  if (i.shared <= 0) return no_span();
  Span s;
  s.tree = end - start;
  s.ctx = min(i.shortest, i.shared);
  s.n = i.shared;
  s.lo = min(window_start(p, i.shortest), s.n);
  s.blocks = (s.tree * p.G + row_block - 1) / row_block;
  s.table_row = i.leader;
  s.first_row = start;
  s.cut = false;
  return s;
}
// One row and the keys of its own.
__device__ __forceinline__ Span row_span(const PrefixParams& p, int32_t shared, int b) {
  const int32_t n = length_of(p, b);
  Span s = no_span();
  s.cut = p.lens[b] > n;
  if (n <= 0) return s;
  s.tree = 1;
  s.ctx = s.n = n;
  s.lo = min(max(shared, window_start(p, n)), n);
  s.table_row = s.first_row = b;
  return s;
}

// What the kernels' bodies are given: entities [0, lead) are groups, those behind rows (a problem has either or both).  starts and info in
// shared memory.
struct PrefixProblem : PrefixParams {
  const int32_t* first;      // starts
  const GroupInfo* group;
  float* partials;
  int64_t* cum;
  int32_t lead, all;
};
__device__ __forceinline__ int entities(const PrefixProblem& p) { return p.all; }
__device__ __forceinline__ Span span_of(const PrefixProblem& p, int e, int row_block) {
  if (e < p.lead) return group_span(p, p.group[e], p.first[e], p.first[e + 1], row_block);
  const int b = e - p.lead;
  return row_span(p, p.group[group_of(p.first, p.groups, b)].shared, b);
}
__device__ __forceinline__ RowView row_view(const PrefixProblem& p, int e, const Span& s, int node) {
  const int32_t n = length_of(p, s.first_row + node);
  RowView v;
  v.bits = 0ull;
  v.ctx = INT32_MAX;                         // (nothing is drafted)
  v.end = min(n, s.n);
  v.lo = e < p.lead ? window_start(p, n) : s.lo;
  return v;
}
__device__ __forceinline__ int32_t window_border(const PrefixProblem& p, int e, const Span& s, int) {
  return e < p.lead ? max(s.lo, window_start(p, p.group[e].longest)) : s.lo;
}
// A group of one active row shares nothing: a span of two rows and more is a group's.
__device__ __forceinline__ bool finished_at_once(const PrefixProblem& p, const Span& s) {
  if (s.tree > 1) return false;
  const int g = group_of(p.first, p.groups, s.first_row);
  const Span shared = group_span(p, p.group[g], p.first[g], p.first[g + 1], 1);
  return shared.n <= shared.lo;
}
__device__ __forceinline__ RowPart whole_of(const PrefixParams& p, bool shared, int64_t row) {
  const int64_t rows = (int64_t)p.batch * p.Hq, r = (shared ? 0 : rows) + row;
  float* ml = p.whole + 2 * rows * p.D;
  return {p.whole + r * p.D, ml + r, ml + 2 * rows + r};
}
__device__ __forceinline__ RowPart whole_row(const PrefixProblem& p, const Span& s, int64_t row) { return whole_of(p, s.tree > 1, row); }

// Sum over the block of one value each.
__device__ __forceinline__ int64_t block_sum(int64_t v) {
  __shared__ int64_t part[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (lane == 0) part[warp] = v;
  __syncthreads();
  int64_t all = 0;
  for (int w = 0; w < warps; ++w) all += part[w];
  return all;
}

// What every block finds out for itself: starts and group infos in shared memory.  Starts that do not ascend from 0 to the batch share
// nothing and are recorded.
__device__ __forceinline__ void survey_groups(const PrefixParams& p, int32_t* first, GroupInfo* info) {
  // (until the last step info holds: the longest length and, inverted, its first row as one word; the shortest; the number of active rows)
  bool wrong = false;
  for (int g = threadIdx.x; g <= p.groups; g += blockDim.x) {
    const int32_t s = p.starts[g];
    first[g] = s;
    wrong |= g == 0 ? s != 0 : s < p.starts[g - 1];
    wrong |= g == p.groups && s != p.batch;
    if (g < p.groups) info[g] = {0, 0, INT32_MAX, 0};
  }
  if (__syncthreads_or(wrong)) {
    for (int g = threadIdx.x; g < p.groups; g += blockDim.x) info[g] = {0, 0, 0, 0};
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.status, kErrBadPage);
    __syncthreads();
    return;
  }
  const int lane = threadIdx.x & 31;
  for (int b0 = threadIdx.x - lane; b0 < p.batch; b0 += blockDim.x) {
    const int b = b0 + lane;
    const int32_t n = b < p.batch ? length_of(p, b) : 0;
    const int g = group_of(first, p.groups, min(b, p.batch - 1));
    unsigned long long best = n > 0 ? ((unsigned long long)(uint32_t)n << 32) | (0xffffffffu - (uint32_t)b) : 0ull;
    int32_t least = n > 0 ? n : INT32_MAX, active = n > 0 ? 1 : 0;
    const bool alone = __shfl_sync(0xffffffffu, g, 0) != __shfl_sync(0xffffffffu, g, 31);   // the warp's rows are of several groups
    if (!alone) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
        active += __shfl_xor_sync(0xffffffffu, active, o);
      }
    }
    if ((alone || lane == 0) && active > 0) {
      atomicMax(reinterpret_cast<unsigned long long*>(&info[g]), best);
      atomicMin(&info[g].shortest, least);
      atomicAdd(&info[g].longest, active);
    }
  }
  __syncthreads();
  for (int g = threadIdx.x; g < p.groups; g += blockDim.x) {
    const unsigned long long best = *reinterpret_cast<const unsigned long long*>(&info[g]);
    const int32_t longest = (int32_t)(best >> 32), active = info[g].longest;
    GroupInfo i;
    i.shared = active > 1 ? max(min(p.prefix_lens[g], longest), 0) / kPage * kPage : 0;
    i.leader = (int32_t)(0xffffffffu - (uint32_t)best);
    i.shortest = info[g].shortest;
    i.longest = longest;
    info[g] = i;
  }
  __syncthreads();
}

// How many of the blocks take the groups: by what a tile of 64 keys (of 128 or 256 rows) and a page of a sequence's own keys cost.
__device__ __forceinline__ int group_blocks(int64_t group_units, int64_t row_units, int64_t row_blocks, int blocks, bool wide) {
  if (group_units == 0) return 0;
  const int64_t a = group_units * (wide ? 7 : 5), b = row_units + 2 * row_blocks;
  int64_t n = (a * blocks + (a + b) / 2) / (a + b);
  n = min(n, group_units);
  if (row_units > 0) n = min(n, (int64_t)blocks - 1);
  return (int)max(n, (int64_t)1);
}

enum PrefixMode { kPrefixWarp, kPrefixNarrow, kPrefixWide };   // the groups by the warp kernel, or by the tensor-core one with 128 or 256 rows

template <int D, int kMode>
struct PrefixSmem {
  static constexpr bool kMma = kMode != kPrefixWarp;
  using Mma = MmaTree<D == 256 ? 128 : D, kMode == kPrefixWide>;
  static constexpr int kWarps = kMma ? kRowWarps : WarpTree<D>::kWarps == 12 ? 12 : D == 256 ? 5 : 8;
  static constexpr int kThreads = kMma ? kMmaThreads : kWarps * 32;
  static constexpr size_t kRing = (size_t)kWarps * WarpTree<D>::kStages * (WarpTree<D>::kTile + 8);
  static constexpr size_t kTiles = kMma ? 1024 + (size_t)Mma::kPieces * Mma::kPiece + (size_t)Mma::kQTiles * Mma::kQTile : 0;
  // blocks with groups need units for those only, the others for the rows (and, without the tensor cores, for both)
  __host__ __device__ static constexpr size_t tables(int groups) { return (size_t)(groups + 1) * 16 + (size_t)((groups + 4) / 4) * 16; }
  static size_t bytes(int batch, int groups) {
    const size_t rows = kRing + (size_t)(batch + (kMma ? 0 : groups) + 1) * 8, tiles = kTiles + (size_t)(groups + 1) * 8;
    return tables(groups) + (kMma && tiles > rows ? tiles : rows);
  }
};

// Shared memory: group infos, starts, then the tiles of the block's role and behind them its entities' units.
template <int D, int kMode>
__global__ void __launch_bounds__(PrefixSmem<D, kMode>::kThreads, 1) prefix_kernel(const __grid_constant__ CUtensorMap map,
                                                                                   const __grid_constant__ PrefixParams p) {
  using S = PrefixSmem<D, kMode>;
  extern __shared__ __align__(128) unsigned char smem[];
  GroupInfo* info = reinterpret_cast<GroupInfo*>(smem);
  int32_t* first = reinterpret_cast<int32_t*>(smem + (size_t)(p.groups + 1) * 16);
  unsigned char* room = smem + S::tables(p.groups);
  survey_groups(p, first, info);

  PrefixProblem x;
  static_cast<PrefixParams&>(x) = p;
  x.first = first;
  x.group = info;
  int group_n = 0;
  int64_t group_units = 0, row_units = 0;
  if (S::kMma) {
    constexpr int kRowBlock = kMode == kPrefixWide ? 256 : 128;
    int64_t a = 0, b = 0;
    for (int g = threadIdx.x; g < p.groups; g += S::kThreads) {
      const Span s = group_span(p, info[g], first[g], first[g + 1], kRowBlock);
      a += (int64_t)tiles_of(s, kMmaKeys) * s.blocks * p.Hkv;
    }
    for (int r = threadIdx.x; r < p.batch; r += S::kThreads)
      b += (int64_t)tiles_of(row_span(p, info[group_of(first, p.groups, r)].shared, r), kPage) * p.Hkv;
    group_units = block_sum(a);
    row_units = block_sum(b);
    group_n = group_blocks(group_units, row_units, (int64_t)p.batch * p.Hkv, gridDim.x, kMode == kPrefixWide);
  }
  const bool grouped = (int)blockIdx.x < group_n;
  if (grouped) {
    if constexpr (S::kMma) {
      x.lead = x.all = p.groups;
      x.partials = p.group_parts;
      x.cum = p.group_cum;
      int64_t* cum = reinterpret_cast<int64_t*>(room + S::kTiles);
      mma_body<D, kMode == kPrefixWide>(map, x, room, cum, blockIdx.x, group_n);
    }
  } else {
    x.lead = S::kMma ? 0 : p.groups;
    x.all = x.lead + p.batch;
    x.partials = p.row_parts;
    x.cum = p.row_cum;
    int64_t* cum = reinterpret_cast<int64_t*>(room + S::kRing);
    scan_units(x, cum, WarpTree<D>::kRows, kPage, (int)blockIdx.x == group_n);
    if (!S::kMma) row_units = cum[x.all];
    if (!S::kMma || threadIdx.x < S::kWarps * 32) {
      if constexpr (S::kMma) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");   // 256 x 224 + 128 x 56 = 384 x 168
      warp_body<D, S::kWarps>(x, room, cum, blockIdx.x - group_n, gridDim.x - group_n);
    } else {
      if constexpr (S::kMma) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
      pdl_launch_dependents();
      pdl_wait();
    }
  }
  if (blockIdx.x == 0) {
    for (int g = threadIdx.x; g < p.groups; g += S::kThreads) p.info[g] = info[g];
    if (threadIdx.x == 0) *p.split = {group_units, row_units, group_n, (int32_t)gridDim.x - group_n};
  }
}

// A warp per row of the output; a lane has D / 32 neighbouring columns.  The row's parts are looked up 32 at a time, a lane each (whose slot,
// maximum and sum), then added up column by column.
constexpr int kPrefixCombineThreads = 128;
template <int D, int kMode>
__global__ void __launch_bounds__(kPrefixCombineThreads) prefix_combine_kernel(const PrefixParams p) {
  using S = PrefixSmem<D, kMode>;
  constexpr int kCols = D / 32, kRowBlock = kMode == kPrefixWide ? 256 : kMode == kPrefixNarrow ? 128 : WarpTree<D>::kRows;
  constexpr int kGroupKeys = S::kMma ? kMmaKeys : kPage;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * (kPrefixCombineThreads / 32) + (threadIdx.x >> 5);
  if (row >= (int64_t)p.batch * p.Hq) return;
  const int b = (int)(row / p.Hq), h = (int)(row - (int64_t)b * p.Hq), g = h / p.G;
  const int gi = group_of(p.starts, p.groups, b);
  const int32_t start = p.starts[gi], end = p.starts[gi + 1];
  const bool active = length_of(p, b) > 0;
  pdl_launch_dependents();
  pdl_wait();                                // up to here only the lengths and starts were read
  const GroupInfo info = p.info[gi];
  const PrefixSplit split = *p.split;
  const Span gs = group_span(p, info, start, end, kRowBlock), rs = row_span(p, info.shared, b);
  const int32_t gt = active ? tiles_of(gs, kGroupKeys) : 0, rt = tiles_of(rs, kPage);
  // the workers that had keys of this row
  int64_t gw = 0, rw = 0, gfirst = 0, rfirst = 0, gworkers = 1, rworkers = 1;
  int gn = 0, rn = 0;                        // parts
  const int R = (b - start) * p.G + (h - g * p.G), rb = R / kRowBlock;
  const int64_t group_units = S::kMma ? split.group_units : split.row_units;
  if (gt > 0) {
    gworkers = S::kMma ? workers_for(group_units, split.group_blocks, kMmaKeys)
                       : workers_for(group_units, (int64_t)split.row_blocks * S::kWarps, kPage);
    gfirst = (S::kMma ? p.group_cum : p.row_cum)[gi] + ((int64_t)g * gs.blocks + rb) * gt;
    gw = worker_of(group_units, gfirst, gworkers);
    gn = (int)(worker_of(group_units, gfirst + gt - 1, gworkers) - gw) + 1;
  }
  if (rt > 0) {
    rworkers = workers_for(split.row_units, (int64_t)split.row_blocks * S::kWarps, kPage);
    rfirst = p.row_cum[(S::kMma ? 0 : p.groups) + b] + (int64_t)g * rt;
    rw = worker_of(split.row_units, rfirst, rworkers);
    rn = (int)(worker_of(split.row_units, rfirst + rt - 1, rworkers) - rw) + 1;
  }
  if (gs.n <= gs.lo && rn == 1) return;      // finished by its worker
  float acc[kCols];
#pragma unroll
  for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
  float m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int i0 = 0; i0 < gn + rn; i0 += 32) {
    const int i = i0 + lane, n = min(gn + rn - i0, 32);
    RowPart part = {nullptr, nullptr, nullptr};
    float mw = -INFINITY, lw = 0.f;
    if (lane < n) {
      const bool shared = i < gn;
      if ((shared ? gn : rn) == 1) {
        part = whole_of(p, shared, row);
      } else {
        const int64_t w = shared ? gw + i : rw + (i - gn), U = shared ? group_units : split.row_units;
        const int64_t slot = 2 * w + (worker_begin(U, w, shared ? gworkers : rworkers) >= (shared ? gfirst : rfirst) ? 0 : 1);
        const int block = shared ? kRowBlock : WarpTree<D>::kRows, r = shared ? R - rb * kRowBlock : h - g * p.G;
        float* at = (shared && S::kMma ? p.group_parts : p.row_parts) + slot * (int64_t)(block * (D + 2));
        part = {at + r * D, at + block * D + r, at + block * (D + 1) + r};
      }
      mw = __ldcg(part.m);
      lw = __ldcg(part.l);
    }
    // A part that saw nothing has the maximum -inf, O = 0 and the sum 0 (or NaN, from a NaN score): weight 1.
    float top = fmaxf(m, mw);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float keep = m == -INFINITY ? 1.f : fast_exp2(m - top), f = mw == -INFINITY ? 1.f : fast_exp2(mw - top);
    float sum = lane < n ? lw * f : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    l = l * keep + sum;
    m = top;
#pragma unroll
    for (int j = 0; j < kCols; ++j) acc[j] *= keep;
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
      const float fk = __shfl_sync(0xffffffffu, f, k);
      const float* o = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(part.o), k)) + lane * kCols;
      float v[kCols];
      if constexpr (kCols == 2) {
        const float2 a = __ldcg(reinterpret_cast<const float2*>(o));
        v[0] = a.x; v[1] = a.y;
      } else {
#pragma unroll
        for (int j = 0; j < kCols; j += 4) {
          const float4 a = __ldcg(reinterpret_cast<const float4*>(o + j));
          v[j] = a.x; v[j + 1] = a.y; v[j + 2] = a.z; v[j + 3] = a.w;
        }
      }
#pragma unroll
      for (int j = 0; j < kCols; ++j) acc[j] += v[j] * fk;
    }
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  uint32_t w[kCols / 2];
#pragma unroll
  for (int j = 0; j < kCols; j += 2) w[j / 2] = pack_bf16(acc[j] * inv, acc[j + 1] * inv);
  __nv_bfloat16* out = p.out + row * D + lane * kCols;
#pragma unroll
  for (int j = 0; j < kCols / 2; ++j) reinterpret_cast<uint32_t*>(out)[j] = w[j];
  if (p.lse && lane == 0) p.lse[row] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : l == 0.f ? -INFINITY : l;
}

}  // namespace opw_tree
