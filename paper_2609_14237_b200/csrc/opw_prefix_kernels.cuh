// Device code of decode attention behind shared prefixes (include/opw_prefix.h).
//
// The shared keys of a group are a problem of their own: its rows are the group's members x G query heads of a kv head, all of which see
// (almost) the same keys, so that a key tile that is read once serves up to 256 rows on the tensor cores.  The keys behind the prefix are
// the ordinary split-KV decode problem, G rows a sequence.  Both are the problems that the kernels of tree attention take
// (opw_tree_kernels.cuh), solved in ONE launch: some blocks run the tensor-core kernel over the groups, the others a warp kernel over the
// sequences, divided by what either costs.  The parts of a row's result -- one per worker that had keys of it -- are left in fp32
// and merged by a second kernel.
//
// Measured, 32/8 heads of 128, in a replayed graph.  16 groups of 16 behind 16k, 16 to 2048 keys of their own: 369 us for 2.16 GB, 5.9 TB/s (90 % of
// what a copy reaches); either half ends where the other does to 10 %.  64 behind 8k, 1 to 1024 of their own: 44.5 us, floor 26: of it 3 us of
// survey, 6 of merge, and 35 in which 48 blocks take 2 x 128 rows of 128 tiles a head (0.8 us a tile while the whole chip reads, 0.6 of compute)
// and 100 the 17000 pages of the rows.  The two launched one after the other had no share of each other's idle unit, and a launch more.  What it
// took from 62 us: shares that count the ends of short rows (tail of 27 us gone), rows of one sequence with the products the other way
// round (row_body), whole numbers of blocks a segment, partials stored in whole pieces.
#pragma once

#include "opw_tree_mma.cuh"

namespace opw_tree {

constexpr int kMaxPrefixBatch = 2048, kMaxPrefixGroups = 1024;
// What things cost, for equal shares, in halves of the time of a page of a sequence's own keys (0.2 us a block, 1.4 us a warp where the whole
// chip reads): a tile of 64 shared keys with up to 128 rows and with 256 (0.6 and 1.1 us of compute; four pages' bytes); in tiles, the
// ends of a segment of shared keys (queries in, a partial out); in pages, the ends of a row.
constexpr int kPage2 = 2, kNarrowTile = 11, kWideTile = 16, kGroupEnds = 8, kRowEnds = 2;

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
  float* partials;       // this problem's partial slots; units before each of its entities, for the merge
  int64_t* cum;
  float* whole;          // [2][batch * Hq][D] outputs, [2][batch * Hq] maxima, sums: rows that one worker has seen all of
  GroupInfo* info;
  PrefixSplit* split;
  uint32_t* status;
  int64_t num_pages;
  int32_t batch, groups, Hq, Hkv, G, D, max_pages, window;
  int32_t lead, all;     // this problem's entities: [0, lead) are groups, those behind rows
  int32_t stages;        // places of a warp's ring, where warps take the keys
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
  Span s = no_span();                        // (a length that was cut is recorded by survey_groups)
  if (n <= 0) return s;
  s.tree = 1;
  s.ctx = s.n = n;
  s.lo = min(max(shared, window_start(p, n)), n);
  s.table_row = s.first_row = b;
  return s;
}

// What the kernels' bodies are given, as a kernel parameter (a copy would live in registers that they do not have).  Short rows and groups are many ends and few keys: shares of equal work count the ends (64 rows of 1 to 1024 own keys: the
// last warp was done 27 us after the average one without).
template <int kEnds_>
struct PrefixProblem : PrefixParams {
  static constexpr int kEnds = kEnds_, kLeastPages = kEnds_ + 1;
  static constexpr bool kMerged = true;      // it takes groups only, and all of their rows go to the merge
};
// What every block finds out for itself, at the beginning of its shared memory: the groups' infos, then starts.
__device__ __forceinline__ GroupInfo* infos() {
  extern __shared__ __align__(128) unsigned char smem[];
  return reinterpret_cast<GroupInfo*>(smem);
}
__device__ __forceinline__ int32_t* starts_of(const PrefixParams& p) { return reinterpret_cast<int32_t*>(infos() + p.groups + 1); }
template <int kEnds>
__device__ __forceinline__ int entities(const PrefixProblem<kEnds>& p) { return p.all; }
template <int kEnds>
__device__ __forceinline__ Span span_of(const PrefixProblem<kEnds>& p, int e, int row_block) {
  const int32_t* starts = starts_of(p);
  if (e < p.lead) return group_span(p, infos()[e], starts[e], starts[e + 1], row_block);
  const int b = e - p.lead;
  return row_span(p, infos()[group_of(starts, p.groups, b)].shared, b);
}
static __device__ __noinline__ RowView prefix_row_view(const int32_t* len, int32_t max_pages, int32_t window, int32_t end, int32_t lo) {
  const int32_t n = (int32_t)min((int64_t)max(*len, 0), min((int64_t)max_pages * kPage, (int64_t)INT32_MAX));
  RowView v;
  v.bits = 0ull;
  v.ctx = INT32_MAX;                         // (nothing is drafted)
  v.end = min(n, end);
  v.lo = max(lo, window > 0 ? n - window : 0);
  return v;
}
template <int kEnds>
__device__ __forceinline__ RowView row_view(const PrefixProblem<kEnds>& p, int, const Span& s, int node) {
  return prefix_row_view(p.lens + s.first_row + node, p.max_pages, p.window, s.n, s.tree > 1 ? 0 : s.lo);
}
template <int kEnds>
__device__ __forceinline__ int32_t window_border(const PrefixProblem<kEnds>& p, int e, const Span& s, int) {
  return e < p.lead ? max(s.lo, window_start(p, infos()[e].longest)) : s.lo;
}
// A group of one active row shares nothing: a span of two rows and more is a group's.
template <int kEnds>
__device__ __forceinline__ bool finished_at_once(const PrefixProblem<kEnds>& p, const Span& s) {
  if (s.tree > 1) return false;
  const int32_t* starts = starts_of(p);
  const int g = group_of(starts, p.groups, s.first_row);
  const Span shared = group_span(p, infos()[g], starts[g], starts[g + 1], 1);
  return shared.n <= shared.lo;
}
__device__ __forceinline__ RowPart whole_of(const PrefixParams& p, bool shared, int64_t row) {
  const int64_t rows = (int64_t)p.batch * p.Hq, r = (shared ? 0 : rows) + row;
  float* ml = p.whole + 2 * rows * p.D;
  return {p.whole + r * p.D, ml + r, ml + 2 * rows + r};
}
template <int kEnds>
__device__ __forceinline__ RowPart whole_row(const PrefixProblem<kEnds>& p, const Span& s, int64_t row) { return whole_of(p, s.tree > 1, row); }

// Sums over the block of four values each.
template <int kWarps>
__device__ __forceinline__ void block_sums(int64_t (&v)[4]) {
  __shared__ int64_t part[kWarps][4];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < 4; ++k) part[warp][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[k] = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v[k] += part[w][k];
  }
}

__device__ __forceinline__ uint32_t transposed(uint32_t x) {      // of the warp's 8 x 8 matrix of 16 bits
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// The warp kernel (warp_body) for up to eight rows that see the same keys, a sequence's own: the products the other way round, keys and
// dimensions along the 16 of an m16n8k16, rows along the 8,
//     S^T (16 keys x 8) = K Q^T,   O^T (16 dimensions x 8) += V^T P^T,
// which takes half the instructions of a tile whose upper eight rows are empty.  Hidden keys are hidden from all rows, so that clearing their
// values is all that a masked page needs.  The ring has as many places a warp as fit beside the tables (p.stages).
// 100 SMs read 48 GB/s each this way beside 48 that take groups, 1.4 us a page and warp; with the tile of 16 rows 44.
template <int D, int kWarps, class Problem>
__device__ __forceinline__ void row_body(const Problem& p, unsigned char* smem, const int64_t* cum, int block, int blocks) {
  constexpr int KS = D / 16, ROWB = D * 2, TILE = WarpTree<D>::kTile, kEnds = Problem::kEnds;
  constexpr uint32_t kFirst = 1u << 28, kLast = 1u << 29, kBad = 1u << 30, kNone = 1u << 31, kPageBits = kFirst - 1;   // kNone: no tile
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, stages = p.stages;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + (size_t)kWarps * stages * TILE);
  const int batch = entities(p);
  const int64_t U = cum[batch];
  const int64_t workers = workers_for<Problem>(U, (int64_t)blocks * kWarps, kPage), worker = (int64_t)warp * blocks + block;
  const uint32_t ring = smem_u32(smem + (size_t)warp * stages * TILE);
  const uint32_t bar0 = smem_u32(bars + warp * stages);
  if (lane == 0) {
    for (int s = 0; s < stages; ++s) mbar_init(bar0 + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  __syncwarp();
  const bool idle = worker >= workers;
  const int64_t u0 = idle ? U : worker_begin(U, worker, workers), u1 = idle ? U : worker_begin(U, worker + 1, workers);
  struct Desc { int32_t tile; uint32_t page; };
  auto describe = [&](int64_t u) -> Desc {
    Desc d = {0, 0u};
    if (u >= u1) return d;
    const int b = find_sequence(cum, batch, u);
    const Span s = span_of(p, b, WarpTree<D>::kRows);
    const int32_t cnt = tiles_of(s, kPage);
    const int64_t rem = u - cum[b];
    const int32_t g = (int32_t)(rem / (cnt + kEnds)), i = (int32_t)(rem - (int64_t)g * (cnt + kEnds)) - kEnds;
    if (i < 0) {
      d.page = kNone;
      return d;
    }
    const int32_t lp = s.lo / kPage + i;
    int64_t pid = p.page_table[(int64_t)s.table_row * p.max_pages + lp];
    d.page = (uint32_t)lp | (i == 0 ? kFirst : 0u) | (i == cnt - 1 ? kLast : 0u);
    if (pid < 0 || pid >= p.num_pages) {      // never dereference a bad page: mask it out
      atomicOr(p.status, kErrBadPage);
      pid = 0;
      d.page |= kBad;
    }
    d.tile = (int32_t)(pid * p.Hkv + g);
    return d;
  };
  int64_t wbase = u0;
  Desc wa = describe(u0 + lane), wb = describe(u0 + 32 + lane);
  pdl_launch_dependents();
  pdl_wait();                                 // up to here only this step's lengths, starts and the page table were read
  if (block == 0)
    for (int i = threadIdx.x; i <= batch; i += kWarps * 32) p.cum[i] = cum[i];

  const uint64_t policy = l2_evict_first_policy();
  auto issue = [&](int64_t u, int slot) {
    const int rel = (int)(u - wbase);
    const int32_t ta = __shfl_sync(0xffffffffu, wa.tile, rel & 31), tb = __shfl_sync(0xffffffffu, wb.tile, rel & 31);
    const uint32_t pa = __shfl_sync(0xffffffffu, wa.page, rel & 31), pb = __shfl_sync(0xffffffffu, wb.page, rel & 31);
    if (lane == 0) {
      const uint32_t bar = bar0 + 8 * slot;
      if ((rel < 32 ? pa : pb) & kNone) {     // nothing to copy: the place's barrier completes all the same
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
      } else {
        mbar_expect_tx(bar, TILE);
        bulk_load(ring + slot * TILE, reinterpret_cast<const unsigned char*>(p.pool) + (int64_t)(rel < 32 ? ta : tb) * TILE, TILE, bar, policy);
      }
    }
  };
  int inflight = 0;
  for (int s = 0; s < stages && u0 + s < u1; ++s) { issue(u0 + s, s); ++inflight; }

  const int mi = lane >> 3, rr = lane & 7, qrow = lane >> 2, qcol = (lane & 3) * 2;
  const uint32_t k_off = (uint32_t)((rr + 8 * (mi & 1)) * ROWB), v_off = (uint32_t)(kPage * ROWB + (rr + 8 * (mi >> 1)) * ROWB);
  uint32_t qb[KS][2];
  float o[KS][4], mx[2], l[2];                // of rows qcol and qcol + 1: dimensions 16 j + qrow and + 8
  int b = 0, g = 0;
  Span sp = no_span();
  bool from_first = false, on_first_row = true, failed = false, fresh = true;
  int slot = 0;
  uint32_t phase = 0;

  for (int64_t u = u0; u < u1; ++u) {
    if (u - wbase == 32) {
      wbase += 32;
      wa = wb;
      wb = describe(wbase + 32 + lane);
    }
    const uint32_t page = __shfl_sync(0xffffffffu, wa.page, (int)(u - wbase));
    const bool none = page & kNone, last = page & kLast;
    if (!none && (fresh || (page & kFirst))) {   // a new row: its queries, an empty state
      fresh = false;
      from_first = page & kFirst;
      b = find_sequence(cum, batch, u);
      sp = span_of(p, b, WarpTree<D>::kRows);
      g = (int)((u - cum[b]) / (tiles_of(sp, kPage) + kEnds));
      const __nv_bfloat16* q = p.q + ((int64_t)sp.first_row * p.Hq + (int64_t)g * p.G + qrow) * D + qcol;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qb[ks][0] = qrow < p.G ? *reinterpret_cast<const uint32_t*>(q + ks * 16) : 0u;
        qb[ks][1] = qrow < p.G ? *reinterpret_cast<const uint32_t*>(q + ks * 16 + 8) : 0u;
      }
      mx[0] = mx[1] = -INFINITY;
      l[0] = l[1] = 0.f;
#pragma unroll
      for (int j = 0; j < KS; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    }
    if (!mbar_wait(bar0 + 8 * slot, phase)) { failed = true; break; }
    --inflight;
    if (!none) {
      const uint32_t tile = ring + slot * TILE;
      const int32_t key0 = (int32_t)(page & kPageBits) * kPage;
      uint32_t seen = ~0u;                    // bit i: key key0 + i
      if (key0 + kPage > sp.n || key0 < sp.lo || (page & kBad)) {
        const int32_t end = min(sp.n - key0, kPage), begin = max(sp.lo - key0, 0);
        seen = (page & kBad) ? 0u : ((1u << max(end, 0)) - 1u) & ~((1u << min(begin, kPage)) - 1u);
        for (int i = lane; i < kPage * (ROWB / 16); i += 32) {   // what nobody sees holds anything: its values are cleared
          const int t = i / (ROWB / 16);
          if (!((seen >> t) & 1u))
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(tile + (uint32_t)(kPage * ROWB + i * 16)), "r"(0u) : "memory");
        }
        __syncwarp();
      }
      // ---- S^T = K Q^T ----
      float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};   // (two chains)
#pragma unroll
      for (int ks = 0; ks < KS; ks += 2) {
        uint32_t r0, r1, r2, r3;
        ldsm_x4(tile + k_off + (((2 * ks + (mi >> 1)) ^ rr) << 4), r0, r1, r2, r3);
        mma_bf16(x, r0, r1, r2, r3, qb[ks][0], qb[ks][1]);
        ldsm_x4(tile + k_off + (((2 * ks + 2 + (mi >> 1)) ^ rr) << 4), r0, r1, r2, r3);
        mma_bf16(y, r0, r1, r2, r3, qb[ks + 1][0], qb[ks + 1][1]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {           // keys qrow (e < 2) and qrow + 8 of rows qcol + (e & 1)
        x[e] = (x[e] + y[e]) * p.scale_log2e;
        if (!((seen >> (qrow + 8 * (e >> 1))) & 1u)) x[e] = -INFINITY;
      }
      // ---- online softmax (base 2) ----
      float top[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float t = fmaxf(x[r], x[2 + r]);
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
        top[r] = fmaxf(mx[r], fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16)));
      }
      if (__any_sync(0xffffffffu, top[0] > mx[0] || top[1] > mx[1])) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float a = mx[r] == -INFINITY ? 0.f : fast_exp2(mx[r] - top[r]);   // nothing summed yet: all zero
          l[r] *= a;
#pragma unroll
          for (int j = 0; j < KS; ++j) { o[j][r] *= a; o[j][2 + r] *= a; }
          mx[r] = top[r];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float m = mx[e & 1] == -INFINITY ? 0.f : mx[e & 1];
        x[e] = fast_exp2(x[e] - m);
        l[e & 1] += x[e];
      }
      // P is rounded to bf16 for the product, the sum is not: the roundings average out over the keys
      const uint32_t b0 = transposed(pack_bf16(x[0], x[1])), b1 = transposed(pack_bf16(x[2], x[3]));
      // ---- O^T += V^T P^T ----
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        uint32_t r0, r1, r2, r3;
        ldsm_x4_t(tile + v_off + (((2 * j + (mi & 1)) ^ rr) << 4), r0, r1, r2, r3);
        mma_bf16(o[j], r0, r1, r2, r3, b0, b1);
      }
      __syncwarp();
    }
    if (u + stages < u1) {
      if (lane == 0 && !none) fence_proxy_async();
      issue(u + stages, slot);
      ++inflight;
    }
    if (++slot == stages) { slot = 0; phase ^= 1u; }

    if (!none && (last || u == u1 - 1)) {     // the row, or this worker's part of it, is done
      const bool complete = from_first && last, finish = complete && finished_at_once(p, sp);
      float* pb = p.partials + (2 * worker + (on_first_row ? 0 : 1)) * (int64_t)(WarpTree<D>::kRows * (D + 2));
      float inv[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 4);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 8);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 16);
        inv[r] = l[r] > 0.f ? 1.f / l[r] : l[r] == 0.f ? 0.f : l[r];
      }
      const int64_t row0 = (int64_t)sp.first_row * p.Hq + (int64_t)g * p.G;
      if (finish) {
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          const uint32_t w0 = transposed(pack_bf16(o[j][0] * inv[0], o[j][1] * inv[1]));
          const uint32_t w1 = transposed(pack_bf16(o[j][2] * inv[0], o[j][3] * inv[1]));
          if (qrow < p.G) {
            __nv_bfloat16* out = p.out + (row0 + qrow) * D + 16 * j + qcol;
            *reinterpret_cast<uint32_t*>(out) = w0;
            *reinterpret_cast<uint32_t*>(out + 8) = w1;
          }
        }
        if (p.lse && lane < 4)
#pragma unroll
          for (int r = 0; r < 2; ++r)
            if (qcol + r < p.G) p.lse[row0 + qcol + r] = l[r] > 0.f ? (mx[r] + log2f(l[r])) * 0.6931471805599453f : l[r] == 0.f ? -INFINITY : l[r];
      } else {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int n = qcol + r;
          if (n >= p.G) continue;
          const RowPart part = complete ? whole_row(p, sp, row0 + n)
                                        : RowPart{pb + n * D, pb + WarpTree<D>::kRows * D + n, pb + WarpTree<D>::kRows * (D + 1) + n};
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            part.o[16 * j + qrow] = o[j][r];
            part.o[16 * j + 8 + qrow] = o[j][2 + r];
          }
          if (lane < 4) {
            *part.m = mx[r];
            *part.l = l[r];
          }
        }
      }
      on_first_row = false;
    }
  }
  if (failed) {
    // A copy did not arrive in time: record it, then give every copy still in flight a bounded chance to land.
    if (lane == 0) atomicOr(p.status, kErrTimeout);
    for (int i = 0; i < inflight; ++i) {
      (void)mbar_wait(bar0 + 8 * slot, phase);
      if (++slot == stages) { slot = 0; phase ^= 1u; }
    }
  }
}

// Fills infos and starts.  Starts that do not ascend from 0 to the batch share nothing and are recorded, as are lengths beyond the table (here,
// where a block looks at every row: there may be no block for the rows' own keys).
__device__ __forceinline__ void survey_groups(const PrefixParams& p) {
  int32_t* first = starts_of(p);
  GroupInfo* info = infos();
  auto length = [&](int b) {
    const int32_t n = length_of(p, b);
    if (blockIdx.x == 0 && p.lens[b] > n) atomicOr(p.status, kErrBadPage);
    return n;
  };
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
    const int32_t n = b < p.batch ? length(b) : 0;
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

// How many of the blocks take the groups.  Both counts of units include the ends.  Shares of a few equal segments are taken a whole number a
// segment, a few blocks more or, where that costs no more than the ends of the segments that shares would meet two of, less.
// masked: tiles that windows hide in part, which take about twice the time.
__device__ __forceinline__ int group_blocks(int64_t group_units, int64_t segments, int64_t masked, int64_t row_units, int blocks, bool wide) {
  if (group_units == 0) return 0;
  const int64_t a = (group_units + masked) * (wide ? kWideTile : kNarrowTile), b = row_units * kPage2;
  int64_t n = (a * blocks + (a + b) / 2) / (a + b);
  n = min(n, group_units);
  if (row_units > 0) n = min(n, (int64_t)blocks - 1);
  n = max(n, (int64_t)1);
  const int64_t each = n / segments, more = (each + 1) * segments;
  if (more <= n + n / 8 && 8 * (blocks - more) >= 7 * (blocks - n)) n = more;
  else if (each > 0 && (group_units / segments + each - 1) / each <= (group_units + n - 1) / n + kGroupEnds) n = each * segments;
  return (int)n;
}

enum PrefixMode { kPrefixWarp, kPrefixNarrow, kPrefixWide };   // the groups by the warp kernel, or by the tensor-core one with 128 or 256 rows

// kHigh: more than eight query heads a kv head, so that a row's own keys want the upper half of the warp kernel's tile.
template <int D, int kMode, bool kHigh>
struct PrefixSmem {
  static constexpr bool kMma = kMode != kPrefixWarp;
  using Mma = MmaTree<D == 256 ? 128 : D, kMode == kPrefixWide>;
  // Warps that take keys by themselves: of the tensor-core kernel's 384 threads eight, who get the registers of the other four
  static constexpr int kWarps = kMma ? 8 : D == 64 ? 12 : D == 128 ? 8 : 5;
  static constexpr int kThreads = kMma ? kMmaThreads : kWarps * 32;
  static constexpr int kMaxStages = kMma && !kHigh ? (D == 64 ? 6 : 3) : WarpTree<D>::kStages;
  __host__ __device__ static constexpr size_t ring(int stages) { return (size_t)kWarps * stages * (WarpTree<D>::kTile + 8); }
  static constexpr size_t kTiles = kMma ? 1024 + (size_t)Mma::kPieces * Mma::kPiece + (size_t)Mma::kQTiles * Mma::kQTile : 0;
  // blocks with groups need units for those only, the others for the rows (and, without the tensor cores, for both)
  __host__ __device__ static constexpr size_t tables(int groups) { return (size_t)(groups + 1) * 16 + (size_t)((groups + 4) / 4) * 16; }
  static size_t bytes(int batch, int groups, int stages) {
    const size_t rows = ring(stages) + (size_t)(batch + (kMma ? 0 : groups) + 1) * 8, tiles = kTiles + (size_t)(groups + 1) * 8;
    return tables(groups) + (kMma && tiles > rows ? tiles : rows);
  }
  static constexpr size_t kMost = 227 * 1024 - 4608;              // the kernels' static shared memory is below 4.5 KB
  static int stages(int batch, int groups) {
    int n = kMaxStages;
    while (n > WarpTree<D>::kStages && bytes(batch, groups, n) > kMost) --n;
    return n;
  }
};

// Shared memory: group infos, starts, then the tiles of the block's role and behind them its entities' units.
template <int D, int kMode, bool kHigh>
__global__ void __launch_bounds__(PrefixSmem<D, kMode, kHigh>::kThreads, 1) prefix_kernel(
    const __grid_constant__ CUtensorMap map, const __grid_constant__ PrefixProblem<kGroupEnds> groups, const __grid_constant__ PrefixProblem<kRowEnds> p) {
  using S = PrefixSmem<D, kMode, kHigh>;
  const GroupInfo* info = infos();
  const int32_t* first = starts_of(p);
  unsigned char* room = reinterpret_cast<unsigned char*>(infos()) + S::tables(p.groups);
  survey_groups(p);

  int group_n = 0;
  int64_t group_units = 0, row_units = 0;
  if (S::kMma) {
    constexpr int kRowBlock = kMode == kPrefixWide ? 256 : 128;
    int64_t sums[4] = {0, 0, 0, 0};          // units of the groups, their segments, units of the rows, masked tiles
    for (int g = threadIdx.x; g < p.groups; g += S::kThreads) {
      const Span s = group_span(p, info[g], first[g], first[g + 1], kRowBlock);
      const int32_t t = tiles_of(s, kMmaKeys), n = t > 0 ? s.blocks * p.Hkv : 0;
      sums[0] += (int64_t)(t + kGroupEnds) * n;
      sums[1] += n;
      if (p.window > 0) sums[3] += (int64_t)(max(min(window_start(p, info[g].longest), s.n) - s.lo, 0) / kMmaKeys) * n;
    }
    for (int r = threadIdx.x; r < p.batch; r += S::kThreads) {
      const int32_t t = tiles_of(row_span(p, info[group_of(first, p.groups, r)].shared, r), kPage);
      if (t > 0) sums[2] += (int64_t)(t + kRowEnds) * p.Hkv;
    }
    block_sums<S::kThreads / 32>(sums);
    group_units = sums[0];
    row_units = sums[2];
    group_n = group_blocks(group_units, sums[1], sums[3], row_units, gridDim.x, kMode == kPrefixWide);
  }
  const bool grouped = (int)blockIdx.x < group_n;
  if (grouped) {
    if constexpr (S::kMma)
      mma_body<D, kMode == kPrefixWide>(map, groups, room, reinterpret_cast<int64_t*>(room + S::kTiles), blockIdx.x, group_n);
  } else {
    int64_t* cum = reinterpret_cast<int64_t*>(room + S::ring(p.stages));
    scan_units(p, cum, WarpTree<D>::kRows, kPage, false);
    if (!S::kMma) row_units = cum[p.all];
    if (S::kThreads == S::kWarps * 32 || threadIdx.x < S::kWarps * 32) {
      // 256 x 224 + 128 x 56 = 256 x 200 + 128 x 104 = 384 x 168
      if constexpr (S::kMma) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kHigh ? 224 : 200));
      if constexpr (S::kMma && !kHigh) row_body<D, S::kWarps>(p, room, cum, blockIdx.x - group_n, gridDim.x - group_n);
      else warp_body<D, S::kWarps>(p, room, cum, blockIdx.x - group_n, gridDim.x - group_n);
    } else {
      if constexpr (S::kMma) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHigh ? 56 : 104));
      pdl_launch_dependents();
      pdl_wait();
    }
  }
  if (blockIdx.x == 0) {
    for (int g = threadIdx.x; g < p.groups; g += S::kThreads) p.info[g] = info[g];
    if (threadIdx.x == 0) *p.split = {group_units, row_units, group_n, (int32_t)gridDim.x - group_n};
  }
}

// worker_of and worker_begin; nearly always a division of 32 bits (of 64 it takes about 100 instructions, and there are six in a row)
__device__ __forceinline__ int64_t worker_at(int64_t U, int64_t u, int64_t workers) {
  const int64_t x = (u + 1) * workers - 1;
  return (x | U) <= UINT32_MAX ? (int64_t)((uint32_t)x / (uint32_t)U) : x / U;
}
__device__ __forceinline__ int64_t begin_at(int64_t U, int64_t worker, int64_t workers) {
  const int64_t x = U * worker;
  return x <= UINT32_MAX ? (int64_t)((uint32_t)x / (uint32_t)workers) : x / workers;
}

// kSplit warps per row of the output, 1 or all four of a block (few rows: each warp a quarter of the parts, which meet in shared memory); a lane
// has D / 32 neighbouring columns.  The row's parts are looked up 32 at a time, a lane each (whose slot, maximum and sum), then added up
// column by column.
constexpr int kPrefixCombineThreads = 128;
template <int D, int kMode, bool kHigh, int kSplit>
__global__ void __launch_bounds__(kPrefixCombineThreads) prefix_combine_kernel(const __grid_constant__ PrefixParams groups,
                                                                            const __grid_constant__ PrefixParams p) {
  using S = PrefixSmem<D, kMode, kHigh>;
  using Rows = PrefixProblem<kRowEnds>;
  using Groups = PrefixProblem<S::kMma ? kGroupEnds : kRowEnds>;
  constexpr int kCols = D / 32, kRowBlock = kMode == kPrefixWide ? 256 : kMode == kPrefixNarrow ? 128 : WarpTree<D>::kRows;
  constexpr int kGroupKeys = S::kMma ? kMmaKeys : kPage;
  __shared__ float acc_s[kSplit > 1 ? kSplit : 1][kSplit > 1 ? D : 1];
  __shared__ float2 ml_s[kSplit];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, piece = kSplit > 1 ? warp : 0;
  const int64_t row = kSplit > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (kPrefixCombineThreads / 32) + warp;
  if (row >= (int64_t)p.batch * p.Hq) return;
  const int b = (int)(row / p.Hq), h = (int)(row - (int64_t)b * p.Hq), g = h / p.G;
  const int gi = group_of(p.starts, p.groups, b);
  const int32_t start = p.starts[gi], end = p.starts[gi + 1];
  const bool active = length_of(p, b) > 0;
  pdl_launch_dependents();
  pdl_wait();                                // up to here only the lengths and starts were read
  const GroupInfo info = p.info[gi];         // (all that the looking up needs in one round trip)
  const PrefixSplit split = *p.split;
  const int64_t gcum = (S::kMma ? groups : p).cum[gi], rcum = p.cum[p.lead + b];
  const Span gs = group_span(p, info, start, end, kRowBlock), rs = row_span(p, info.shared, b);
  const int32_t gt = active ? tiles_of(gs, kGroupKeys) : 0, rt = tiles_of(rs, kPage);
  // the workers that had keys of this row (gfirst, rfirst: where its segment begins, with its ends)
  int64_t gw = 0, rw = 0, gfirst = 0, rfirst = 0, gworkers = 1, rworkers = 1;
  int gn = 0, rn = 0;                        // parts
  const int R = (b - start) * p.G + (h - g * p.G), rb = R / kRowBlock;
  const int64_t group_units = S::kMma ? split.group_units : split.row_units;
  if (gt > 0) {
    gworkers = workers_for<Groups>(group_units, S::kMma ? split.group_blocks : (int64_t)split.row_blocks * S::kWarps, kGroupKeys);
    gfirst = gcum + ((int64_t)g * gs.blocks + rb) * (gt + Groups::kEnds);
    gw = worker_at(group_units, gfirst + Groups::kEnds, gworkers);
    gn = (int)(worker_at(group_units, gfirst + Groups::kEnds + gt - 1, gworkers) - gw) + 1;
  }
  if (rt > 0) {
    rworkers = workers_for<Rows>(split.row_units, (int64_t)split.row_blocks * S::kWarps, kPage);
    rfirst = rcum + (int64_t)g * (rt + kRowEnds);
    rw = worker_at(split.row_units, rfirst + kRowEnds, rworkers);
    rn = (int)(worker_at(split.row_units, rfirst + kRowEnds + rt - 1, rworkers) - rw) + 1;
  }
  if (gs.n <= gs.lo && rn == 1) return;      // finished by its worker
  float acc[kCols];
#pragma unroll
  for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
  float m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int i0 = 0; i0 < gn + rn; i0 += 32 * kSplit) {
    const int i = i0 + lane * kSplit + piece, n = min((gn + rn - i0 - piece + kSplit - 1) / kSplit, 32);   // (n <= 0: none for this warp)
    RowPart part = {nullptr, nullptr, nullptr};
    float mw = -INFINITY, lw = 0.f;
    if (lane < n) {
      const bool shared = i < gn;
      if ((shared ? gn : rn) == 1) {
        part = whole_of(p, shared, row);
      } else {
        const int64_t w = shared ? gw + i : rw + (i - gn), U = shared ? group_units : split.row_units;
        const int64_t slot = 2 * w + (begin_at(U, w, shared ? gworkers : rworkers) >= (shared ? gfirst : rfirst) ? 0 : 1);
        const int block = shared ? kRowBlock : WarpTree<D>::kRows, r = shared ? R - rb * kRowBlock : h - g * p.G;
        float* at = (shared && S::kMma ? groups : p).partials + slot * (int64_t)(block * (D + 2));
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
#pragma unroll (kSplit > 1 ? 8 : 4)
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
  if constexpr (kSplit > 1) {
#pragma unroll
    for (int j = 0; j < kCols; ++j) acc_s[piece][lane * kCols + j] = acc[j];
    if (lane == 0) ml_s[piece] = make_float2(m, l);
    __syncthreads();
    if (piece != 0) return;
    float top = m;
#pragma unroll
    for (int k = 1; k < kSplit; ++k) top = fmaxf(top, ml_s[k].x);
    float a = m == -INFINITY ? 1.f : fast_exp2(m - top);          // (weights as above)
    l *= a;
#pragma unroll
    for (int j = 0; j < kCols; ++j) acc[j] *= a;
#pragma unroll
    for (int k = 1; k < kSplit; ++k) {
      a = ml_s[k].x == -INFINITY ? 1.f : fast_exp2(ml_s[k].x - top);
      l += ml_s[k].y * a;
#pragma unroll
      for (int j = 0; j < kCols; ++j) acc[j] += acc_s[k][lane * kCols + j] * a;
    }
    m = top;
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
