// Device code of tree attention (include/opw_draft.h): the queries of a sequence's drafted tokens, nodes x G rows per kv head,
// over the paged cache.  sm_100a only.
//
// Row r of (sequence b, kv head g) is node r / G with query head g * G + r % G.  Rows are taken in blocks, and a
// "unit" is one (b, g, row block, key tile); units are ordered that way and the U units of a launch are cut into equal
// contiguous shares, one per worker.  A share meets at most two row blocks that it does not cover completely, its first
// and its last; those leave (unnormalised O, maximum, sum) in the worker's two partial slots and are merged by
// tree_combine_kernel, the others are finished on the spot.  Shares follow from the lengths alone: deterministic.
//
// A key is hidden from a row by the window (position), by the row's mask word (drafted keys) or by the end of the sequence.
// Only tiles that hold such a key take the masked path.  There a hidden score becomes -inf, so that whatever the
// key row holds has no effect; and since 0 * NaN is NaN in the product with V, cached values that are not finite are
// taken out of the tile and added, by plain arithmetic, to the rows that do see them.
#pragma once

#define OPW_NAMESPACE opw_tree
#define OPW_NO_STAGE_KERNELS
#include "opw_kernels.cuh"

namespace opw_tree {

constexpr int kMaxTreeBatch = 4096;

struct TreeParams {
  static constexpr int kEnds = 0;        // units that a segment (entity, kv head, row block) counts for besides its tiles, in front of them
  static constexpr int kLeastPages = 4;  // units a worker has at least where they are pages
  static constexpr bool kMerged = false; // the tensor-core kernel finishes the rows that it has seen all of
  const __nv_bfloat16* pool;
  const __nv_bfloat16* q;
  const uint64_t* mask;
  const int32_t* positions;
  const int32_t* ctx_lens;
  const int32_t* tree_lens;
  const int32_t* page_table;
  __nv_bfloat16* out;
  float* lse;
  float* partials;       // [workers * 2][row_block * (D + 2)]: O rows, then maxima, then sums
  int64_t* cum;          // [batch + 1] units before sequence b (written by block 0 for the combine)
  uint32_t* status;
  int64_t num_pages;
  int32_t batch, nodes, Hq, Hkv, G, max_pages, window;
  float scale_log2e;
};

// What of sequence b takes part: context length, tree size, first key that any node can see, end, row blocks; the row of the page table
// and the first row of the queries.
struct Span {
  int32_t ctx, tree, lo, n, blocks, table_row, first_row;
  bool cut;              // the lengths did not fit the table or the call: recorded as OPW_ERR_BAD_PAGE
};
__device__ __forceinline__ Span span_of(const TreeParams& p, int b, int row_block) {
  Span s;
  s.ctx = p.ctx_lens[b];
  s.tree = p.tree_lens[b];
  s.table_row = b;
  s.first_row = b * p.nodes;
  s.cut = false;
  if (s.ctx < 0 || s.tree <= 0) { s.ctx = s.tree = s.lo = s.n = s.blocks = 0; return s; }
  if (s.tree > p.nodes) { s.tree = p.nodes; s.cut = true; }
  int64_t n = (int64_t)s.ctx + s.tree;
  const int64_t cap = (int64_t)p.max_pages * kPage;
  if (n > cap) { n = cap; s.cut = true; }
  s.n = (int32_t)n;
  s.lo = (p.window > 0 && s.ctx >= p.window) ? s.ctx - p.window + 1 : 0;
  if (s.lo > s.n) s.lo = s.n;
  s.blocks = (s.tree * p.G + row_block - 1) / row_block;
  return s;
}
// key tiles of `keys` keys (a multiple of the page) that cover [lo, n), counted from lo's page
__device__ __forceinline__ int32_t tiles_of(const Span& s, int keys) {
  if (s.n <= s.lo) return 0;
  const int32_t first = s.lo / kPage * kPage;
  return (s.n - first + keys - 1) / keys;
}

// The kernels below take any problem that answers as this one does: `entities` of it, each with its span, whose row r is node r / G with
// query head g * G + r % G, what a row of it sees, and where a row's result goes.  (Attention behind shared prefixes is the other one.)
__device__ __forceinline__ int entities(const TreeParams& p) { return p.batch; }
// Where a row's unnormalised output, maximum and sum go.
struct RowPart {
  float *o, *m, *l;
};
__device__ __forceinline__ RowPart whole_row(const TreeParams&, const Span&, int64_t) { return {nullptr, nullptr, nullptr}; }   // (never asked)
// Is a row that one worker has seen all of finished there and then, as opposed to left in fp32 for a merge?
__device__ __forceinline__ bool finished_at_once(const TreeParams&, const Span&) { return true; }

// Units before each entity, for the whole block: cum[0..entities] in shared memory.  `record`: note lengths that were cut (one block does).
template <class Problem>
__device__ __forceinline__ void scan_units(const Problem& p, int64_t* cum, int row_block, int keys, bool record) {
  __shared__ int64_t wsum[32];
  __shared__ int64_t carry;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) carry = 0;
  __syncthreads();
  const int batch = entities(p);
  for (int base = 0; base < batch; base += blockDim.x) {
    const int b = base + threadIdx.x;
    int64_t cnt = 0;
    if (b < batch) {
      const Span s = span_of(p, b, row_block);
      if (s.cut && record) atomicOr(p.status, kErrBadPage);
      const int32_t tiles = tiles_of(s, keys);
      cnt = tiles > 0 ? (int64_t)(tiles + Problem::kEnds) * s.blocks * p.Hkv : 0;
    }
    int64_t incl = cnt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) wsum[warp] = incl;
    __syncthreads();
    int64_t before = carry;
    for (int w = 0; w < warp; ++w) before += wsum[w];
    if (b < batch) cum[b] = before + incl - cnt;
    __syncthreads();
    if (threadIdx.x == blockDim.x - 1) carry = before + incl;
    __syncthreads();
  }
  if (threadIdx.x == 0) cum[batch] = carry;
  __syncthreads();
}
// How many of the launched workers share U units: never more than there are units, and with single pages as units (a warp each) at least
// four of them per worker -- a short step would otherwise leave a partial per page (63 of them at 1000 keys: the
// combine took 110 us).
template <class Problem>
__device__ __forceinline__ int64_t workers_for(int64_t U, int64_t launched, int keys) {
  const int64_t most = keys == kPage ? U / Problem::kLeastPages : U;
  return most < 1 ? 1 : most < launched ? most : launched;
}
// the sequence that holds unit u < cum[batch]
__device__ __forceinline__ int find_sequence(const int64_t* cum, int batch, int64_t u) {
  int lo = 0, hi = batch;                    // cum[lo] <= u < cum[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cum[mid] <= u) lo = mid; else hi = mid;
  }
  return lo;
}

// Which keys a row sees.
struct RowView {
  uint64_t bits;         // drafted keys that exist, those outside the window taken out
  int32_t lo, end, ctx;  // context keys [lo, end); drafted key m is key ctx + m
};
// (Called, not inlined, as all of the rare paths here: the kernels' loops have to stay in the instruction cache.  With everything
// inlined the tensor-core kernel had 180 KB of code and spent most of its time fetching it.)
static __device__ __noinline__ RowView row_view(const uint64_t* mask, const int32_t* pos, int32_t window, int32_t ctx, int32_t n, int32_t tree,
                                         int node) {
  RowView v;
  v.bits = mask[node];
  v.lo = 0;
  v.ctx = ctx;
  v.end = min(ctx, n);
  const int32_t drafted = n - ctx;
  if (drafted < 64) v.bits &= drafted > 0 ? (1ull << drafted) - 1ull : 0ull;
  if (window > 0) {
    v.lo = max(max(pos[node], ctx) - window + 1, 0);       // (at least 0: lo - base must not pass 32 bits)
#pragma unroll 1
    for (int m = 0; m < tree; ++m)
      if (max(pos[m], ctx) < v.lo) v.bits &= ~(1ull << m);
  }
  return v;
}
__device__ __forceinline__ RowView row_view(const TreeParams& p, int b, const Span& s, int node) {
  return row_view(p.mask + (int64_t)b * p.nodes, p.positions + (int64_t)b * p.nodes, p.window, s.ctx, s.n, s.tree, node);
}
// The bounded wait with its loop out of line.
static __device__ __noinline__ bool mbar_wait_loop(uint32_t bar, uint32_t parity) {
  const uint64_t t0 = global_timer_ns();
#pragma unroll 1
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (global_timer_ns() - t0 > kWaitLimitNs) return false;
  }
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
  return mbar_try_wait(bar, parity) || mbar_wait_loop(bar, parity);
}
// Bit i: the row sees key base + i, i < 32.
__device__ __forceinline__ uint32_t visible_word(const RowView& v, int32_t base) {
  auto ones = [](int32_t k) { return k >= 32 ? ~0u : (1u << max(k, 0)) - 1u; };
  uint32_t w = ones(v.end - base) & ~ones(v.lo - base);
  const int32_t o = v.ctx - base;
  if (o < 32 && o > -64) w |= o >= 0 ? (uint32_t)v.bits << o : (uint32_t)(v.bits >> -o);
  return w;
}
// The first context key that the window hides from no node (a whole warp asks).
__device__ __forceinline__ int32_t window_border(const TreeParams& p, int b, const Span& s, int lane) {
  if (p.window == 0) return 0;
  int32_t border = s.lo;
  const int32_t* pos = p.positions + (int64_t)b * p.nodes;
  for (int i = lane; i < s.tree; i += 32) border = max(border, max(pos[i], s.ctx) - p.window + 1);
  return __reduce_max_sync(0xffffffffu, border);
}
__device__ __forceinline__ bool any_not_finite(const uint4& w) {   // of eight bf16
  auto bad = [](uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; };
  return bad(w.x) || bad(w.y) || bad(w.z) || bad(w.w);
}
__device__ __forceinline__ float bf16_at(uint32_t addr) {
  uint16_t h;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(addr));
  return __uint_as_float((uint32_t)h << 16);
}

// ---------------------------------------------------------------------------------
// few rows: every warp streams its own units, as the stage's decode kernel does
// ---------------------------------------------------------------------------------
// A unit is one page, K and V of a head in one bulk copy; a row block is 16 rows, the accumulators of one mma.sync tile in registers.
// At these sizes the products are next to nothing (16 rows: 8 flops a byte) and the copy is what bounds it; a warp that
// waits for nobody else keeps the memory busy with two pages in flight each.  64 sequences of 1k to 4k keys, a tree of 2: 669 MB in 112 us,
// 6.0 TB/s, 91 % of what a copy reaches.  At head_dim 256 the accumulators take 128 registers more: 255 and a spill of 21 words stored and 17 loaded;
// a tree of 2 still runs at 5.0 TB/s, but a larger one reads its pages once per 16 rows (16 x 16k keys, 512 rows: 2385 us, floor 169).
template <int D>
struct WarpTree {
  static constexpr int kTile = 2 * kPage * D * 2;
  static constexpr int kRows = 16;
  static constexpr int kWarps = D == 64 ? 12 : D == 128 ? 8 : 6;
  static constexpr int kStages = 2;
  static size_t smem(int batch) {
    return (size_t)kWarps * kStages * kTile + (size_t)kWarps * kStages * 8 + (size_t)(batch + 1) * 8;
  }
};

// kWarps warps of a block take part; worker numbers go across the blocks first.  `block` of `blocks` are this problem's.  smem: the rings,
// then their barriers; cum: the entities' units (scan_units).
template <int D, int kWarps, class Problem>
__device__ __forceinline__ void warp_body(const Problem& p, unsigned char* smem, const int64_t* cum, int block, int blocks) {
  using C = WarpTree<D>;
  constexpr int kEnds = Problem::kEnds;
  constexpr int KS = D / 16, NT = D / 8, ROWB = D * 2, TILE = C::kTile;
  constexpr uint32_t kFirst = 1u << 28, kLast = 1u << 29, kBad = 1u << 30, kNone = 1u << 31, kPageBits = kFirst - 1;   // kNone: no tile
  const int warps = kWarps, stages = C::kStages;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + (size_t)warps * stages * TILE);
  const int batch = entities(p);
  const int64_t U = cum[batch];
  const int64_t workers = workers_for<Problem>(U, (int64_t)blocks * warps, kPage), worker = (int64_t)warp * blocks + block;
  const uint32_t ring = smem_u32(smem + (size_t)warp * stages * TILE);
  const uint32_t bar0 = smem_u32(bars + warp * stages);
  if (lane == 0) {
    for (int s = 0; s < stages; ++s) mbar_init(bar0 + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  __syncwarp();

  const bool idle = worker >= workers;         // (few units: the first workers are on different SMs)
  const int64_t u0 = idle ? U : worker_begin(U, worker, workers), u1 = idle ? U : worker_begin(U, worker + 1, workers);
  struct Desc { int32_t tile; uint32_t page; };
  auto describe = [&](int64_t u) -> Desc {
    Desc d = {0, 0u};
    if (u >= u1) return d;
    const int b = find_sequence(cum, batch, u);
    const Span s = span_of(p, b, C::kRows);
    const int32_t cnt = tiles_of(s, kPage);
    const int64_t rem = u - cum[b];
    const int32_t ri = (int32_t)(rem / (cnt + kEnds)), i = (int32_t)(rem - (int64_t)ri * (cnt + kEnds)) - kEnds, g = ri / s.blocks;
    if (kEnds > 0 && i < 0) {
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
  pdl_launch_dependents();                    // (as in the tensor-core kernel)
  pdl_wait();                                 // up to here only this step's lengths and the page table were read
  if (block == 0)
    for (int i = threadIdx.x; i <= batch; i += kWarps * 32) p.cum[i] = cum[i];

  const uint64_t policy = l2_evict_first_policy();
  auto issue = [&](int64_t u, int slot) {
    const int rel = (int)(u - wbase);
    const int32_t a = __shfl_sync(0xffffffffu, wa.tile, rel & 31), b = __shfl_sync(0xffffffffu, wb.tile, rel & 31);
    if (kEnds > 0) {
      const uint32_t pa = __shfl_sync(0xffffffffu, wa.page, rel & 31), pb = __shfl_sync(0xffffffffu, wb.page, rel & 31);
      if ((rel < 32 ? pa : pb) & kNone) {     // nothing to copy: the place's barrier completes all the same
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar0 + 8 * slot) : "memory");
        return;
      }
    }
    if (lane == 0) {
      const uint32_t bar = bar0 + 8 * slot;
      mbar_expect_tx(bar, TILE);
      bulk_load(ring + slot * TILE, reinterpret_cast<const unsigned char*>(p.pool) + (int64_t)(rel < 32 ? a : b) * TILE, TILE, bar,
                policy);
    }
  };
  int inflight = 0;
  for (int s = 0; s < stages && u0 + s < u1; ++s) { issue(u0 + s, s); ++inflight; }

  const int mi = lane >> 3, rr = lane & 7, qrow = lane >> 2, qcol = (lane & 3) * 2;
  const uint32_t k_off = (uint32_t)((rr + 8 * (mi >> 1)) * ROWB), v_off = (uint32_t)(kPage * ROWB + (rr + 8 * (mi & 1)) * ROWB);
  uint32_t qa[KS][4];
  float o[NT][4], mx[2], l[2];
  int b = 0, g = 0, rb = 0, rows = 0;
  int32_t border = 0;
  Span sp = {0, 0, 0, 0, 1, 0, 0, false};
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
    const bool last = page & kLast;
    if (kEnds > 0 && (page & kNone)) {
      if (!mbar_wait(bar0 + 8 * slot, phase)) { failed = true; break; }
      --inflight;
      if (u + stages < u1) {
        issue(u + stages, slot);
        ++inflight;
      }
      if (++slot == stages) { slot = 0; phase ^= 1u; }
      continue;
    }
    if (fresh || (page & kFirst)) {           // a new row block: its queries, an empty state
      fresh = false;
      from_first = page & kFirst;
      b = find_sequence(cum, batch, u);
      sp = span_of(p, b, C::kRows);
      const int32_t ri = (int32_t)((u - cum[b]) / (tiles_of(sp, kPage) + kEnds));
      g = ri / sp.blocks;
      rb = ri - g * sp.blocks;
      rows = sp.tree * p.G - rb * C::kRows;   // of this block; may exceed it
      border = window_border(p, b, sp, lane);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = h * 8 + qrow;
        const bool live = r < rows;
        const int R = rb * C::kRows + r, node = R / p.G;
        const __nv_bfloat16* qb = p.q + (((int64_t)sp.first_row + node) * p.Hq + (int64_t)g * p.G + (R - node * p.G)) * D + qcol;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          qa[ks][h] = live ? *reinterpret_cast<const uint32_t*>(qb + ks * 16) : 0u;
          qa[ks][2 + h] = live ? *reinterpret_cast<const uint32_t*>(qb + ks * 16 + 8) : 0u;
        }
        mx[h] = -INFINITY;
        l[h] = 0.f;
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) o[nt][0] = o[nt][1] = o[nt][2] = o[nt][3] = 0.f;
    }
    if (!mbar_wait(bar0 + 8 * slot, phase)) { failed = true; break; }
    --inflight;
    const uint32_t tile = ring + slot * TILE;
    const int32_t key0 = (int32_t)(page & kPageBits) * kPage;

    // ---- S = Q K^T ----
    float x[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) x[nt][0] = x[nt][1] = x[nt][2] = x[nt][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint32_t r0, r1, r2, r3;
      ldsm_x4(tile + k_off + ((((2 * ks + (mi & 1)) ^ rr)) << 4), r0, r1, r2, r3);
      mma_bf16(x[0], qa[ks][0], qa[ks][1], qa[ks][2], qa[ks][3], r0, r1);
      mma_bf16(x[1], qa[ks][0], qa[ks][1], qa[ks][2], qa[ks][3], r2, r3);
    }
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[nt][e] *= p.scale_log2e;

    const bool masked = key0 + kPage > sp.ctx || key0 < border || (page & kBad);
    uint32_t odd = 0;                         // keys of the tile whose values are not all finite
    if (masked) {
      // Slots nobody may read (behind the end, before the window, a bad page) hold anything: their values are
      // cleared.  The others are searched for values that are not finite.
      for (int t = 0; t < kPage; ++t) {
        const bool dead = key0 + t >= sp.n || key0 + t < sp.lo || (page & kBad);
        bool found = false;
        for (int off = lane * 16; off < ROWB; off += 512) {
          const uint32_t a = tile + (uint32_t)(kPage * ROWB + t * ROWB + off);
          uint4 w = make_uint4(0u, 0u, 0u, 0u);
          if (!dead) {
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(a));
            found |= any_not_finite(w);
          } else {
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(a), "r"(0u) : "memory");
          }
        }
        if (__any_sync(0xffffffffu, found)) odd |= 1u << t;
      }
      __syncwarp();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = h * 8 + qrow;
        if (r < rows && !(page & kBad)) {
          const uint32_t seen = visible_word(row_view(p, b, sp, (rb * C::kRows + r) / p.G), key0);
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (!((seen >> (nt * 8 + qcol + e)) & 1u)) x[nt][2 * h + e] = -INFINITY;
        } else {
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) x[nt][2 * h] = x[nt][2 * h + 1] = -INFINITY;
        }
      }
    }

    // ---- online softmax (base 2) ----
    uint32_t pa[4];
    float top[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float t = fmaxf(fmaxf(x[0][2 * h], x[0][2 * h + 1]), fmaxf(x[1][2 * h], x[1][2 * h + 1]));
      t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
      top[h] = fmaxf(mx[h], fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2)));
    }
    if (__any_sync(0xffffffffu, top[0] > mx[0] || top[1] > mx[1])) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float a = mx[h] == -INFINITY ? 0.f : fast_exp2(mx[h] - top[h]);   // nothing summed yet: all zero
        l[h] *= a;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) { o[nt][2 * h] *= a; o[nt][2 * h + 1] *= a; }
        mx[h] = top[h];
      }
    }
    float pr[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float m = mx[h] == -INFINITY ? 0.f : mx[h];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          pr[nt][2 * h + e] = fast_exp2(x[nt][2 * h + e] - m);
          l[h] += pr[nt][2 * h + e];
        }
    }
    // P is rounded to bf16 for the product, the sum is not: the roundings average out over the keys
    pa[0] = pack_bf16(pr[0][0], pr[0][1]);
    pa[1] = pack_bf16(pr[0][2], pr[0][3]);
    pa[2] = pack_bf16(pr[1][0], pr[1][1]);
    pa[3] = pack_bf16(pr[1][2], pr[1][3]);
    if (odd) {                                // rare: values that are not finite leave the tile
      for (uint32_t rest = odd; rest; rest &= rest - 1) {
        const int t = __ffs(rest) - 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = h * 8 + qrow;
          if (r >= rows || !((visible_word(row_view(p, b, sp, (rb * C::kRows + r) / p.G), key0) >> t) & 1u)) continue;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t a = tile + (uint32_t)(kPage * ROWB + t * ROWB + ((nt ^ (t & 7)) << 4) + (qcol + e) * 2);
              const float val = bf16_at(a);
              if (!isfinite(val)) o[nt][2 * h + e] += val;
            }
        }
      }
      __syncwarp();
      for (uint32_t rest = odd; rest; rest &= rest - 1) {
        const int t = __ffs(rest) - 1;
        for (int off = lane * 2; off < ROWB; off += 64) {
          const uint32_t a = tile + (uint32_t)(kPage * ROWB + t * ROWB + off);
          if (!isfinite(bf16_at(a))) asm volatile("st.shared.u16 [%0], %1;" ::"r"(a), "h"((uint16_t)0) : "memory");
        }
      }
      __syncwarp();
    }
    // ---- O += P V ----
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      uint32_t r0, r1, r2, r3;
      ldsm_x4_t(tile + v_off + ((((2 * j + (mi >> 1)) ^ rr)) << 4), r0, r1, r2, r3);
      mma_bf16(o[2 * j], pa[0], pa[1], pa[2], pa[3], r0, r1);
      mma_bf16(o[2 * j + 1], pa[0], pa[1], pa[2], pa[3], r2, r3);
    }
    __syncwarp();
    if (u + stages < u1) {
      if (lane == 0) fence_proxy_async();
      issue(u + stages, slot);
      ++inflight;
    }
    if (++slot == stages) { slot = 0; phase ^= 1u; }

    if (last || u == u1 - 1) {                // the row block, or this worker's part of it, is done
      const bool complete = from_first && last, finish = complete && finished_at_once(p, sp);
      float* pb = p.partials + (2 * worker + (on_first_row ? 0 : 1)) * (int64_t)(C::kRows * (D + 2));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float t = l[h];
        t += __shfl_xor_sync(0xffffffffu, t, 1);
        t += __shfl_xor_sync(0xffffffffu, t, 2);
        const int r = h * 8 + qrow;
        if (r >= rows) continue;
        const int R = rb * C::kRows + r, node = R / p.G;
        const int64_t row = ((int64_t)sp.first_row + node) * p.Hq + (int64_t)g * p.G + (R - node * p.G);
        if (finish) {
          const float inv = t > 0.f ? 1.f / t : 0.f;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            *reinterpret_cast<uint32_t*>(p.out + row * D + nt * 8 + qcol) =
                pack_bf16(o[nt][2 * h] * inv, o[nt][2 * h + 1] * inv);
          if (p.lse && (lane & 3) == 0)
            p.lse[row] = t > 0.f ? (mx[h] + log2f(t)) * 0.6931471805599453f : t == 0.f ? -INFINITY : t;
        } else {
          const RowPart part = complete ? whole_row(p, sp, row) : RowPart{pb + r * D, pb + C::kRows * D + r, pb + C::kRows * (D + 1) + r};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            *reinterpret_cast<float2*>(part.o + nt * 8 + qcol) = make_float2(o[nt][2 * h], o[nt][2 * h + 1]);
          if ((lane & 3) == 0) {
            *part.m = mx[h];
            *part.l = t;
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

template <int D>
__global__ void __launch_bounds__(WarpTree<D>::kWarps * 32, 1) tree_warp_kernel(TreeParams p) {
  using C = WarpTree<D>;
  extern __shared__ __align__(128) unsigned char smem[];
  int64_t* cum = reinterpret_cast<int64_t*>(smem + (size_t)C::kWarps * C::kStages * (C::kTile + 8));
  scan_units(p, cum, C::kRows, kPage, blockIdx.x == 0);
  warp_body<D, C::kWarps>(p, smem, cum, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------------------------
// combine: merges the partials of row blocks that several workers share, and writes the rows that no worker has
// ---------------------------------------------------------------------------------
struct TreeCombineParams {
  TreeParams t;
  int32_t D, row_block, keys, max_blocks;    // max_blocks: row blocks of a full tree of `nodes`
  int64_t workers;
};
constexpr int kTreeCombineThreads = 256;

// grid (batch * Hkv * max_blocks, rows of a block / (32 / kGroups), D / (32 V)).  Eight threads own V * 32 columns of a row, every eighth
// float4 each, and walk the row's partials once, carrying (O, m, l) like an online softmax.  kGroups > 1, V = 1: few rows of many
// partials each, where the walk is a chain of L2 round trips -- the columns go to blocks of their own, the partials are dealt
// out to that many groups of threads, which meet in shared memory, and eight are in flight per thread.  (One sequence of 8000
// keys, 125 partials a row: 21 us with whole rows and four groups of two in flight, 19 us this way and on the tensor-core kernel.)
// It adds 4 us to a call of one short sequence and 6 to 64 trees of 8 (measured by leaving it out): a launch and its round trips.
template <int D, int kGroups, int V>
__global__ void __launch_bounds__(kTreeCombineThreads, V == 1 ? 1 : D == 256 ? 2 : 3) tree_combine_kernel(const TreeCombineParams c) {
  constexpr int kRows = 32 / kGroups, kDeep = V == 1 ? 8 : 2;     // partials in flight (four: two blocks an SM, chain of 4 11.8 us, now 11.5)
  const TreeParams& p = c.t;
  __shared__ int32_t slot_s[kTreeCombineThreads];
  __shared__ float4 acc_s[kGroups > 1 ? kTreeCombineThreads : 1][kGroups > 1 ? V : 1];
  __shared__ float2 ml_s[kGroups > 1 ? kTreeCombineThreads : 1];
  const int rb = blockIdx.x % c.max_blocks, bg = blockIdx.x / c.max_blocks, g = bg % p.Hkv, b = bg / p.Hkv;
  const Span s = span_of(p, b, c.row_block);
  const int live = s.tree * p.G;
  const int lane8 = (threadIdx.x & 7) + 8 * V * blockIdx.z, group = threadIdx.x / (8 * kRows);
  const int r = blockIdx.y * kRows + (threadIdx.x >> 3) % kRows, R = rb * c.row_block + r;   // row of the block, of (b, g)
  const int32_t cnt = tiles_of(s, c.keys);
  const int node = R / p.G;
  const int64_t row = ((int64_t)b * p.nodes + node) * p.Hq + (int64_t)g * p.G + (R - node * p.G);
  pdl_launch_dependents();
  pdl_wait();                                                    // up to here only the lengths were read
  const int64_t U = p.cum[p.batch], before = p.cum[b];
  if ((cnt == 0 || R >= live) && R < p.nodes * p.G && group == 0) {
    // a node that is not there (or a sequence without a key): zeros
#pragma unroll
    for (int j = 0; j < V; ++j) *reinterpret_cast<uint2*>(p.out + row * D + (lane8 + 8 * j) * 4) = make_uint2(0u, 0u);
    if (p.lse && lane8 == 0) p.lse[row] = -INFINITY;
  }
  if (cnt == 0 || rb * c.row_block + (int)blockIdx.y * kRows >= live) return;   // (the same for the whole block)
  const int64_t workers = workers_for<TreeParams>(U, c.workers, c.keys);
  const int64_t first = before + ((int64_t)g * s.blocks + rb) * cnt, end = first + cnt;
  const int64_t wf = worker_of(U, first, workers), wl = worker_of(U, end - 1, workers);
  if (wf == wl) return;                                          // finished by its worker
  const int64_t slot_floats = (int64_t)c.row_block * (D + 2);
  float4 acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  // A part that saw nothing has the maximum -inf, O = 0 and the sum 0 (or NaN, from a NaN score): weight 1.
  auto merge = [&](float mw, float lw, const float4* v) {
    const float top = fmaxf(m, mw), a = m == -INFINITY ? 1.f : fast_exp2(m - top), f = mw == -INFINITY ? 1.f : fast_exp2(mw - top);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      acc[j].x = acc[j].x * a + v[j].x * f; acc[j].y = acc[j].y * a + v[j].y * f;
      acc[j].z = acc[j].z * a + v[j].z * f; acc[j].w = acc[j].w * a + v[j].w * f;
    }
    l = l * a + lw * f;
    m = top;
  };
  const bool merges = R < live && r < c.row_block;
#pragma unroll 1
  for (int64_t w0 = wf; w0 <= wl; w0 += kTreeCombineThreads) {
    const int n = (int)min(wl - w0 + 1, (int64_t)kTreeCombineThreads);
    if ((int)threadIdx.x < n) {                                  // the partial slot of worker w for this block
      const int64_t w = w0 + threadIdx.x;                        // (no share is empty: there are at least as many units as workers)
      slot_s[threadIdx.x] = (int32_t)(2 * w + (worker_begin(U, w, workers) >= first ? 0 : 1));
    }
    __syncthreads();
    if (merges) {
#pragma unroll 1
      for (int i = group; i < n; i += kDeep * kGroups) {
        float4 v[kDeep][V];
        float mw[kDeep], lw[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
          const int k = i + u * kGroups;
          const float* q = p.partials + (int64_t)slot_s[k < n ? k : i] * slot_floats;
#pragma unroll
          for (int j = 0; j < V; ++j) v[u][j] = __ldcg(reinterpret_cast<const float4*>(q + r * D) + lane8 + 8 * j);
          mw[u] = __ldcg(q + c.row_block * D + r);
          lw[u] = __ldcg(q + c.row_block * (D + 1) + r);
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
          if (i + u * kGroups < n) merge(mw[u], lw[u], v[u]);
      }
    }
    __syncthreads();
  }
  if (kGroups > 1) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc_s[threadIdx.x][j] = acc[j];
    ml_s[threadIdx.x] = make_float2(m, l);
    __syncthreads();
    if (group != 0) return;
#pragma unroll 1
    for (int k = 1; k < kGroups; ++k) {                          // in group order: deterministic
      const int other = threadIdx.x + k * 8 * kRows;
      merge(ml_s[other].x, ml_s[other].y, acc_s[other]);
    }
  }
  if (!merges) return;
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    uint2 w2;
    w2.x = pack_bf16(acc[j].x * inv, acc[j].y * inv);
    w2.y = pack_bf16(acc[j].z * inv, acc[j].w * inv);
    *reinterpret_cast<uint2*>(p.out + row * D + (lane8 + 8 * j) * 4) = w2;
  }
  if (p.lse && lane8 == 0) p.lse[row] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : l == 0.f ? -INFINITY : l;
}

}  // namespace opw_tree
