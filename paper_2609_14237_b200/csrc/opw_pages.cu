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

// Pages and places of the new tokens of ragged requests.  One cluster:
//   rows named twice          every block, in bits of its own shared memory
//   row starts                every block scans the requests' tokens
//   entries without a page    each block looks at its share of the requests' table entries and counts
//   pages dealt               the counts meet through shared memory; every block scans them
//   table, counts, places of the rows   all threads of the cluster, a page or a row each, whose request is found by bisection
// Nothing is written before the cluster barrier behind the counts, so no block sees a table that is half changed.  It is a chain of round
// trips (requests, entries, list, counts) and barriers.  1000 decodes and 24 prompts of together 31000 tokens 14 us (with a warp per long request
// instead of a thread per page 22).
// One block instead of a cluster of eight where there are few requests and no more for a thread to do than a row, or without maps a page (what they
// add is known on the device only; a table's whole rows is what there may be).  Us in one block and in eight, the release of the dealt pages included:
// with maps 64 and 256 decodes 7.6, 8.7 and 8.3, 9.3; 256 requests of 32 tokens 11.4, 9.9; 8 of 1024 14.4, 9.4; without maps 64 decodes
// 7.4, 8.5; 8, 64 and 256 prompts of 8000 tokens 27, 11, then 106, 29 and 223, 94.
constexpr int kExtendBlocks = 8, kExtendFew = 256, kExtendThreads = 1024, kExtendMax = 8192, kExtendRows = 1 << 18;
constexpr int kLongPages = 4;              // entries that a thread looks at by itself; beyond, its warp does
struct ExtendParams {
  const int32_t* rows;
  const int32_t* old_lens;
  const int32_t* new_tokens;
  int32_t* table;
  int32_t* refs;
  const int32_t* free_list;
  const int32_t* free_count;
  const int32_t* free_begin;
  int32_t* free_end;
  int32_t* row_starts;
  int32_t* new_lens;
  int32_t* seq;
  int32_t* slots;
  uint32_t* status;
  int64_t num_pages, max_list;
  int32_t n, num_rows, max_pages, max_rows;
};
size_t extend_smem(int n, int num_rows) { return (size_t)(2 * ((num_rows + 31) / 32) + 4 * n + 2) * 4; }

template <int kBlocks>
__global__ void __launch_bounds__(kExtendThreads, 1) extend_kernel(const ExtendParams p) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ int32_t extend_s[];
  __shared__ int64_t wsum[kExtendThreads / 32];
  __shared__ int32_t given_s;
  const int bits = (p.num_rows + 31) / 32, n = p.n;
  uint32_t* once = reinterpret_cast<uint32_t*>(extend_s);        // rows that are named, and named twice
  uint32_t* twice = once + bits;
  int32_t* need = extend_s + 2 * bits;                            // pages a request lacks, -1 if it is refused or idle
  int32_t* entry = need + n;                                      // its first entry without a page; -2 - entry where others behind it have one
  int32_t* before = entry + n;                                    // pages that the requests before it lack
  int32_t* start = before + n;                                    // [n + 1] its first row
  const int rank = (int)cluster.block_rank(), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  for (int i = tid; i < 2 * bits; i += kExtendThreads) once[i] = 0u;
  const int per = (n + kExtendThreads - 1) / kExtendThreads, f0 = min(tid * per, n), f1 = min(f0 + per, n);   // requests this thread scans
  // exclusive prefix over the threads of one value each; `all`: the sum
  auto scan = [&](int64_t v, int64_t& all) -> int64_t {
    int64_t incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) wsum[warp] = incl;
    __syncthreads();
    if (warp == 0) {
      int64_t w = wsum[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
      }
      wsum[lane] = w;
    }
    __syncthreads();
    const int64_t front = (warp ? wsum[warp - 1] : 0) + incl - v;
    all = wsum[31];
    __syncthreads();
    return front;
  };
  const int64_t count = min((int64_t)*p.free_count, p.max_list), begin = p.free_begin ? max(*p.free_begin, 0) : 0;
  int64_t tokens = 0, all_tokens;
  for (int f = f0; f < f1; ++f) tokens += max(p.new_tokens[f], 0);
  if (tid == 0) given_s = 0;
  int64_t at = scan(tokens, all_tokens);                          // (its barriers also close the clearing of the bits)
  const int64_t room = p.max_rows >= 0 ? p.max_rows : INT32_MAX;
  for (int f = f0; f < f1; ++f) {
    const int32_t row = p.rows[f];
    if (row >= 0 && row < p.num_rows) {
      const uint32_t bit = 1u << (row & 31);
      if (atomicOr(once + (row >> 5), bit) & bit) atomicOr(twice + (row >> 5), bit);
    }
    start[f] = (int32_t)min(at, room);
    at += max(p.new_tokens[f], 0);
    before[f] = at > room;                                        // do its rows not fit?
  }
  if (tid == 0) start[n] = (int32_t)min(all_tokens, room);
  __syncthreads();

  // a thread per request of this block's share; long ones by the warp
  const int s0 = (int)((int64_t)n * rank / kBlocks), s1 = (int)((int64_t)n * (rank + 1) / kBlocks);
  for (int g0 = s0 + warp * 32; g0 < s1; g0 += kExtendThreads) {
    const int f = g0 + lane;
    int32_t row = -1, c = 0, first = 0, end = 0, lacks = -1, hole = INT32_MAX;   // hole: the first entry without a page
    bool bad = false;
    if (f < s1) {
      row = p.rows[f];
      c = p.old_lens[f];
      const int32_t m = p.new_tokens[f];
      if (row >= 0) {
        bad = row >= p.num_rows || (twice[row >> 5] >> (row & 31) & 1u) || c < 0 || m < 0 ||
              (int64_t)c + m > min((int64_t)p.max_pages * kPage, (int64_t)INT32_MAX) || before[f] != 0;
        if (!bad) {
          lacks = 0;
          if (m > 0) {
            first = c / kPage;
            end = (c + m - 1) / kPage + 1;
          }
        }
      }
    }
    auto look = [&](int32_t id, int32_t c, int32_t i, bool& wrong) -> int {   // does entry i, which holds id, lack a page?
      if (id < 0) {
        wrong |= i == c / kPage && c % kPage != 0;                // the tokens in it are gone
        return 1;
      }
      wrong |= id >= p.num_pages || p.refs[id] != 1;              // tokens must not be written to a page that others hold
      return 0;
    };
    if (end - first <= kLongPages) {
      int32_t id[kLongPages];
#pragma unroll
      for (int k = 0; k < kLongPages; ++k) id[k] = first + k < end ? p.table[(int64_t)row * p.max_pages + first + k] : 0;
#pragma unroll
      for (int k = 0; k < kLongPages; ++k)
        if (first + k < end && look(id[k], c, first + k, bad)) {
          ++lacks;
          hole = min(hole, first + k);
        }
    }
    uint32_t rest = __ballot_sync(0xffffffffu, end - first > kLongPages);
    for (; rest; rest &= rest - 1) {
      const int who = __ffs(rest) - 1;
      const int32_t r = __shfl_sync(0xffffffffu, row, who), cc = __shfl_sync(0xffffffffu, c, who);
      const int32_t a = __shfl_sync(0xffffffffu, first, who), e = __shfl_sync(0xffffffffu, end, who);
      const int32_t* entries = p.table + (int64_t)r * p.max_pages;
      int32_t sum = 0, least = INT32_MAX;
      bool wrong = false;
      for (int i0 = a; i0 < e; i0 += 4 * 32) {
        int32_t id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = i0 + 32 * k + lane;
          id[k] = i < e ? entries[i] : 0;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = i0 + 32 * k + lane;
          if (i < e && look(id[k], cc, i, wrong)) {
            ++sum;
            least = min(least, i);
          }
        }
      }
      sum = __reduce_add_sync(0xffffffffu, sum);
      least = __reduce_min_sync(0xffffffffu, least);
      wrong = __any_sync(0xffffffffu, wrong);
      if (lane == who) {
        lacks = sum;
        hole = least;
        bad = wrong;
      }
    }
    if (bad) {
      lacks = -1;
      atomicOr(p.status, kErrBadPage);
    }
    if (f < s1) {
      need[f] = lacks;
      entry[f] = lacks <= 0 ? 0 : end - hole == lacks ? hole : -2 - hole;
    }
  }
  cluster.sync();
  for (int f = tid; f < n; f += kExtendThreads) {                 // the other blocks' counts
    int r = (int)((int64_t)f * kBlocks / n);
    while (f >= (int)((int64_t)n * (r + 1) / kBlocks)) ++r;
    while (f < (int)((int64_t)n * r / kBlocks)) --r;
    if (r != rank) {
      need[f] = *cluster.map_shared_rank(need + f, r);
      entry[f] = *cluster.map_shared_rank(entry + f, r);
    }
  }
  cluster.sync();                                                 // (nobody leaves, or changes the table, while its counts are read)
  int64_t pages = 0, all_pages;
  for (int f = f0; f < f1; ++f) pages += max(need[f], 0);
  at = scan(pages, all_pages);
  // what is dealt out is a prefix of the list: up to the end of the last request that it is long enough for
  const int64_t avail = max(count - begin, (int64_t)0);
  int32_t mine = 0;
  for (int f = f0; f < f1; ++f) {
    const int32_t k = max(need[f], 0);
    before[f] = (int32_t)min(at, (int64_t)INT32_MAX);
    at += k;
    if (k > 0 && at <= avail) mine = (int32_t)at;
  }
  mine = __reduce_max_sync(0xffffffffu, mine);
  if (lane == 0 && mine > 0) atomicMax(&given_s, mine);
  __syncthreads();
  const int32_t given = given_s;
  auto served = [&](int f) { return need[f] == 0 || (need[f] > 0 && (int64_t)before[f] + need[f] <= given); };

  const int all = kBlocks * kExtendThreads, gt = rank * kExtendThreads + tid;
  auto deal = [&](int32_t* to, int64_t k) {                       // the k-th page from where dealing begins
    const int32_t id = p.free_list[begin + k];
    if (id < 0 || id >= p.num_pages || atomicCAS(p.refs + id, 0, 1) != 0) atomicOr(p.status, kErrBadPage);
    else *to = id;
  };
  auto request_of = [&](const int32_t* from, int32_t x) {         // the last request f with from[f] <= x
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (from[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
  };
  // (Counters of pages and rows have no sign: the ends are below 2^31, and the next of a thread's may lie beyond it.)
  for (uint32_t k = gt; k < (uint32_t)given; k += all) {          // (requests that lack nothing lie before the one found)
    const int f = request_of(before, (int32_t)k);
    if (entry[f] >= 0) deal(p.table + (int64_t)p.rows[f] * p.max_pages + entry[f] + ((int32_t)k - before[f]), k);
  }
  for (int g0 = gt - lane; g0 < n; g0 += all) {
    const int f = g0 + lane;
    bool holes = false;
    if (f < n) {
      const int32_t c = p.old_lens[f];
      if (p.row_starts) p.row_starts[f] = start[f];
      if (p.new_lens) p.new_lens[f] = served(f) ? c + p.new_tokens[f] : c;
      holes = need[f] > 0 && entry[f] < 0 && served(f);
    }
    uint32_t rest = __ballot_sync(0xffffffffu, holes);
    for (; rest; rest &= rest - 1) {                              // pages here and there: the warp walks them
      const int h = g0 + __ffs(rest) - 1;
      int32_t* entries = p.table + (int64_t)p.rows[h] * p.max_pages;
      const int end = (p.old_lens[h] + p.new_tokens[h] - 1) / kPage + 1;
      int32_t k = before[h];
      for (int i0 = -2 - entry[h]; i0 < end; i0 += 32) {
        const int i = i0 + lane;
        const bool wants = i < end && entries[i] < 0;
        const uint32_t who_wants = __ballot_sync(0xffffffffu, wants);
        if (wants) deal(entries + i, k + __popc(who_wants & ((1u << lane) - 1u)));
        k += __popc(who_wants);
      }
    }
  }
  if (gt == 0) {
    if (p.row_starts) p.row_starts[n] = start[n];
    if (p.free_end) *p.free_end = (int32_t)(begin + given);
  }
  // eight rows in a row a thread (one where there are few): one bisection, then along the requests; what is read of them is read side by side
  const bool wide = ((uintptr_t)p.seq | (uintptr_t)p.slots) % 16 == 0;
  if (kBlocks == 1 || p.max_rows <= all) {                        // (one block is never given more)
    if (gt < p.max_rows) {
      const int f = gt < start[n] ? request_of(start, gt) : n;
      const bool live = f < n && served(f);
      p.seq[gt] = live ? p.rows[f] : -1;
      p.slots[gt] = live ? p.old_lens[f] + (gt - start[f]) : -1;
    }
    return;
  }
  const uint32_t placed = (uint32_t)start[n], max_rows = (uint32_t)p.max_rows;
  for (uint32_t r0 = 8 * gt; r0 < max_rows; r0 += 8 * all) {
    int32_t seq[8], slot[8];
    int f = r0 < placed ? request_of(start, (int32_t)r0) : n;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      while (f < n && r0 + i >= (uint32_t)start[f + 1]) ++f;
      const bool live = f < n && served(f);
      seq[i] = live ? f : -1;
      slot[i] = live ? (int32_t)(r0 + i) - start[f] : -1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (seq[i] >= 0) {
        slot[i] += p.old_lens[seq[i]];
        seq[i] = p.rows[seq[i]];
      }
    if (wide && r0 + 8 <= max_rows) {
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        *reinterpret_cast<int4*>(p.seq + r0 + i) = make_int4(seq[i], seq[i + 1], seq[i + 2], seq[i + 3]);
        *reinterpret_cast<int4*>(p.slots + r0 + i) = make_int4(slot[i], slot[i + 1], slot[i + 2], slot[i + 3]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + i < max_rows) {
          p.seq[r0 + i] = seq[i];
          p.slots[r0 + i] = slot[i];
        }
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

extern "C" opw_status_t opw_kv_extend(opw_attn_stage_t* stage, int32_t n, const int32_t* rows, const int32_t* old_lens,
                                      const int32_t* new_tokens, int32_t num_rows, int32_t* page_table, int32_t* refcounts,
                                      int64_t num_pages, const int32_t* free_list, int64_t max_list, const int32_t* free_count,
                                      const int32_t* free_begin, int32_t* free_end, int32_t* row_starts, int32_t* new_lens,
                                      int32_t max_rows, int32_t* seq, int32_t* slots, void* cuda_stream) {
  if (!stage || n < 0 || num_rows < 1 || num_pages < 1 || num_pages > INT32_MAX || max_list < 0 || max_list > INT32_MAX || max_rows < -1)
    return OPW_ERR_INVALID_ARG;
  if ((seq == nullptr) != (slots == nullptr) || (seq ? max_rows < 0 : max_rows > 0)) return OPW_ERR_INVALID_ARG;
  if (!free_count || (max_list > 0 && !free_list) || (n > 0 && (!rows || !old_lens || !new_tokens || !page_table || !refcounts)))
    return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)rows | (uintptr_t)old_lens | (uintptr_t)new_tokens | (uintptr_t)page_table | (uintptr_t)refcounts | (uintptr_t)free_list |
       (uintptr_t)free_count | (uintptr_t)free_begin | (uintptr_t)free_end | (uintptr_t)row_starts | (uintptr_t)new_lens | (uintptr_t)seq |
       (uintptr_t)slots) % 4)
    return OPW_ERR_INVALID_ARG;
  const opw_stage_view v = opw_view_of(stage);
  if (n > opw_pages::kExtendMax || num_rows > opw_pages::kExtendRows) return OPW_ERR_CAPACITY;
  // what is written must not meet what other blocks still read, nor each other
  const size_t each = (size_t)n * 4, map = max_rows > 0 ? (size_t)max_rows * 4 : 0;
  const struct { const void* at; size_t bytes; } ins[] = {{rows, each}, {old_lens, each}, {new_tokens, each}, {free_list, (size_t)max_list * 4}, {free_count, 4}};
  const struct { const void* at; size_t bytes; } outs[] = {{page_table, (size_t)num_rows * v.max_pages * 4}, {refcounts, (size_t)num_pages * 4},
                                                           {free_end, 4}, {row_starts, each + 4}, {new_lens, each}, {seq, map}, {slots, map}};
  constexpr int kOuts = sizeof(outs) / sizeof(outs[0]);
  for (int i = 0; i < kOuts; ++i) {
    if (!outs[i].at || outs[i].bytes == 0) continue;
    auto meets = [&](const void* in, size_t bytes) { return in && bytes && opw_overlap(outs[i].at, outs[i].bytes, in, bytes); };
    for (const auto& in : ins)
      if (meets(in.at, in.bytes)) return OPW_ERR_INVALID_ARG;
    if (outs[i].at != free_begin && meets(free_begin, 4)) return OPW_ERR_INVALID_ARG;
    if (outs[i].at == free_begin && outs[i].at != free_end) return OPW_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (meets(outs[j].at, outs[j].bytes)) return OPW_ERR_INVALID_ARG;
  }
  opw_pages::ExtendParams p;
  p.rows = rows;
  p.old_lens = old_lens;
  p.new_tokens = new_tokens;
  p.table = page_table;
  p.refs = refcounts;
  p.free_list = free_list;
  p.free_count = free_count;
  p.free_begin = free_begin;
  p.free_end = free_end;
  p.row_starts = row_starts;
  p.new_lens = new_lens;
  p.seq = seq;
  p.slots = slots;
  p.status = v.status;
  p.num_pages = num_pages;
  p.max_list = max_list;
  p.n = n;
  p.num_rows = num_rows;
  p.max_pages = v.max_pages;
  p.max_rows = max_rows;
  opw_device_guard guard(v.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  const size_t smem = opw_pages::extend_smem(n, num_rows);
  const bool few = n <= opw_pages::kExtendFew && (max_rows >= 0 ? max_rows : (int64_t)n * v.max_pages) <= opw_pages::kExtendThreads;
  auto launch = [&](auto kernel, int blocks) {
    if (smem > 40 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)opw_pages::extend_smem(opw_pages::kExtendMax, opw_pages::kExtendRows));
      if (e != cudaSuccess) return e;
    }
    return opw_launch(kernel, dim3(blocks), dim3(opw_pages::kExtendThreads), smem, static_cast<cudaStream_t>(cuda_stream), v.pdl, blocks, p);
  };
  const cudaError_t e = few ? launch(opw_pages::extend_kernel<1>, 1) : launch(opw_pages::extend_kernel<opw_pages::kExtendBlocks>, opw_pages::kExtendBlocks);
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  *v.launches += 1;
  return OPW_OK;
}
