// Verification of drafted tokens against the target's probabilities (include/opw_draft.h).
#include <cstdint>

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "opw_draft.h"
#include "opw_stage.h"
#include "opw_words.cuh"

namespace opw_verify {

namespace cg = cooperative_groups;
using opw_words::pdl_wait;

constexpr uint32_t kErrBadPage = 1u;      // bit of the stage's status word
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;         // (above 8 a cluster size has to be allowed)

struct Params {
  const void* target;
  const void* draft;
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* tree_lens;
  const float* uniforms;
  int32_t* path;
  int32_t* path_lens;
  int32_t* next_tokens;
  uint32_t* status;
  int64_t target_stride, draft_stride;
  int32_t nodes, vocab;
};

enum Draw { kAgain = OPW_DRAW_AGAIN, kDistinct = OPW_DRAW_DISTINCT, kCertain = OPW_DRAW_CERTAIN };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// A node's distribution after n of its branches were refused, without a division per token.  With R_0 = r_0 and C_0 = S_0 = 1,
//     R_{j+1} = max(R_j - c_j Q_j, 0),   c_j = C_j / S_j,   C_{j+1} = sum of R_{j+1},   r_j = R_j / C_j,   q_j = Q_j / S_j,
// and as max(max(x - a, 0) - b, 0) = max(x - a - b, 0) for a, b >= 0, nearly all of it is one number, a = the sum of the c_j:
//     kAgain     R = max(p - a q, 0)
//     kDistinct  the same, but for the refused tokens, whose R stays what their refusal left; S = the sum of q without them
//     kCertain   R = p, but for the refused tokens, whose R is max(R - C, 0)
// So a refusal costs a pass over the row for the new sum (kCertain: the first at a node only), and a token a product and a sum however many were
// refused.  kDistinct keeps the refused tokens in a list, kCertain those of all the node's children, and the passes leave the listed ones out: they
// may be all but 1e-20 of the sum (a sure drafter's likeliest token), so that the rest is added up by itself and never found by subtraction.
struct List {                             // each token once
  int32_t token[OPW_TREE_MAX_NODES];
  double r[OPW_TREE_MAX_NODES];           // its R
};
template <Draw kDraw>
__device__ __forceinline__ double left_of(float p, float q, double a) {
  const double r = (double)fmaxf(p, 0.f); // (negative and NaN: 0)
  return kDraw == kCertain ? r : fmax(fma(-a, (double)fmaxf(q, 0.f), r), 0.0);
}

template <bool X>
struct Flag {
  static constexpr bool value = X;
};

// The 16-byte word at token v of a row, 0 for what lies outside of the row.
template <typename T>
struct alignas(16) Word {
  static constexpr int kN = 16 / sizeof(T);
  T x[kN];
  __device__ __forceinline__ void load_inside(const T* row, int v) { *reinterpret_cast<uint4*>(x) = __ldg(reinterpret_cast<const uint4*>(row + v)); }
  __device__ __forceinline__ void load(const T* row, int v, int vocab, bool wide) {
    if (wide && v >= 0 && v + kN <= vocab) {
      load_inside(row, v);
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) x[i] = v + i >= 0 && v + i < vocab ? row[v + i] : T(0.f);
    }
  }
};

// A cluster per sequence; its blocks decide alike and share the rows of the vocabulary, a contiguous part a warp.
//
// What decides is scalar: the target's and the drafter's probability of each node's token, gathered at the start in one round trip.
// Only a refusal needs a row's sum, and the token that follows: the smallest v at which the running sum of R passes u * total.  The
// sums of the warps' parts say which part holds v, and its block reads that part again, a word a thread.
// All sums are in 64 bits, so that the token does not depend on how a row is split but for differences of 1e-16.
//
// Measured, fp32: a chain of 4 over 32000 tokens 6.4 us, 64 trees of 8 over 131072 30 to 31 (floor 7.7: 50 MB; bf16 26).  A pass is bound by the
// loads in flight (four words of either row a lane, 1024 threads an SM: 5.4 TB/s over 256 sequences).  The 31 us: 18 until each of the sequences has
// made one pass over its rows (read from HBM, 67 MB where all of them refuse; of it 6 are one sequence's launch, gather, barriers and choice of the
// token), and 4.3 for each further pass, the rows now in L2, of the sequence that refuses most, here three.  One sum a thread instead of four: 38
// us; a walk along the list of refusals for each token: 109.  kDistinct takes 16 registers more (three blocks an SM instead of four) and spills a few
// where a token of the list is left out: 128 trees of 13 over 50001 in bf16 33.8 us, where the rest found by subtraction took 35.8.
template <typename T, Draw kDraw>
__global__ void __launch_bounds__(kThreads, kDraw == kDistinct ? 3 : 4) verify_kernel(const Params p) {
  constexpr int kN = Word<T>::kN, kStep = 32 * kN, kDeep = 4;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ int32_t token_s[OPW_TREE_MAX_NODES], parent_s[OPW_TREE_MAX_NODES];
  __shared__ float u_s[OPW_TREE_MAX_NODES], p_s[OPW_TREE_MAX_NODES], q_s[OPW_TREE_MAX_NODES];
  __shared__ List list;
  __shared__ double sum_s[kWarps], rest_s[kWarps], part_s[kMaxCluster + kWarps];
  __shared__ double2 total_s[2];          // of the block: sums of R (of all tokens by the formula) and of q; two in turn
  __shared__ int32_t pick_s, some_s, listed_s;
  const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int b = blockIdx.x / blocks, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const int64_t row0 = (int64_t)b * p.nodes;
  const bool lead = rank == 0 && tid == 0;
  int x0 = 0, up0 = -1;
  float u0 = 0.f;
  if (tid < p.nodes) {                    // (one round trip with the length)
    x0 = p.tokens[row0 + tid];
    up0 = p.parents[row0 + tid];
    u0 = p.uniforms[row0 + tid];
  }
  int t = p.tree_lens[b];
  if (t > p.nodes) {
    t = p.nodes;
    if (lead) atomicOr(p.status, kErrBadPage);
  }
  if (t <= 0) {                           // (the same for the whole cluster)
    if (rank == 0 && tid < p.nodes) p.path[row0 + tid] = -1;
    if (lead) {
      p.path_lens[b] = 0;
      p.next_tokens[b] = -1;
    }
    return;
  }
  const T* target = static_cast<const T*>(p.target) + row0 * p.target_stride;
  const T* draft = kDraw == kCertain ? nullptr : static_cast<const T*>(p.draft) + row0 * p.draft_stride;
  if (tid < t) {
    const bool ok = tid > 0 && x0 >= 0 && x0 < p.vocab && up0 >= 0 && up0 < tid;
    if (tid > 0 && !ok && rank == 0) atomicOr(p.status, kErrBadPage);
    token_s[tid] = x0;
    parent_s[tid] = ok ? up0 : -1;        // a node that hangs nowhere is never asked for
    u_s[tid] = u0;
    p_s[tid] = ok ? to_float(target[up0 * p.target_stride + x0]) : 0.f;
    q_s[tid] = kDraw == kCertain ? 1.f : ok ? to_float(draft[up0 * p.draft_stride + x0]) : 0.f;
  }
  if (rank == 0 && tid < p.nodes) p.path[row0 + tid] = tid == 0 ? 0 : -1;
  if (tid == 0) {
    pick_s = INT32_MAX;
    some_s = -1;
  }
  __syncthreads();

  int turn = 0, now = 0, took = 1, n = 0; // node, length of the path, tokens in the list (0 until a refusal)
  const T* prow = target;
  const T* qrow = draft;
  bool wide = false;                      // the two rows' 16-byte words begin at the same tokens
  int shift = 0;                          // tokens from where the row's first word begins to token 0
  int64_t steps = 0;
  auto at_node = [&](int i) {
    prow = target + i * p.target_stride;
    qrow = kDraw == kCertain ? prow : draft + i * p.draft_stride;
    wide = ((uintptr_t)prow - (uintptr_t)qrow) % 16 == 0;
    shift = wide ? (int)((uintptr_t)prow % 16 / sizeof(T)) : 0;
    steps = ((int64_t)p.vocab + shift + kStep - 1) / kStep;
  };
  auto begin_of = [&](int block, int w) { // of a warp's part of the row
    return (int)(steps * ((int64_t)block * kWarps + w) / ((int64_t)blocks * kWarps) * kStep) - shift;
  };
  int first = 0, last = -1;               // this warp's part of the node's row, once it is asked for
  uint64_t mine = 0ull;                   // bit j: the list's token j lies in it
  auto find_part = [&]() {
    if (last >= first) return;
    first = begin_of(rank, warp);
    last = begin_of(rank, warp + 1);
  };
  at_node(0);
  // sums over the vocabulary without the list, by the formula: this block's warps' in sum_s, the totals of R and q
  auto pass = [&](double a, bool needs_q) -> double2 {
    find_part();
    // (four sums side by side: one would be a chain of 64-bit additions)
    double sums[4] = {0.0, 0.0, 0.0, 0.0}, rests[4] = {0.0, 0.0, 0.0, 0.0};
    auto add = [&](const Word<T>& x, const Word<T>& y, bool with_q) {
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const double pd = (double)fmaxf(to_float(x.x[i]), 0.f);
        if (kDraw == kCertain || !with_q) {
          sums[i & 3] += pd;
        } else {
          const double qd = (double)fmaxf(to_float(y.x[i]), 0.f), r = fma(-a, qd, pd);
          if (r > 0.0) sums[i & 3] += r;
          if (kDraw == kDistinct) rests[i & 3] += qd;
        }
      }
    };
    auto leave_out = [&](auto& x, auto& y, int v0) {              // the list's tokens of these words count as 0
      constexpr int kWords = sizeof(x) / sizeof(Word<T>);
      uint32_t out = 0u;                  // bit per token of this lane's words
      for (uint64_t rest = mine; rest; rest &= rest - 1) {
        const int e = list.token[__ffsll(rest) - 1] - v0;
        if ((unsigned)e < (unsigned)(kWords * kStep) && e % kStep / kN == lane) out |= 1u << (e / kStep * kN + e % kN);
      }
      if (out) {
#pragma unroll
        for (int k = 0; k < kWords; ++k)
#pragma unroll
          for (int i = 0; i < kN; ++i)
            if (out >> (k * kN + i) & 1u) x[k].x[i] = y[k].x[i] = T(0.f);
      }
    };
    auto walk = [&](auto with_q) {
      constexpr bool kQ = decltype(with_q)::value;
      const int inside = min(last, p.vocab);
      for (int v0 = first; v0 < last;) {
        if (wide && v0 >= 0 && v0 + kDeep * kStep <= inside) {    // whole words, kDeep of a row in flight
          Word<T> x[kDeep], y[kDeep];
#pragma unroll
          for (int k = 0; k < kDeep; ++k) {
            x[k].load_inside(prow, v0 + k * kStep + lane * kN);
            if (kQ) y[k].load_inside(qrow, v0 + k * kStep + lane * kN);
          }
          if (kDraw != kAgain && mine) leave_out(x, y, v0);
#pragma unroll
          for (int k = 0; k < kDeep; ++k) add(x[k], y[k], kQ);
          v0 += kDeep * kStep;
        } else {
          Word<T> x[1], y[1];
          x[0].load(prow, v0 + lane * kN, p.vocab, wide);
          if (kQ) y[0].load(qrow, v0 + lane * kN, p.vocab, wide);
          if (kDraw != kAgain && mine) leave_out(x, y, v0);
          add(x[0], y[0], kQ);
          v0 += kStep;
        }
      }
    };
    if (needs_q) walk(Flag<true>{});
    else walk(Flag<false>{});
    double sum = (sums[0] + sums[1]) + (sums[2] + sums[3]), rest = (rests[0] + rests[1]) + (rests[2] + rests[3]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (kDraw == kDistinct) rest += __shfl_xor_sync(0xffffffffu, rest, o);
    }
    if (lane == 0) {
      sum_s[warp] = sum;
      rest_s[warp] = rest;
    }
    __syncthreads();
    if (tid == 0) {
      double2 all = make_double2(0.0, 0.0);
      for (int w = 0; w < kWarps; ++w) {
        all.x += sum_s[w];
        all.y += rest_s[w];
      }
      total_s[turn & 1] = all;
    }
    cluster.sync();
    double2 all = make_double2(0.0, 0.0);
    for (int k = 0; k < blocks; ++k) {
      const double2 o = *cluster.map_shared_rank(&total_s[turn & 1], k);
      all.x += o.x;
      all.y += o.y;
    }
    ++turn;
    return all;
  };
  auto listed_sum = [&]() {               // of their R
    double d = 0.0;
#pragma unroll 1
    for (int j = 0; j < n; ++j) d += list.r[j];
    return d;
  };
  auto listed_in = [&](int from, int to) {                        // the same of the tokens in [from, to)
    double d = 0.0;
    if (kDraw != kAgain)
      for (int j = 0; j < n; ++j)
        if (list.token[j] >= from && list.token[j] < to) d += list.r[j];
    return d;
  };

  bool at_hand = false;                   // the sums in shared memory are those of R by the formula with this a
  double a = 0.0, c_total = 1.0, s_total = 1.0;
  double raw = 0.0;                       // kCertain: the row's sum, once it is known
  for (int i = 1; i < t; ++i) {
    if (parent_s[i] != now) continue;
    const int32_t x = token_s[i];
    int listed = -1;                      // its place in the list
    if (kDraw != kAgain && n > 0) {
      const uint32_t lo = __ballot_sync(0xffffffffu, lane < n && list.token[lane] == x);
      const uint32_t hi = n > 32 ? __ballot_sync(0xffffffffu, lane + 32 < n && list.token[(lane + 32) & 63] == x) : 0u;
      listed = lo ? __ffs(lo) - 1 : hi ? __ffs(hi) + 31 : -1;
    }
    const double r = listed >= 0 ? list.r[listed] : left_of<kDraw>(p_s[i], q_s[i], a);
    const double q = kDraw == kCertain ? 1.0 : listed >= 0 ? 0.0 : (double)fmaxf(q_s[i], 0.f);
    if ((double)u_s[i] * q * c_total < r * s_total) {
      if (lead) p.path[row0 + took] = i;
      now = i;
      ++took;
      n = 0;
      a = 0.0;
      c_total = s_total = 1.0;
      at_hand = false;
      at_node(now);
      first = 0;
      last = -1;
      mine = 0ull;
      continue;
    }
    const double c = c_total / s_total;
    double next = a;
    if (kDraw != kCertain) next += c;
    if (kDraw != kAgain) {
      const double after = fmax(r - c * q, 0.0);
      find_part();
      __syncthreads();                    // everybody has read the list
      if (kDraw == kCertain && n == 0) {
        if (warp == 0) {                  // the children's tokens, each where it comes first; this one is the first child
          bool here = lane < t && parent_s[lane] == now, here2 = lane + 32 < t && parent_s[(lane + 32) & 63] == now;
          const int32_t x1 = token_s[lane], x2 = token_s[(lane + 32) & 63];
          uint32_t some = __ballot_sync(0xffffffffu, here);
          if (here) here = __ffs(__match_any_sync(some, x1)) - 1 == lane;
          some = __ballot_sync(0xffffffffu, here2);
          if (here2) here2 = __ffs(__match_any_sync(some, x2)) - 1 == lane;
          const uint32_t lo = __ballot_sync(0xffffffffu, here), before = (1u << lane) - 1u;
          if (t > 32)
            for (uint32_t rest = lo; rest; rest &= rest - 1)
              if (__shfl_sync(0xffffffffu, x1, __ffs(rest) - 1) == x2) here2 = false;
          const uint32_t hi = __ballot_sync(0xffffffffu, here2);
          const int k1 = __popc(lo & before), k2 = __popc(lo) + __popc(hi & before);
          if (here) {
            list.token[k1] = x1;
            list.r[k1] = lane == i ? after : (double)fmaxf(p_s[lane], 0.f);
          }
          if (here2) {
            list.token[k2] = x2;
            list.r[k2] = lane + 32 == i ? after : (double)fmaxf(p_s[lane + 32], 0.f);
          }
          if (lane == 0) listed_s = __popc(lo) + __popc(hi);
        }
        listed = 0;
      } else {
        if (listed < 0) {                 // (kDistinct)
          listed = n++;
          if (x >= first && x < last) mine |= 1ull << listed;
        }
        if (tid == 0) {
          list.token[listed] = x;
          list.r[listed] = after;
        }
      }
      __syncthreads();
      if (kDraw == kCertain && n == 0) {
        n = listed_s;
        const int32_t x1 = list.token[lane], x2 = list.token[lane + 32];
        mine = __ballot_sync(0xffffffffu, lane < n && x1 >= first && x1 < last) |
               (uint64_t)__ballot_sync(0xffffffffu, lane + 32 < n && x2 >= first && x2 < last) << 32;
      }
    }
    double2 all;
    if (kDraw == kCertain && at_hand) all.x = raw;
    else all = pass(next, kDraw != kCertain);
    if (kDraw == kCertain) raw = all.x;
    const double left = kDraw == kAgain ? all.x : all.x + listed_sum();
    if (left > 0.0) {
      a = next;
      c_total = left;
      at_hand = true;
    } else {                              // nothing would be left: R stays
      at_hand = kDraw == kCertain;
      if (kDraw != kAgain) {
        __syncthreads();
        if (tid == 0) list.r[listed] = r;
        __syncthreads();
      }
    }
    if (kDraw == kDistinct) {
      s_total = all.y;
      if (!(s_total > 0.0)) s_total = 1.0;                        // (Q is 0 everywhere then)
    }
  }
  const bool needs_q = kDraw != kCertain && a > 0.0;
  if (!at_hand) raw = pass(a, needs_q).x;
  else if (kDraw != kCertain) raw = 0.0;
  const double total = at_hand && kDraw != kCertain ? c_total : kDraw == kAgain ? raw : raw + listed_sum();

  // The token that follows: block, warp, thread, element of the first running sum above u * total; if rounding leaves none, the last
  // element that has anything.
  if (tid < blocks) part_s[tid] = cluster.map_shared_rank(&total_s[(turn - 1) & 1], tid)->x + listed_in(begin_of(tid, 0), begin_of(tid + 1, 0));
  else if (tid >= 32 && tid < 32 + kWarps)
    part_s[kMaxCluster + tid - 32] = sum_s[tid - 32] + listed_in(begin_of(rank, tid - 32), begin_of(rank, tid - 31));
  cluster.sync();                         // (nobody leaves while its sums are read)
  const double limit = (double)fmaxf(u_s[0], 0.f) * total;
  double at = 0.0;
  auto choose = [&](const double* part, int count) {              // the part that holds it; `at` becomes the sum before
    int found = -1;
    double before = at;
    for (int k = 0; k < count; ++k) {
      const double s = part[k];
      if (s > 0.0) {
        found = k;
        before = at;
        if (at + s > limit) break;
        at += s;
      }
    }
    at = before;
    return found;
  };
  const int block = choose(part_s, blocks);
  if (lead) {
    p.path_lens[b] = took;
    if (block < 0) p.next_tokens[b] = -1;
  }
  if (block != rank) return;
  const int w = choose(part_s + kMaxCluster, kWarps);
  if (w < 0) {                            // (rounding: the block's sum was next to nothing)
    if (tid == 0) p.next_tokens[b] = -1;
    return;
  }
  const int begin = begin_of(rank, w), end = begin_of(rank, w + 1);
  for (int v0 = begin; v0 < end; v0 += kThreads * kN) {
    const int v = v0 + tid * kN;
    double r[kN], sum = 0.0;
    if (v < end) {
      Word<T> x, y;
      x.load(prow, v, p.vocab, wide);
      if (needs_q) y.load(qrow, v, p.vocab, wide);
#pragma unroll
      for (int i = 0; i < kN; ++i) r[i] = left_of<kDraw>(to_float(x.x[i]), needs_q ? to_float(y.x[i]) : 0.f, a);
      if (kDraw != kAgain)
        for (int j = 0; j < n; ++j) {
          const int e = list.token[j] - v;
#pragma unroll
          for (int i = 0; i < kN; ++i)
            if (e == i) r[i] = list.r[j];
        }
#pragma unroll
      for (int i = 0; i < kN; ++i) sum += r[i];
    }
    double incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) sum_s[warp] = incl;
    __syncthreads();
    double run = at;
    for (int k = 0; k < warp; ++k) run += sum_s[k];
    for (int k = 0; k < kWarps; ++k) at += sum_s[k];
    run += incl - sum;
    if (sum > 0.0) {
      int pick = -1, some = -1;
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        run += r[i];
        if (r[i] > 0.0) {
          some = v + i;
          if (pick < 0 && run > limit) pick = v + i;
        }
      }
      if (pick >= 0) atomicMin(&pick_s, pick);
      atomicMax(&some_s, some);
    }
    __syncthreads();
    if (pick_s != INT32_MAX) break;
  }
  if (tid == 0) p.next_tokens[b] = pick_s != INT32_MAX ? pick_s : some_s;
}

template <typename T, Draw kDraw>
cudaError_t launch_as(const opw_stage_view& s, const Params& p, int batch, int cluster, cudaStream_t stream) {
  if (cluster > 8) {
    const cudaError_t e = cudaFuncSetAttribute(verify_kernel<T, kDraw>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return opw_launch(verify_kernel<T, kDraw>, dim3((unsigned)batch * cluster), dim3(kThreads), 0, stream, s.pdl, cluster, p);
}
template <typename T>
cudaError_t launch(const opw_stage_view& s, const Params& p, int draw, int batch, int cluster, cudaStream_t stream) {
  return draw == kAgain      ? launch_as<T, kAgain>(s, p, batch, cluster, stream)
         : draw == kDistinct ? launch_as<T, kDistinct>(s, p, batch, cluster, stream)
                             : launch_as<T, kCertain>(s, p, batch, cluster, stream);
}

}  // namespace opw_verify

extern "C" opw_status_t opw_tree_verify(opw_attn_stage_t* stage, int32_t batch, int32_t nodes, int32_t vocab, int32_t dtype, int32_t draw,
                                        const void* target, int64_t target_stride, const void* draft, int64_t draft_stride,
                                        const int32_t* tokens, const int32_t* parents, const int32_t* tree_lens, const float* uniforms,
                                        int32_t* path, int32_t* path_lens, int32_t* next_tokens, void* cuda_stream) {
  if (!stage || batch < 0 || nodes < 1 || nodes > OPW_TREE_MAX_NODES || vocab < 1) return OPW_ERR_INVALID_ARG;
  const opw_stage_view s = opw_view_of(stage);
  if (dtype != OPW_PROBS_F32 && dtype != OPW_PROBS_BF16) return OPW_ERR_INVALID_ARG;
  if (draw != OPW_DRAW_AGAIN && draw != OPW_DRAW_DISTINCT && draw != OPW_DRAW_CERTAIN) return OPW_ERR_INVALID_ARG;
  if (batch == 0) return OPW_OK;
  if (!target || !tokens || !parents || !tree_lens || !uniforms || !path || !path_lens || !next_tokens) return OPW_ERR_INVALID_ARG;
  if ((draft == nullptr) != (draw == OPW_DRAW_CERTAIN)) return OPW_ERR_INVALID_ARG;
  const size_t width = dtype == OPW_PROBS_F32 ? 4 : 2;
  if (((uintptr_t)target | (uintptr_t)draft) % width ||
      ((uintptr_t)tokens | (uintptr_t)parents | (uintptr_t)tree_lens | (uintptr_t)uniforms | (uintptr_t)path | (uintptr_t)path_lens |
       (uintptr_t)next_tokens) % 4)
    return OPW_ERR_INVALID_ARG;
  if (target_stride < vocab || (draft && draft_stride < vocab)) return OPW_ERR_INVALID_ARG;
  if (batch > 65535 || vocab > (1 << 24)) return OPW_ERR_CAPACITY;
  const size_t all = (size_t)batch * nodes * 4, per_seq = (size_t)batch * 4;
  auto rows_of = [&](int64_t stride) { return ((size_t)(batch * (int64_t)nodes - 1) * stride + vocab) * width; };
  const struct { const void* at; size_t bytes; } outs[3] = {{path, all}, {path_lens, per_seq}, {next_tokens, per_seq}};
  for (int i = 0; i < 3; ++i) {
    auto meets = [&](const void* in, size_t bytes) { return in && opw_overlap(outs[i].at, outs[i].bytes, in, bytes); };
    if (meets(target, rows_of(target_stride)) || meets(draft, rows_of(draft_stride)) || meets(tokens, all) || meets(parents, all) ||
        meets(uniforms, all) || meets(tree_lens, per_seq))
      return OPW_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (meets(outs[j].at, outs[j].bytes)) return OPW_ERR_INVALID_ARG;
  }
  opw_verify::Params p;
  p.target = target;
  p.draft = draft;
  p.tokens = tokens;
  p.parents = parents;
  p.tree_lens = tree_lens;
  p.uniforms = uniforms;
  p.path = path;
  p.path_lens = path_lens;
  p.next_tokens = next_tokens;
  p.status = s.status;
  p.target_stride = target_stride;
  p.draft_stride = draft_stride;
  p.nodes = nodes;
  p.vocab = vocab;
  // Blocks per sequence, a power of two: as many as four an SM allow, and no more than give every warp four steps of a row in fp32, two in bf16.
  // (Without replacement three are resident, so that 128 sequences' last blocks begin when others have ended; half as many are slower still.)
  // Us with 1, 2, 4, 8 and 16 blocks, fp32, then bf16:
  //   again     1 tree of 64, 150000 tokens   90, 54, 33, 24, 20     60, 38, 27, 20, 18       a chain of 4 over 32000 11.5, 8.7, 7.0, 6.5, 6.8
  //             16 trees of 8, 131072        106, 59, 34, 23, 18     93, 52, 31, 21, 18
  //             64 trees of 8, 131072        127, 72, 43, 31, 37    108, 60, 37, 27, 34
  //   distinct  64 trees of 8, 131072        127, 72, 48, 39, 49    106, 61, 40, 34, 46       1 tree of 64, 150000, 48, 30, 21, 19, 17
  //             128 trees of 13, 50001        69, 50, 38, 49, 87     57, 43, 34, 43, 75
  //             256 chains of 4, 131072       66, 62, 57, 69, 120    48, 48, 48, 64, 115      (fp32: 62 by the rule)
  //   certain   64 trees of 8, 131072         60, 35, 24, 19, 30     31, 20, 16, 15, 26
  //             256 chains of 4, 131072       48, 36, 37, 44, 79     30, 24, 27, 37, 72
  int cluster = 1;
  while (cluster < opw_verify::kMaxCluster && (int64_t)batch * cluster * 2 <= 4 * s.sms && vocab > cluster * opw_verify::kWarps * 4 * 128) cluster *= 2;
  opw_device_guard guard(s.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == OPW_PROBS_F32 ? opw_verify::launch<float>(s, p, draw, batch, cluster, stream)
                                               : opw_verify::launch<__nv_bfloat16>(s, p, draw, batch, cluster, stream);
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  *s.launches += 1;
  return OPW_OK;
}
