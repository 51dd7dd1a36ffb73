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
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;

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

// What the branches that the current node has refused leave of its distribution.  r_{j+1} = max(r_j - q_j, 0) / total without a division:
//     R_0 = r_0, R_{j+1} = max(R_j - c_j Q_j, 0),   r_j = R_j / C_j,  q_j = Q_j / S_j,  c_j = C_j / S_j,
// C_0 = S_0 = 1, C_{j+1} = sum of R_{j+1} and, for kDistinct, Q_{j+1} = Q_j without its token and S_{j+1} its sum.
struct Refused {
  int32_t token[OPW_TREE_MAX_NODES];
  double c[OPW_TREE_MAX_NODES];           // c_j; 0 where nothing was left: R stays
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// R_n of token v, and its Q_n.
template <Draw kDraw>
__device__ __forceinline__ double left_of(int32_t v, float p32, float q32, const Refused& f, int n, double& q) {
  double r = (double)fmaxf(p32, 0.f);     // (a NaN counts as 0)
  q = kDraw == kCertain ? 0.0 : (double)fmaxf(q32, 0.f);
  for (int j = 0; j < n; ++j) {
    const bool same = kDraw != kAgain && f.token[j] == v;
    const double c = f.c[j];
    if (c > 0.0) r = fmax(r - c * (kDraw == kCertain ? (same ? 1.0 : 0.0) : q), 0.0);
    if (kDraw == kDistinct && same) q = 0.0;
  }
  return r;
}

// The 16-byte word at token v of a row, 0 for what lies outside of the row.
template <typename T>
struct Lane {
  static constexpr int kN = 16 / sizeof(T);
  float x[kN];
  __device__ __forceinline__ void load(const T* row, int v, int vocab, bool wide) {
    if (wide && v >= 0 && v + kN <= vocab) {
      const uint4 w = __ldg(reinterpret_cast<const uint4*>(row + v));
      const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int i = 0; i < kN; ++i) x[i] = to_float(e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) x[i] = v + i >= 0 && v + i < vocab ? to_float(row[v + i]) : 0.f;
    }
  }
};

// A cluster per sequence; its blocks decide alike and share the rows of the vocabulary.
//
// What decides is scalar: the target's and the drafter's probability of each node's token, gathered at the start in one round trip.
// Only a refusal needs a whole row (the total of what it leaves), and the token that follows: the smallest v at which the running sum
// of what is left passes u * total.  A pass leaves the sums of each warp's contiguous part of the row, and the part that holds
// v is then read again, so that a sequence reads a row (target and drafter) once for each refusal, or once if there was none.
// All sums are in 64 bits, so that the token does not depend on how a row is split but for differences of 1e-16.
template <typename T, Draw kDraw>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const Params p) {
  constexpr int kN = Lane<T>::kN, kStep = 32 * kN;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ int32_t token_s[OPW_TREE_MAX_NODES], parent_s[OPW_TREE_MAX_NODES];
  __shared__ float u_s[OPW_TREE_MAX_NODES], p_s[OPW_TREE_MAX_NODES], q_s[OPW_TREE_MAX_NODES];
  __shared__ Refused refused;
  __shared__ double sum_s[kWarps], rest_s[kWarps];
  __shared__ double2 total_s[2];          // of the block: what is left, what remains of the proposal; two in turn
  const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int b = blockIdx.x / blocks, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  int t = p.tree_lens[b];
  const bool lead = rank == 0 && tid == 0;
  if (t > p.nodes) {
    t = p.nodes;
    if (lead) atomicOr(p.status, kErrBadPage);
  }
  const int64_t row0 = (int64_t)b * p.nodes;
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
    const int x = tid ? p.tokens[row0 + tid] : 0, up = tid ? p.parents[row0 + tid] : -1;
    const bool ok = tid == 0 || (x >= 0 && x < p.vocab && up >= 0 && up < tid);
    if (!ok && rank == 0) atomicOr(p.status, kErrBadPage);
    token_s[tid] = x;
    parent_s[tid] = ok ? up : -1;         // a node that hangs nowhere is never asked for
    u_s[tid] = p.uniforms[row0 + tid];
    p_s[tid] = ok && tid ? to_float(target[up * p.target_stride + x]) : 0.f;
    q_s[tid] = ok && tid && kDraw != kCertain ? to_float(draft[up * p.draft_stride + x]) : 0.f;
  }
  if (rank == 0 && tid < p.nodes) p.path[row0 + tid] = tid == 0 ? 0 : -1;
  __syncthreads();

  int turn = 0, now = 0, took = 1, n = 0; // node, length of the path, refusals at this node
  const T* prow = target;
  const T* qrow = draft;
  int first = 0, last = 0;                // this warp's part of the row, from where the row's 16-byte words begin (at or before token 0)
  bool wide = false;                      // the two rows' words begin at the same tokens
  auto at_node = [&](int i) {
    prow = target + i * p.target_stride;
    qrow = kDraw == kCertain ? prow : draft + i * p.draft_stride;
    wide = ((uintptr_t)prow - (uintptr_t)qrow) % 16 == 0;
    const int shift = wide ? (int)((uintptr_t)prow % 16 / sizeof(T)) : 0;
    const int64_t parts = (int64_t)blocks * kWarps, steps = ((int64_t)p.vocab + shift + kStep - 1) / kStep, w = (int64_t)rank * kWarps + warp;
    first = (int)(steps * w / parts * kStep) - shift;
    last = (int)(steps * (w + 1) / parts * kStep) - shift;
  };
  at_node(0);
  // sums over the vocabulary of R_n and Q_n: this block's warps' of R_n in sum_s, and the totals
  auto pass = [&](int n) -> double2 {
    double sum = 0.0, rest = 0.0;
    const bool needs_q = kDraw != kCertain && n > 0;
#pragma unroll 2
    for (int v0 = first; v0 < last; v0 += kStep) {
      const int v = v0 + lane * kN;
      Lane<T> a, c;
      a.load(prow, v, p.vocab, wide);
      if (needs_q) c.load(qrow, v, p.vocab, wide);
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        double q;
        sum += left_of<kDraw>(v + i, a.x[i], needs_q ? c.x[i] : 0.f, refused, n, q);
        if (kDraw == kDistinct) rest += q;
      }
    }
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

  bool at_hand = false;                   // the sums in shared memory are those of R_n
  double total = 1.0, q_total = 1.0;      // C_n, S_n
  for (int i = 1; i < t; ++i) {
    if (parent_s[i] != now) continue;
    double q;
    const int32_t x = token_s[i];
    const double r = left_of<kDraw>(x, p_s[i], q_s[i], refused, n, q);
    if (kDraw == kCertain) q = 1.0;
    if ((double)u_s[i] * q * total < r * q_total) {
      if (lead) p.path[row0 + took] = i;
      now = i;
      ++took;
      n = 0;
      total = q_total = 1.0;
      at_hand = false;
      at_node(now);
      continue;
    }
    __syncthreads();                      // everybody has read the list
    if (tid == 0) {
      refused.token[n] = x;
      refused.c[n] = total / q_total;
    }
    __syncthreads();
    const double2 all = pass(++n);
    at_hand = all.x > 0.0;
    if (at_hand) total = all.x;
    else {                                // (every thread has left the pass: its last barrier is behind the reads of the list)
      if (tid == 0) refused.c[n - 1] = 0.0;
      __syncthreads();
    }
    if (kDraw == kDistinct) q_total = all.y > 0.0 ? all.y : 1.0;   // (Q is 0 everywhere then)
  }
  if (!at_hand) total = pass(n).x;

  // the token that follows: block, warp, step, lane, element of the first running sum above u * total; if rounding leaves none, the last
  // element that has anything.  (One warp ends up here.)
  const double limit = (double)fmaxf(u_s[0], 0.f) * total;
  double before = 0.0, at = 0.0;
  int found = -1;
  for (int k = 0; k < blocks; ++k) {
    const double s = cluster.map_shared_rank(&total_s[(turn - 1) & 1], k)->x;
    if (s > 0.0) {
      found = k;
      before = at;
      if (at + s > limit) break;
    }
    at += s;
  }
  cluster.sync();                         // nobody leaves while its sums are read
  if (lead) {
    p.path_lens[b] = took;
    if (found < 0) p.next_tokens[b] = -1;
  }
  if (found != rank) return;
  int mine = -1;
  at = before;
  for (int w = 0; w < kWarps; ++w) {
    const double s = sum_s[w];
    if (s > 0.0) {
      mine = w;
      before = at;
      if (at + s > limit) break;
    }
    at += s;
  }
  if (mine != warp) return;
  int32_t best = -1;                      // the last element with anything, so far
  at = before;
  const bool needs_q = kDraw != kCertain && n > 0;
  for (int v0 = first; v0 < last; v0 += kStep) {
    const int v = v0 + lane * kN;
    Lane<T> a, c;
    a.load(prow, v, p.vocab, wide);
    if (needs_q) c.load(qrow, v, p.vocab, wide);
    double r[kN], sum = 0.0, q;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      r[i] = left_of<kDraw>(v + i, a.x[i], needs_q ? c.x[i] : 0.f, refused, n, q);
      sum += r[i];
    }
    double incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const uint32_t over = __ballot_sync(0xffffffffu, at + incl > limit && sum > 0.0), some = __ballot_sync(0xffffffffu, sum > 0.0);
    if (some) {
      const int who = over ? __ffs(over) - 1 : 31 - __clz(some);
      int32_t pick = -1;
      double run = at + incl - sum;
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        if (r[i] > 0.0 && !(pick >= 0 && over && run > limit)) pick = v + i;
        run += r[i];
      }
      best = __shfl_sync(0xffffffffu, pick, who);
    }
    if (over) break;
    at += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (lane == 0) p.next_tokens[b] = best;
}

template <typename T>
cudaError_t launch(const opw_stage_view& s, const Params& p, int draw, int batch, int cluster, cudaStream_t stream) {
  const dim3 grid((unsigned)batch * cluster), block(kThreads);
  if (draw == kAgain) return opw_launch(verify_kernel<T, kAgain>, grid, block, 0, stream, s.pdl, cluster, p);
  if (draw == kDistinct) return opw_launch(verify_kernel<T, kDistinct>, grid, block, 0, stream, s.pdl, cluster, p);
  return opw_launch(verify_kernel<T, kCertain>, grid, block, 0, stream, s.pdl, cluster, p);
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
  // Blocks per sequence: as many as fit the chip twice over, and no more than give every warp a step.
  int cluster = 1;
  while (cluster < opw_verify::kMaxCluster && (int64_t)batch * cluster * 2 <= 2 * s.sms && vocab > cluster * opw_verify::kWarps * 128) cluster *= 2;
  opw_device_guard guard(s.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == OPW_PROBS_F32 ? opw_verify::launch<float>(s, p, draw, batch, cluster, stream)
                                               : opw_verify::launch<__nv_bfloat16>(s, p, draw, batch, cluster, stream);
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  *s.launches += 1;
  return OPW_OK;
}
