// Rotary encoding with append, and the commit of an accepted path (include/opw_draft.h).
#include <cmath>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "opw_draft.h"
#include "opw_stage.h"

namespace opw_draft {

constexpr int kPage = 16;
constexpr uint32_t kErrBadPage = 1u;      // bit of the stage's status word
constexpr int kLayersPerLaunch = 64;

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---------------------------------------------------------------------------------
// rotary encoding and append
// ---------------------------------------------------------------------------------
struct RopeParams {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  __nv_bfloat16* q_out;
  __nv_bfloat16* pool;
  const double* table;        // [rot / 2] turns per position, then the amplitude
  const int32_t* seq;
  const int32_t* slots;
  const int32_t* positions;
  const int32_t* page_table;
  uint32_t* status;
  int64_t q_stride, k_stride, v_stride, num_pages;
  int32_t Hq, Hkv, D, rot, max_batch, max_pages, layout_half;
};

constexpr int kRopeThreads = 256;
constexpr int kMaxPairs = 128;

__device__ __forceinline__ void unpack8(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One block per token row: the row's cosines and sines are computed once (the angle in 64 bits: turns =
// position * turns_per_position, reduced to [-1/2, 1/2] before it is rounded to 32) and serve all heads.
// The heads then pass through registers in 16-byte words; a thread takes both words of a rotated pair, so
// that q may be rotated in place.  kVec 0: pairs a word apart within the head (half layout, rot % 16 == 0);
// 1: pairs inside a word (interleaved, rot % 8 == 0); 2: any even rot -- a warp takes a whole head at a time
// and looks partners up in shared memory.
template <int kVec>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const RopeParams p) {
  __shared__ float2 cs[kMaxPairs];
  __shared__ float stage[kVec == 2 ? kRopeThreads / 32 : 1][kVec == 2 ? 256 : 1];
  pdl_launch_dependents();
  pdl_wait();
  const int r = blockIdx.x;
  const int32_t b = p.seq[r];
  if (b < 0) return;
  const int32_t pos = p.positions[r], slot = p.slots[r];
  const int D = p.D, pairs = p.rot >> 1, words = D >> 3;
  if (threadIdx.x < pairs) {
    const double turns = (double)pos * p.table[threadIdx.x];
    const float amp = (float)p.table[pairs];
    float sn, cn;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cn);
    cs[threadIdx.x] = make_float2(amp * cn, amp * sn);
  }
  // where the row's keys and values go: null if it is not appended
  __nv_bfloat16* kv = nullptr;
  const int lp = slot / kPage, t = slot % kPage;
  if (b < p.max_batch && slot >= 0 && lp < p.max_pages) {
    const int32_t pid = p.page_table[(int64_t)b * p.max_pages + lp];
    if (pid >= 0 && pid < p.num_pages) kv = p.pool + ((int64_t)pid * p.Hkv * 2 * kPage + t) * D;
  }
  if (kv == nullptr && threadIdx.x == 0) atomicOr(p.status, kErrBadPage);
  __syncthreads();

  const __nv_bfloat16* qr = p.q ? p.q + r * p.q_stride : nullptr;
  const __nv_bfloat16* kr = p.k + r * p.k_stride;
  const __nv_bfloat16* vr = p.v + r * p.v_stride;
  __nv_bfloat16* qo = p.q_out ? p.q_out + (int64_t)r * p.Hq * D : nullptr;
  const int first = p.q ? 0 : p.Hq, last = kv ? p.Hq + 2 * p.Hkv : p.Hq;   // heads: queries, keys, values
  const int64_t tile = (int64_t)kPage * D;
  auto source = [&](int h) {
    return h < p.Hq ? qr + h * D : h < p.Hq + p.Hkv ? kr + (h - p.Hq) * D : vr + (h - p.Hq - p.Hkv) * D;
  };
  // word c of head h of the output: cached rows have their words permuted by the slot
  auto target = [&](int h, int c) -> uint4* {
    if (h < p.Hq) return reinterpret_cast<uint4*>(qo + h * D) + c;
    const int g = h < p.Hq + p.Hkv ? h - p.Hq : h - p.Hq - p.Hkv;
    return reinterpret_cast<uint4*>(kv + (2 * g + (h >= p.Hq + p.Hkv)) * tile) + (c ^ (t & 7));
  };

  if (kVec == 2) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int h = first + warp; h < last; h += kRopeThreads / 32) {
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      float x[8];
      if (lane < words) {
        w = reinterpret_cast<const uint4*>(source(h))[lane];
        unpack8(w, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) stage[warp][lane * 8 + e] = x[e];
      }
      __syncwarp();
      if (lane < words && h < p.Hq + p.Hkv) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = lane * 8 + e;
          if (d < p.rot) {
            int i, other;
            bool upper;
            if (p.layout_half) { upper = d >= pairs; i = upper ? d - pairs : d; other = upper ? i : d + pairs; }
            else { upper = d & 1; i = d >> 1; other = d ^ 1; }
            const float2 c = cs[i];
            const float y = stage[warp][other];
            x[e] = upper ? x[e] * c.x + y * c.y : x[e] * c.x - y * c.y;
          }
        }
        w = pack8(x);
      }
      if (lane < words) *target(h, lane) = w;
      __syncwarp();
    }
    return;
  }
  // Units of work: a head's rotated words (half layout: two per unit), then the words that pass.
  const int rot_units = kVec == 0 ? p.rot >> 4 : p.rot >> 3;
  const int pass0 = p.rot >> 3;                                  // first word that passes
  const int per_head = rot_units + words - pass0;
  const int turned = (p.Hq + p.Hkv - first) * per_head;           // units of heads that are rotated
  const int q_units = (p.Hq - first) * per_head;
  const int total = kv ? turned + p.Hkv * words : q_units;
  for (int u = threadIdx.x; u < total; u += kRopeThreads) {
    if (u >= turned) {                                            // values
      const int i = u - turned, h = p.Hq + p.Hkv + i / words, c = i % words;
      *target(h, c) = reinterpret_cast<const uint4*>(source(h))[c];
      continue;
    }
    const int h = first + u / per_head, j = u % per_head;
    const uint4* src = reinterpret_cast<const uint4*>(source(h));
    if (j >= rot_units) {
      const int c = pass0 + j - rot_units;
      *target(h, c) = src[c];
      continue;
    }
    float a[8], y[8];
    if (kVec == 0) {
      float z[8];
      unpack8(src[j], a);
      unpack8(src[j + rot_units], z);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 c = cs[j * 8 + e];
        y[e] = a[e] * c.x - z[e] * c.y;
        z[e] = z[e] * c.x + a[e] * c.y;
      }
      *target(h, j) = pack8(y);
      *target(h, j + rot_units) = pack8(z);
    } else {
      unpack8(src[j], a);
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float2 c = cs[j * 4 + e / 2];
        y[e] = a[e] * c.x - a[e + 1] * c.y;
        y[e + 1] = a[e + 1] * c.x + a[e] * c.y;
      }
      *target(h, j) = pack8(y);
    }
  }
}

// ---------------------------------------------------------------------------------
// commit of an accepted path
// ---------------------------------------------------------------------------------
struct CommitParams {
  void* pool[kLayersPerLaunch];
  const int32_t* accepted;
  const int32_t* accepted_lens;
  const int32_t* ctx_lens;
  const int32_t* page_table;
  int32_t* new_lens;
  uint32_t* status;
  int64_t num_pages[kLayersPerLaunch];
  int32_t nodes, Hkv, max_pages;
};

constexpr int kCommitThreads = 256;

// grid (tiles of a page = K and V of every head, sequences, layers).  A block owns one head's K or V rows of one
// sequence: it takes all rows it has to move into registers (at most 64 rows of 32 words), waits, and
// stores them, so sources and targets may overlap in any order.
template <int kWords>
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const __grid_constant__ CommitParams p) {
  constexpr int kPer = 64 * kWords / kCommitThreads;
  pdl_wait();
  const int b = blockIdx.y, tile = blockIdx.x;
  const int32_t ctx = p.ctx_lens[b];
  int32_t m = p.accepted_lens[b];
  if (m < 0 || ctx < 0) m = 0;
  const bool lead = tile == 0 && blockIdx.z == 0 && threadIdx.x == 0;
  if (m > p.nodes) {
    m = p.nodes;
    if (lead) atomicOr(p.status, kErrBadPage);
  }
  if (lead && p.new_lens) p.new_lens[b] = ctx + m;
  const int64_t num_pages = p.num_pages[blockIdx.z];
  uint4* pool = static_cast<uint4*>(p.pool[blockIdx.z]);
  const int32_t* table = p.page_table + (int64_t)b * p.max_pages;
  // word of row ctx + i of this head, or -1
  auto place = [&](int i, int c) -> int64_t {
    const int64_t s = (int64_t)ctx + i;
    const int64_t lp = s / kPage;
    const int t = (int)(s % kPage);
    if (lp >= p.max_pages) return -1;
    const int32_t pid = table[lp];
    if (pid < 0 || pid >= num_pages) return -1;
    return (((int64_t)pid * 2 * p.Hkv + tile) * kPage + t) * kWords + (c ^ (t & 7));
  };
  uint4 held[kPer];
  int64_t to[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int idx = threadIdx.x + u * kCommitThreads;
    const int i = idx / kWords, c = idx % kWords;
    to[u] = -1;
    if (i >= m) continue;
    const int32_t a = p.accepted[(int64_t)b * p.nodes + i];
    if (a == i) continue;                          // already in place
    int64_t from = -1;
    if (a >= 0 && a < p.nodes) {
      from = place(a, c);
      to[u] = place(i, c);
    }
    if (from < 0 || to[u] < 0) {
      to[u] = -1;
      atomicOr(p.status, kErrBadPage);
      continue;
    }
    held[u] = pool[from];
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kPer; ++u)
    if (to[u] >= 0) pool[to[u]] = held[u];
}

}  // namespace opw_draft

extern "C" opw_status_t opw_rope_table(const opw_rope_config_t* cfg, double* table) {
  if (!cfg || !table || cfg->struct_size != sizeof(opw_rope_config_t) || cfg->reserved != 0) return OPW_ERR_INVALID_ARG;
  const int r = cfg->rotary_dim;
  if (r < 2 || r > 2 * opw_draft::kMaxPairs || r % 2) return OPW_ERR_INVALID_ARG;
  if (cfg->scaling < OPW_ROPE_PLAIN || cfg->scaling > OPW_ROPE_YARN) return OPW_ERR_INVALID_ARG;
  if (!(cfg->theta > 1.0) || !std::isfinite(cfg->theta)) return OPW_ERR_INVALID_ARG;
  if (!(cfg->amplitude >= 0.0) || !std::isfinite(cfg->amplitude)) return OPW_ERR_INVALID_ARG;
  const bool by_turns = cfg->scaling == OPW_ROPE_BANDS || cfg->scaling == OPW_ROPE_YARN;
  const double factor = cfg->scaling == OPW_ROPE_PLAIN ? 1.0 : cfg->factor;
  if (!(factor >= 1.0) || !std::isfinite(factor)) return OPW_ERR_INVALID_ARG;
  if (cfg->scaling == OPW_ROPE_NTK && r <= 2) return OPW_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925286766559;
  double low = 0.0, high = 0.0;
  if (by_turns) {
    low = cfg->low == 0.0 ? 1.0 : cfg->low;
    high = cfg->high == 0.0 ? (cfg->scaling == OPW_ROPE_BANDS ? 4.0 : 32.0) : cfg->high;
    if (!(cfg->original_context > 0.0) || !std::isfinite(cfg->original_context)) return OPW_ERR_INVALID_ARG;
    if (!(low > 0.0) || !(high > low) || !std::isfinite(high)) return OPW_ERR_INVALID_ARG;
  }
  const double theta = cfg->scaling == OPW_ROPE_NTK ? cfg->theta * std::pow(factor, (double)r / (r - 2)) : cfg->theta;
  // YARN: the (real) index whose pair makes `beta` turns over the original context, rounded outwards
  double i_low = 0.0, i_high = 0.0;
  if (cfg->scaling == OPW_ROPE_YARN) {
    auto index = [&](double beta) { return r * std::log(cfg->original_context / (beta * two_pi)) / (2.0 * std::log(theta)); };
    i_low = std::fmax(std::floor(index(high)), 0.0);
    i_high = std::fmin(std::ceil(index(low)), (double)(r - 1));
    if (!(i_high - i_low >= 0.001)) i_high = i_low + 0.001;
  }
  for (int i = 0; i < r / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / r);
    if (cfg->scaling == OPW_ROPE_LINEAR) {
      f /= factor;
    } else if (cfg->scaling == OPW_ROPE_BANDS) {
      const double s = std::fmin(std::fmax((cfg->original_context * f / two_pi - low) / (high - low), 0.0), 1.0);
      f = (1.0 - s) * f / factor + s * f;
    } else if (cfg->scaling == OPW_ROPE_YARN) {
      const double w = std::fmin(std::fmax((i - i_low) / (i_high - i_low), 0.0), 1.0);
      f = w * f / factor + (1.0 - w) * f;
    }
    table[i] = f / two_pi;
  }
  table[r / 2] = cfg->amplitude > 0.0 ? cfg->amplitude : cfg->scaling == OPW_ROPE_YARN ? 1.0 + 0.1 * std::log(factor) : 1.0;
  return OPW_OK;
}

extern "C" opw_status_t opw_rope_append(opw_attn_stage_t* stage, int32_t layer, int32_t rows, int32_t rotary_dim, int32_t layout,
                                        const double* table, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                        const void* v, int64_t v_stride, const int32_t* seq, const int32_t* slots,
                                        const int32_t* positions, const int32_t* page_table, void* q_out, void* cuda_stream) {
  if (!stage || rows < 0) return OPW_ERR_INVALID_ARG;
  const opw_stage_view s = opw_view_of(stage);
  if (layer < 0 || layer >= s.num_layers) return OPW_ERR_INVALID_ARG;
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > s.D) return OPW_ERR_INVALID_ARG;
  if (layout != OPW_ROPE_HALF && layout != OPW_ROPE_INTERLEAVED) return OPW_ERR_INVALID_ARG;
  if (!table || !k || !v || !seq || !slots || !positions || !page_table || (q == nullptr) != (q_out == nullptr))
    return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out) % 16 || (uintptr_t)table % 8 ||
      ((uintptr_t)seq | (uintptr_t)slots | (uintptr_t)positions | (uintptr_t)page_table) % 4)
    return OPW_ERR_INVALID_ARG;
  const int64_t q_row = (int64_t)s.Hq * s.D, kv_row = (int64_t)s.Hkv * s.D;
  if ((q && (q_stride < q_row || q_stride % 8)) || k_stride < kv_row || k_stride % 8 || v_stride < kv_row || v_stride % 8)
    return OPW_ERR_INVALID_ARG;
  if (q && q == q_out && q_stride != q_row) return OPW_ERR_INVALID_ARG;
  if (rows == 0) return OPW_OK;
  opw_draft::RopeParams p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.pool = static_cast<__nv_bfloat16*>(s.pool[layer]);
  p.table = table;
  p.seq = seq;
  p.slots = slots;
  p.positions = positions;
  p.page_table = page_table;
  p.status = s.status;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.num_pages = s.num_pages[layer];
  p.Hq = s.Hq;
  p.Hkv = s.Hkv;
  p.D = s.D;
  p.rot = rotary_dim;
  p.max_batch = s.max_batch;
  p.max_pages = s.max_pages;
  p.layout_half = layout == OPW_ROPE_HALF;
  opw_device_guard guard(s.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  const dim3 grid(rows), block(opw_draft::kRopeThreads);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (layout == OPW_ROPE_HALF && rotary_dim % 16 == 0)
    e = opw_launch(opw_draft::rope_append_kernel<0>, grid, block, 0, stream, s.pdl, 1, p);
  else if (layout == OPW_ROPE_INTERLEAVED && rotary_dim % 8 == 0)
    e = opw_launch(opw_draft::rope_append_kernel<1>, grid, block, 0, stream, s.pdl, 1, p);
  else
    e = opw_launch(opw_draft::rope_append_kernel<2>, grid, block, 0, stream, s.pdl, 1, p);
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  *s.launches += 1;
  return OPW_OK;
}

extern "C" opw_status_t opw_kv_commit(opw_attn_stage_t* stage, const int32_t* layers, int32_t num_layers, int32_t batch,
                                      int32_t nodes, const int32_t* accepted, const int32_t* accepted_lens,
                                      const int32_t* ctx_lens, const int32_t* page_table, int32_t* new_lens,
                                      void* cuda_stream) {
  if (!stage || batch < 0 || nodes < 1 || nodes > OPW_TREE_MAX_NODES) return OPW_ERR_INVALID_ARG;
  const opw_stage_view s = opw_view_of(stage);
  if (!layers || num_layers < 1 || num_layers > s.num_layers) return OPW_ERR_INVALID_ARG;
  for (int i = 0; i < num_layers; ++i) {
    if (layers[i] < 0 || layers[i] >= s.num_layers) return OPW_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (layers[j] == layers[i]) return OPW_ERR_INVALID_ARG;
  }
  if (!accepted || !accepted_lens || !ctx_lens || !page_table) return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)accepted | (uintptr_t)accepted_lens | (uintptr_t)ctx_lens | (uintptr_t)page_table | (uintptr_t)new_lens) % 4)
    return OPW_ERR_INVALID_ARG;
  if (batch > s.max_batch) return OPW_ERR_CAPACITY;
  const uintptr_t n0 = (uintptr_t)new_lens, n1 = n0 + (size_t)batch * 4;
  for (const int32_t* in : {accepted_lens, ctx_lens})
    if (new_lens && n0 < (uintptr_t)in + (size_t)batch * 4 && (uintptr_t)in < n1) return OPW_ERR_INVALID_ARG;
  if (batch == 0) return OPW_OK;
  opw_draft::CommitParams p;
  p.accepted = accepted;
  p.accepted_lens = accepted_lens;
  p.ctx_lens = ctx_lens;
  p.page_table = page_table;
  p.status = s.status;
  p.nodes = nodes;
  p.Hkv = s.Hkv;
  p.max_pages = s.max_pages;
  opw_device_guard guard(s.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  for (int l0 = 0; l0 < num_layers; l0 += opw_draft::kLayersPerLaunch) {
    const int here = num_layers - l0 < opw_draft::kLayersPerLaunch ? num_layers - l0 : opw_draft::kLayersPerLaunch;
    for (int i = 0; i < here; ++i) {
      p.pool[i] = s.pool[layers[l0 + i]];
      p.num_pages[i] = s.num_pages[layers[l0 + i]];
    }
    p.new_lens = l0 == 0 ? new_lens : nullptr;
    const dim3 grid(2 * s.Hkv, batch, here), block(opw_draft::kCommitThreads);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    if (s.D == 64) e = opw_launch(opw_draft::commit_kernel<8>, grid, block, 0, stream, s.pdl, 1, p);
    else if (s.D == 128) e = opw_launch(opw_draft::commit_kernel<16>, grid, block, 0, stream, s.pdl, 1, p);
    else e = opw_launch(opw_draft::commit_kernel<32>, grid, block, 0, stream, s.pdl, 1, p);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
    *s.launches += 1;
  }
  return OPW_OK;
}
