// Head norms of queries and keys with rotary encoding and append in one pass (include/opw_draft.h).
#include <cmath>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "opw_draft.h"
#include "opw_stage.h"
#include "opw_words.cuh"

namespace opw_norm {

using opw_words::pack8;
using opw_words::pdl_launch_dependents;
using opw_words::pdl_wait;
using opw_words::unpack8;

constexpr int kPage = 16;
constexpr uint32_t kErrBadPage = 1u;      // bit of the stage's status word
constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kWarpRows = 3;              // from this many rows per SM on, a warp takes a row (measurements at the kernel)

struct Params {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  const float* q_weight;      // [D], or [Hq, D] with q_weight_stride D; null: ones
  const float* k_weight;
  __nv_bfloat16* q_out;
  __nv_bfloat16* pool;
  const double* table;        // [rot / 2] turns per position, then the amplitude
  const int32_t* seq;
  const int32_t* slots;
  const int32_t* positions;
  const int32_t* page_table;
  uint32_t* status;
  int64_t q_stride, k_stride, v_stride, num_pages;
  int32_t rows, Hq, Hkv, D, rot, num_rows, max_pages;
  float eps;
};

enum Kind { kHalf, kInterleaved, kHalfOdd };   // halves a whole number of words apart; pairs inside a word; any other half layout

// y = x * w / sqrt(sum x^2 / D + eps) per head, then the rotation, in fp32; rounded to bf16 once.
//
// kGroup threads per token row, a block (256) or a warp (32).  A lane owns 16 elements of a head in two 16-byte words, D / 16 lanes a
// head, so that the sum of squares is D / 16 lanes' shuffles away and both words of a rotated pair (half layout) are in one lane:
//   kHalf         lane j < rot / 16: words j and j + rot / 16; the others two neighbouring words that pass
//   kInterleaved  words 2j and 2j + 1, pairs beyond rot / 2 pass
//   kHalfOdd      words 2j and 2j + 1; partners through shared memory
// The lane keeps its place within the head, so its cosines and (where all heads share them) weights stay in registers.
// kPerHead: a row of weights for each head.
// Measured at 32/8 heads of 128, rotary 128 half, us with a block and with a warp per row: 128 rows 4.9 / 7.7, 512 rows 8.8 / 8.0, 1184 rows -
// / 7.9, 8192 rows - / 43.5 (4.6 TB/s of the bytes that have to move); there rotary 64 interleaved 43.6, 34 half 82, weights per head 48.  Bound by latency: a
// lane has the sum, the shuffles and the root of a head between its load and its store, 24 warps an SM hide it (80 registers), and the next
// head's words are all that is under way meanwhile.  16 warps with two heads each 48.9, 32 warps with spills 44 to 56; two elements at a time
// with weights and rotation in one factor, a third fewer instructions, 44.0.
template <int kKind, int kGroup, bool kPerHead>
__global__ void __launch_bounds__(kThreads, 3) norm_rope_kernel(const Params p) {
  constexpr int kRows = kThreads / kGroup, kWarps = kThreads / 32;
  __shared__ float2 cs_s[kRows][kMaxPairs];
  __shared__ float stage_s[kKind == kHalfOdd ? kWarps : 1][kKind == kHalfOdd ? 32 * 17 : 1];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x % kGroup, lane = threadIdx.x & 31;
  const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / kGroup;
  float2* cs = cs_s[threadIdx.x / kGroup];
  if (r >= p.rows) return;                                        // (a whole group)
  const int D = p.D, pairs = p.rot >> 1, words = D >> 3, lanes = D >> 4;
  // this lane's words of a head
  const int j = tid & (lanes - 1), half = p.rot >> 4, head0 = tid / lanes, step = kGroup / lanes;
  int c0 = 2 * j, c1 = 2 * j + 1;
  if (kKind == kHalf) {
    if (j < half) { c0 = j; c1 = j + half; }
    else { c0 = 2 * half + 2 * (j - half); c1 = c0 + 1; }
  }
  const int32_t b = p.seq[r];
  if (b < 0) return;
  struct Two { uint4 a, c; };
  auto fetch = [&](const __nv_bfloat16* src, int h, int n) {
    Two w = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
    if (h < n) {
      const uint4* s = reinterpret_cast<const uint4*>(src + (int64_t)h * D);
      w.a = s[c0];
      w.c = s[c1];
    }
    return w;
  };
  const __nv_bfloat16* qr = p.q + r * p.q_stride;
  const __nv_bfloat16* kr = p.k + r * p.k_stride;
  const int Hq = p.q ? p.Hq : 0;
  Two q_first = fetch(qr, head0, Hq);                             // under way while the row's place and cosines are found
  const Two k_first = fetch(kr, head0, p.Hkv);
  const int32_t pos = p.positions[r], slot = p.slots[r];
  __nv_bfloat16* kv = nullptr;                                    // where the row's keys and values go: null if it is not appended
  const int lp = slot / kPage, t = slot % kPage;
  if (b < p.num_rows && slot >= 0 && lp < p.max_pages) {
    const int32_t pid = p.page_table[(int64_t)b * p.max_pages + lp];
    if (pid >= 0 && pid < p.num_pages) kv = p.pool + ((int64_t)pid * p.Hkv * 2 * kPage + t) * D;
  }
  if (kv == nullptr && tid == 0) atomicOr(p.status, kErrBadPage);
  for (int i = tid; i < pairs; i += kGroup) {
    const double turns = (double)pos * p.table[i];
    const float amp = (float)p.table[pairs];
    float sn, cn;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cn);
    cs[i] = make_float2(amp * cn, amp * sn);
  }
  const int64_t tile_words = (int64_t)kPage * words;              // of a K or V tile
  const uint32_t swap = (uint32_t)t & 7u;                         // cached rows have their words permuted by the slot
  uint4* k_dst = reinterpret_cast<uint4*>(kv);
  if (kv != nullptr) {                                            // values pass
    const uint4* src = reinterpret_cast<const uint4*>(p.v + r * p.v_stride);
    const int c = tid & (words - 1), step = kGroup / words;
    for (int h0 = tid / words; h0 < p.Hkv; h0 += 4 * step) {
      uint4 w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h0 + u * step < p.Hkv) w[u] = src[(h0 + u * step) * words + c];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h0 + u * step < p.Hkv) k_dst[(2 * (h0 + u * step) + 1) * tile_words + (c ^ swap)] = w[u];
    }
  }
  if (kGroup == 32) __syncwarp();
  else __syncthreads();

  // the cosines and sines of this lane's pairs: (e of word 0, e of word 1), or (2e, 2e + 1 of the 16)
  float2 cs_r[kKind == kHalfOdd ? 1 : 8];
  uint32_t turns = 0;                                             // bit e: pair e is rotated
  if (kKind != kHalfOdd) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = 8 * j + e;                                    // both layouts: lane j has pairs 8j .. 8j + 7
      const bool turn = kKind == kHalf ? j < half : i < pairs;
      cs_r[e] = turn ? cs[i] : make_float2(1.f, 0.f);
      turns |= turn ? 1u << e : 0u;
    }
  }
  float* mine = stage_s[kKind == kHalfOdd ? threadIdx.x >> 5 : 0];
  const float inv_d = 1.f / (float)D;

  auto walk = [&](Two w, const __nv_bfloat16* src, const float* weight, uint4* dst, int64_t dst_words, uint32_t flip, int n) {
    float w0[8], w1[8];
    auto weights = [&](int h) {
      const float* w = weight + (kPerHead ? (int64_t)h * D : 0);
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(w + c0 * 8 + e)), b4 = __ldg(reinterpret_cast<const float4*>(w + c1 * 8 + e));
        w0[e] = a.x; w0[e + 1] = a.y; w0[e + 2] = a.z; w0[e + 3] = a.w;
        w1[e] = b4.x; w1[e + 1] = b4.y; w1[e + 2] = b4.z; w1[e + 3] = b4.w;
      }
    };
    if (weight == nullptr) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w0[e] = w1[e] = 1.f;
    } else if (!kPerHead) {
      weights(0);
    }
    // (all lanes of a warp make the same number of rounds: they meet in the shuffles)
    for (int base = 0; base < n; base += step) {
      const int h = base + head0;
      const Two ahead = fetch(src, h + step, n);
      float x[8], y[8];
      unpack8(w.a, x);
      unpack8(w.c, y);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += x[e] * x[e] + y[e] * y[e];
      for (int o = lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float scale = rsqrtf(sum * inv_d + p.eps);
      if (kPerHead && weight != nullptr && h < n) weights(h);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] *= scale * w0[e];
        y[e] *= scale * w1[e];
      }
      if (kKind == kHalf) {
        if (turns) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float z = x[e] * cs_r[e].x - y[e] * cs_r[e].y;
            y[e] = y[e] * cs_r[e].x + x[e] * cs_r[e].y;
            x[e] = z;
          }
        }
      } else if (kKind == kInterleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float& lo = e < 4 ? x[2 * e & 7] : y[2 * e & 7];
          float& hi = e < 4 ? x[(2 * e & 7) + 1] : y[(2 * e & 7) + 1];
          if ((turns >> e) & 1u) {
            const float z = lo * cs_r[e].x - hi * cs_r[e].y;
            hi = hi * cs_r[e].x + lo * cs_r[e].y;
            lo = z;
          }
        }
      } else {
        float* head = mine + lane / lanes * lanes * 17;         // a lane's 16 values, a word of padding behind
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          head[j * 17 + e] = x[e];
          head[j * 17 + 8 + e] = y[e];
        }
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = 16 * j + e;
          float& own = e < 8 ? x[e & 7] : y[e & 7];
          if (d < p.rot) {
            const bool upper = d >= pairs;
            const int i = upper ? d - pairs : d, other = upper ? i : d + pairs;
            const float2 t2 = cs[i];
            const float o = head[(other >> 4) * 17 + (other & 15)];
            own = upper ? own * t2.x + o * t2.y : own * t2.x - o * t2.y;
          }
        }
      }
      if (h < n) {
        uint4* out = dst + h * dst_words;
        out[c0 ^ flip] = pack8(x);
        out[c1 ^ flip] = pack8(y);
      }
      w = ahead;
    }
  };
  walk(q_first, qr, p.q_weight, reinterpret_cast<uint4*>(p.q_out + r * p.Hq * D), words, 0u, Hq);
  if (kv) walk(k_first, kr, p.k_weight, k_dst, 2 * tile_words, swap, p.Hkv);
}

template <int kKind, int kGroup, bool kPerHead>
cudaError_t launch_as(const opw_stage_view& s, const Params& p, cudaStream_t stream) {
  constexpr int kRows = kThreads / kGroup;
  return opw_launch(norm_rope_kernel<kKind, kGroup, kPerHead>, dim3((unsigned)(((int64_t)p.rows + kRows - 1) / kRows)), dim3(kThreads), 0, stream,
                    s.pdl, 1, p);
}
template <int kKind>
cudaError_t launch(const opw_stage_view& s, const Params& p, bool per_head, cudaStream_t stream) {
  if (p.rows >= kWarpRows * s.sms) return per_head ? launch_as<kKind, 32, true>(s, p, stream) : launch_as<kKind, 32, false>(s, p, stream);
  return per_head ? launch_as<kKind, 256, true>(s, p, stream) : launch_as<kKind, 256, false>(s, p, stream);
}

}  // namespace opw_norm

extern "C" opw_status_t opw_norm_rope_append(opw_attn_stage_t* stage, int32_t layer, int32_t rows, int32_t rotary_dim, int32_t layout,
                                             const double* table, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                             const void* v, int64_t v_stride, const float* q_weight, const float* k_weight,
                                             int32_t weights_per_head, float eps, const int32_t* seq, const int32_t* slots,
                                             const int32_t* positions, int32_t num_rows, const int32_t* page_table, void* q_out,
                                             void* cuda_stream) {
  if (!stage || rows < 0 || num_rows < 1) return OPW_ERR_INVALID_ARG;
  const opw_stage_view s = opw_view_of(stage);
  if (layer < 0 || layer >= s.num_layers) return OPW_ERR_INVALID_ARG;
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > s.D) return OPW_ERR_INVALID_ARG;
  if (layout != OPW_ROPE_HALF && layout != OPW_ROPE_INTERLEAVED) return OPW_ERR_INVALID_ARG;
  if (weights_per_head != 0 && weights_per_head != 1) return OPW_ERR_INVALID_ARG;
  if (!(eps > 0.f) || !std::isfinite(eps)) return OPW_ERR_INVALID_ARG;
  if (rows == 0) return OPW_OK;
  if (!table || !k || !v || !seq || !slots || !positions || !page_table || (q == nullptr) != (q_out == nullptr))
    return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)q_weight | (uintptr_t)k_weight) % 16 || (uintptr_t)table % 8 ||
      ((uintptr_t)seq | (uintptr_t)slots | (uintptr_t)positions | (uintptr_t)page_table) % 4)
    return OPW_ERR_INVALID_ARG;
  const int64_t q_row = (int64_t)s.Hq * s.D, kv_row = (int64_t)s.Hkv * s.D;
  if ((q && (q_stride < q_row || q_stride % 8)) || k_stride < kv_row || k_stride % 8 || v_stride < kv_row || v_stride % 8)
    return OPW_ERR_INVALID_ARG;
  if (q && q == q_out && q_stride != q_row) return OPW_ERR_INVALID_ARG;
  // q_out is written while other rows are still read: it may be q, but not meet the inputs in any other way
  const size_t out_bytes = (size_t)rows * q_row * 2;
  auto meets = [&](const void* in, size_t bytes) { return in && opw_overlap(q_out, out_bytes, in, bytes); };
  auto rows_of = [&](int64_t stride, int64_t row) { return ((size_t)(rows - 1) * stride + row) * 2; };
  const size_t qw = (size_t)(weights_per_head ? q_row : s.D) * 4, kw = (size_t)(weights_per_head ? kv_row : s.D) * 4;
  if (q && ((q != q_out && meets(q, rows_of(q_stride, q_row))) || meets(k, rows_of(k_stride, kv_row)) || meets(v, rows_of(v_stride, kv_row)) ||
            meets(q_weight, qw) || meets(k_weight, kw) || meets(seq, (size_t)rows * 4) || meets(slots, (size_t)rows * 4) ||
            meets(positions, (size_t)rows * 4) || meets(table, (size_t)(rotary_dim / 2 + 1) * 8) ||
            meets(page_table, (size_t)num_rows * s.max_pages * 4)))
    return OPW_ERR_INVALID_ARG;
  opw_norm::Params p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.q_weight = q_weight;
  p.k_weight = k_weight;
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
  p.rows = rows;
  p.Hq = s.Hq;
  p.Hkv = s.Hkv;
  p.D = s.D;
  p.rot = rotary_dim;
  p.num_rows = num_rows;
  p.max_pages = s.max_pages;
  p.eps = eps;
  opw_device_guard guard(s.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool per_head = weights_per_head != 0;
  const cudaError_t e = layout == OPW_ROPE_INTERLEAVED ? opw_norm::launch<opw_norm::kInterleaved>(s, p, per_head, stream)
                        : rotary_dim % 16 == 0         ? opw_norm::launch<opw_norm::kHalf>(s, p, per_head, stream)
                                                       : opw_norm::launch<opw_norm::kHalfOdd>(s, p, per_head, stream);
  if (e != cudaSuccess) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  *s.launches += 1;
  return OPW_OK;
}
