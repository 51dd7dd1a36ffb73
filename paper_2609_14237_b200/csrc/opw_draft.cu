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
  int32_t rows, Hq, Hkv, D, rot, num_rows, max_pages, layout_half;
};

constexpr int kRopeThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kRopeWarpRows = 8;          // from this many rows per SM on, a warp takes a row (measurements at the kernel)

template <bool X>
struct Flag {
  static constexpr bool value = X;
};
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

// kGroup threads per token row, a block (256) or a warp (32, eight rows to a block).  The row's cosines and sines are computed
// once (the angle in 64 bits: turns = position * turns_per_position, reduced to [-1/2, 1/2] before it is rounded to 32)
// and serve all heads.  The heads then pass through registers in 16-byte words; a thread takes both words of a rotated
// pair, so that q may be rotated in place.  kVec 0: pairs a word apart within the head (half layout, rot % 16 == 0); 1: pairs inside
// a word (interleaved, rot % 8 == 0); 2: any even rot -- a warp takes a whole head at a time and looks partners up in
// shared memory.
// Measured at 32/8 heads of 128, rotary 128 half and 64 interleaved, us with a block and with a warp per row: 128 rows
// 3.9 / 6.5 and 3.5 / 5.6, 512 rows 5.1 / 6.7 and 4.2 / 5.7, 1184 rows 12.0 / 11.1 and 9.1 / 9.0, 8192 rows 76.7 / 39.6 and 62.9 / 36.2
// (5.1 and 5.6 TB/s of the bytes that have to move).  A block per row spends most of its life in the latencies before its first load; a warp per
// row keeps more rows in flight.  Block and warp at other shapes, half layout: 5/1 heads of 64, 512 rows 4.0 / 3.8,
// 1184 rows 7.2 / 3.8, 8192 rows 40.7 / 9.5; 64/8 of 128, 512 rows 5.8 / 9.3, 1184 rows 14.0 / 15.2, 2368 rows 28.1 / 22.6; 16/2 of 256, rotary
// 64, 1184 rows 10.1 / 10.7, 2368 rows 25.3 / 20.6.  kVec 2 has the block form only: 8192 rows at rotary 34 take 117 us.  The half layout, with two
// words and eight pairs a thread, spills 17 words (21 loads) in the warp form and 6 in the block form; the interleaved one none.
template <int kVec, int kGroup>
__global__ void __launch_bounds__(kRopeThreads, 4) rope_append_kernel(const RopeParams p) {
  constexpr int kRows = kRopeThreads / kGroup, kWarps = kRopeThreads / 32;
  __shared__ float2 cs_s[kRows][kMaxPairs];
  __shared__ float stage[kVec == 2 ? kWarps : 1][kVec == 2 ? 256 : 1];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x % kGroup;
  const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / kGroup;
  float2* cs = cs_s[threadIdx.x / kGroup];
  auto sync = [] {
    if (kGroup == 32) __syncwarp();
    else __syncthreads();
  };
  if (r >= p.rows) return;                                        // (a whole group)
  const int32_t b = p.seq[r];
  if (b < 0) return;
  const int32_t pos = p.positions[r], slot = p.slots[r];
  const int D = p.D, pairs = p.rot >> 1, words = D >> 3;
  for (int i = tid; i < pairs; i += kGroup) {
    const double turns = (double)pos * p.table[i];
    const float amp = (float)p.table[pairs];
    float sn, cn;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cn);
    cs[i] = make_float2(amp * cn, amp * sn);
  }
  // where the row's keys and values go: null if it is not appended
  __nv_bfloat16* kv = nullptr;
  const int lp = slot / kPage, t = slot % kPage;
  if (b < p.num_rows && slot >= 0 && lp < p.max_pages) {
    const int32_t pid = p.page_table[(int64_t)b * p.max_pages + lp];
    if (pid >= 0 && pid < p.num_pages) kv = p.pool + ((int64_t)pid * p.Hkv * 2 * kPage + t) * D;
  }
  if (kv == nullptr && tid == 0) atomicOr(p.status, kErrBadPage);

  const __nv_bfloat16* qr = p.q ? p.q + r * p.q_stride : nullptr;
  const __nv_bfloat16* kr = p.k + r * p.k_stride;
  const __nv_bfloat16* vr = p.v + r * p.v_stride;
  __nv_bfloat16* qo = p.q_out ? p.q_out + r * p.Hq * D : nullptr;
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
    sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per = 32 / words, c = lane & (words - 1);           // heads a warp takes at a time; this lane's word
    float* mine = stage[warp] + (lane / words) * D;
    for (int h0 = first + tid / 32 * per; h0 < last; h0 += kGroup / 32 * per) {
      const int h = h0 + lane / words;
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      float x[8];
      if (h < last) {
        w = reinterpret_cast<const uint4*>(source(h))[c];
        unpack8(w, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) mine[c * 8 + e] = x[e];
      }
      __syncwarp();
      if (h < p.Hq + p.Hkv && h < last) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = c * 8 + e;
          if (d < p.rot) {
            int i, other;
            bool upper;
            if (p.layout_half) { upper = d >= pairs; i = upper ? d - pairs : d; other = upper ? i : d + pairs; }
            else { upper = d & 1; i = d >> 1; other = d ^ 1; }
            const float2 t2 = cs[i];
            const float y = mine[other];
            x[e] = upper ? x[e] * t2.x + y * t2.y : x[e] * t2.x - y * t2.y;
          }
        }
        w = pack8(x);
      }
      if (h < last) *target(h, c) = w;
      __syncwarp();
    }
    return;
  }
  // A thread keeps its place within the head -- a unit is a rotated word (half layout: the two words of eight pairs) or a
  // word that passes -- and walks the heads: its cosines stay in registers, and nothing is divided per word (with a division per
  // word the kernel was bound by instructions, 55 us for 8192 rows of 24 KB in and out).
  const int rot_units = kVec == 0 ? p.rot >> 4 : p.rot >> 3, pass0 = p.rot >> 3;
  const int per_head = rot_units + words - pass0;
  const int lanes = per_head <= 4 ? 4 : per_head <= 8 ? 8 : per_head <= 16 ? 16 : 32;   // of a head
  constexpr int kDeep = kVec == 0 ? 2 : 4, kPairs = kVec == 0 ? 8 : 4;    // (64 registers, four blocks an SM)
  // heads [h0, h1) of one kind, kDeep at a time, loads first
  auto walk = [&](auto turns, int lane, int per, const __nv_bfloat16* src, uint4* dst, int64_t dst_words, int n, int c, int c2,
                  int d, int d2, const float2* t2, bool turn) {
    constexpr bool kTurn = decltype(turns)::value, kTwo = kTurn && kVec == 0;
    const int step = kGroup / per;
    for (int h0 = lane; h0 < n; h0 += kDeep * step) {
      uint4 w0[kDeep], w1[kTwo ? kDeep : 1];
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const int h = h0 + k * step;
        if (h >= n) break;
        const uint4* q = reinterpret_cast<const uint4*>(src + (int64_t)h * D);
        w0[k] = q[c];
        if (kTwo) w1[k] = q[c2];
      }
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const int h = h0 + k * step;
        if (h >= n) break;
        uint4* out = dst + h * dst_words;
        if (kTurn) {
          float x[8], y[8];
          unpack8(w0[k], x);
          if (kTwo) {
            float z[8];
            unpack8(w1[k], z);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              y[e] = x[e] * t2[e].x - z[e] * t2[e].y;
              z[e] = z[e] * t2[e].x + x[e] * t2[e].y;
            }
            out[d2] = pack8(z);
          } else {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              y[e] = x[e] * t2[e / 2].x - x[e + 1] * t2[e / 2].y;
              y[e + 1] = x[e + 1] * t2[e / 2].x + x[e] * t2[e / 2].y;
            }
          }
          out[d] = turn ? pack8(y) : w0[k];
        } else {
          out[d] = w0[k];
        }
      }
    }
  };
  const uint32_t swap = (uint32_t)t & 7u;                         // cached rows have their words permuted by the slot
  const int64_t tile_words = 2 * tile / 8;
  uint4* k_dst = reinterpret_cast<uint4*>(kv);
  if (kv != nullptr) {                                            // values: they need no cosines
    const int c = tid & (words - 1);
    walk(Flag<false>{}, tid / words, words, vr, k_dst + tile / 8, tile_words, p.Hkv, c, 0, (int)(c ^ swap), 0, nullptr, false);
  }
  sync();
  const int j = tid & (lanes - 1), h0 = tid / lanes;
  if (kVec == 1) {                                                // words that turn and words that pass side by side: one walk
    float2 t2[kPairs];
    const bool turn = j < rot_units;
#pragma unroll
    for (int e = 0; e < kPairs; ++e) t2[e] = turn ? cs[j * kPairs + e] : make_float2(0.f, 0.f);
    if (qr) walk(Flag<true>{}, h0, lanes, qr, reinterpret_cast<uint4*>(qo), words, p.Hq, j, 0, j, 0, t2, turn);
    if (kv) walk(Flag<true>{}, h0, lanes, kr, k_dst, tile_words, p.Hkv, j, 0, (int)(j ^ swap), 0, t2, turn);
  } else if (j < rot_units) {
    float2 t2[kPairs];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) t2[e] = cs[j * kPairs + e];
    const int c2 = j + rot_units;
    if (qr) walk(Flag<true>{}, h0, lanes, qr, reinterpret_cast<uint4*>(qo), words, p.Hq, j, c2, j, c2, t2, true);
    if (kv) walk(Flag<true>{}, h0, lanes, kr, k_dst, tile_words, p.Hkv, j, c2, (int)(j ^ swap), (int)(c2 ^ swap), t2, true);
  } else if (j < per_head) {
    const int c = pass0 + j - rot_units;
    if (qr) walk(Flag<false>{}, h0, lanes, qr, reinterpret_cast<uint4*>(qo), words, p.Hq, c, 0, c, 0, nullptr, false);
    if (kv) walk(Flag<false>{}, h0, lanes, kr, k_dst, tile_words, p.Hkv, c, 0, (int)(c ^ swap), 0, nullptr, false);
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

// grid (groups of a page's K and V tiles, sequences, layers).  A block owns a few heads' K or V rows of one sequence: it takes
// all rows that it has to move into registers (at most 64 rows; 16 words a thread), waits, and stores them, so sources and
// targets may overlap in any order.  Where a row comes from and goes to is looked up once for all of the block's tiles: that chain
// of lookups (lengths, path, page table) is what a block spends its time on.  64 sequences x 8 layers, trees of 64 of which half moves:
// 32 us with a tile per block, 27 this way; the 134 MB take a copy 20.5 us.
template <int kWords>
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const __grid_constant__ CommitParams p) {
  constexpr int kPer = 64 * kWords / kCommitThreads, kTiles = 16 / kPer;
  pdl_wait();
  const int b = blockIdx.y, tile0 = blockIdx.x * kTiles;
  const int32_t ctx = p.ctx_lens[b];
  int32_t m = p.accepted_lens[b];
  if (m < 0 || ctx < 0) m = 0;
  const bool lead = blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0;
  if (m > p.nodes) {
    m = p.nodes;
    if (lead) atomicOr(p.status, kErrBadPage);
  }
  if (lead && p.new_lens) p.new_lens[b] = ctx + m;
  const int64_t num_pages = p.num_pages[blockIdx.z];
  uint4* pool = static_cast<uint4*>(p.pool[blockIdx.z]);
  const int32_t* table = p.page_table + (int64_t)b * p.max_pages;
  // word of row ctx + i in the page's first tile, or -1
  auto place = [&](int i, int c) -> int64_t {
    const int64_t s = (int64_t)ctx + i;
    const int64_t lp = s / kPage;
    const int t = (int)(s % kPage);
    if (lp >= p.max_pages) return -1;
    const int32_t pid = table[lp];
    if (pid < 0 || pid >= num_pages) return -1;
    return ((int64_t)pid * 2 * p.Hkv * kPage + t) * kWords + (c ^ (t & 7));
  };
  uint4 held[kPer][kTiles];
  int64_t to[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int idx = threadIdx.x + u * kCommitThreads;
    const int i = idx / kWords, c = idx % kWords;
    to[u] = -1;
    if (i >= m) continue;
    const int32_t a = p.accepted[(int64_t)b * p.nodes + i];
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
    if (a == i) {                                  // already in place: looked up all the same, for the record (one sequence 1.5 -> 1.7 us)
      to[u] = -1;
      continue;
    }
#pragma unroll
    for (int k = 0; k < kTiles; ++k)
      if (tile0 + k < 2 * p.Hkv) held[u][k] = pool[from + (int64_t)(tile0 + k) * kPage * kWords];
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kPer; ++u)
    if (to[u] >= 0) {
#pragma unroll
      for (int k = 0; k < kTiles; ++k)
        if (tile0 + k < 2 * p.Hkv) pool[to[u] + (int64_t)(tile0 + k) * kPage * kWords] = held[u][k];
    }
}

}  // namespace opw_draft

template <int kVec, int kGroup>
static cudaError_t launch_rope(const opw_stage_view& s, const opw_draft::RopeParams& p, cudaStream_t stream) {
  constexpr int kRows = opw_draft::kRopeThreads / kGroup;
  return opw_launch(opw_draft::rope_append_kernel<kVec, kGroup>, dim3((p.rows + kRows - 1) / kRows), dim3(opw_draft::kRopeThreads), 0,
                    stream, s.pdl, 1, p);
}

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
                                        const int32_t* positions, int32_t num_rows, const int32_t* page_table, void* q_out,
                                        void* cuda_stream) {
  if (!stage || rows < 0 || num_rows < 1) return OPW_ERR_INVALID_ARG;
  const opw_stage_view s = opw_view_of(stage);
  if (layer < 0 || layer >= s.num_layers) return OPW_ERR_INVALID_ARG;
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > s.D) return OPW_ERR_INVALID_ARG;
  if (layout != OPW_ROPE_HALF && layout != OPW_ROPE_INTERLEAVED) return OPW_ERR_INVALID_ARG;
  if (rows == 0) return OPW_OK;
  if (!table || !k || !v || !seq || !slots || !positions || !page_table || (q == nullptr) != (q_out == nullptr))
    return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out) % 16 || (uintptr_t)table % 8 ||
      ((uintptr_t)seq | (uintptr_t)slots | (uintptr_t)positions | (uintptr_t)page_table) % 4)
    return OPW_ERR_INVALID_ARG;
  const int64_t q_row = (int64_t)s.Hq * s.D, kv_row = (int64_t)s.Hkv * s.D;
  if ((q && (q_stride < q_row || q_stride % 8)) || k_stride < kv_row || k_stride % 8 || v_stride < kv_row || v_stride % 8)
    return OPW_ERR_INVALID_ARG;
  if (q && q == q_out && q_stride != q_row) return OPW_ERR_INVALID_ARG;
  // q_out is written while other rows are still read: it may be q, but not meet the inputs in any other way
  const size_t out_bytes = (size_t)rows * q_row * 2;
  auto meets = [&](const void* in, size_t bytes) { return opw_overlap(q_out, out_bytes, in, bytes); };
  auto rows_of = [&](int64_t stride, int64_t row) { return ((size_t)(rows - 1) * stride + row) * 2; };
  if (q && ((q != q_out && meets(q, rows_of(q_stride, q_row))) || meets(k, rows_of(k_stride, kv_row)) || meets(v, rows_of(v_stride, kv_row)) ||
            meets(seq, (size_t)rows * 4) || meets(slots, (size_t)rows * 4) || meets(positions, (size_t)rows * 4) ||
            meets(table, (size_t)(rotary_dim / 2 + 1) * 8) || meets(page_table, (size_t)num_rows * s.max_pages * 4)))
    return OPW_ERR_INVALID_ARG;
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
  p.rows = rows;
  p.Hq = s.Hq;
  p.Hkv = s.Hkv;
  p.D = s.D;
  p.rot = rotary_dim;
  p.num_rows = num_rows;
  p.max_pages = s.max_pages;
  p.layout_half = layout == OPW_ROPE_HALF;
  opw_device_guard guard(s.device);
  if (!guard.ok()) return OPW_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int vec = layout == OPW_ROPE_HALF ? (rotary_dim % 16 == 0 ? 0 : 2) : (rotary_dim % 8 == 0 ? 1 : 2);
  cudaError_t e;
  if (vec == 2) e = launch_rope<2, 256>(s, p, stream);
  else if (rows >= opw_draft::kRopeWarpRows * s.sms) e = vec == 0 ? launch_rope<0, 32>(s, p, stream) : launch_rope<1, 32>(s, p, stream);
  else e = vec == 0 ? launch_rope<0, 256>(s, p, stream) : launch_rope<1, 256>(s, p, stream);
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
  if (batch == 0) return OPW_OK;
  if (!accepted || !accepted_lens || !ctx_lens || !page_table) return OPW_ERR_INVALID_ARG;
  if (((uintptr_t)accepted | (uintptr_t)accepted_lens | (uintptr_t)ctx_lens | (uintptr_t)page_table | (uintptr_t)new_lens) % 4)
    return OPW_ERR_INVALID_ARG;
  if (batch > s.max_batch) return OPW_ERR_CAPACITY;
  const size_t per_seq = (size_t)batch * 4;
  if (new_lens && (opw_overlap(new_lens, per_seq, accepted_lens, per_seq) || opw_overlap(new_lens, per_seq, ctx_lens, per_seq) ||
                   opw_overlap(new_lens, per_seq, accepted, per_seq * nodes) || opw_overlap(new_lens, per_seq, page_table, per_seq * s.max_pages)))
    return OPW_ERR_INVALID_ARG;
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
    const int per = s.D == 64 ? 8 : s.D == 128 ? 4 : 2;            // tiles a block takes (kTiles)
    const dim3 grid((2 * s.Hkv + per - 1) / per, batch, here), block(opw_draft::kCommitThreads);
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
