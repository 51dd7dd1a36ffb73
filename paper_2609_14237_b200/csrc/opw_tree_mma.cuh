// Tree attention on the 5th-generation tensor cores, for trees whose rows (nodes x group) fill matrix tiles.
//
// One CTA per SM: two softmax warpgroups ("slots"), two TMA producers (K, V) and an MMA issuer per slot.  Slot s owns a query
// tile of 128 rows in shared memory and, in TMEM, two score buffers S (128 x 64 fp32, their first 32 columns reused for P in
// bf16) and an accumulator O (128 x D fp32).  Per key tile of 64 keys (four pages):
//     S = Q K^T      tcgen05.mma, both operands in shared memory
//     P = 2^(S - m)  a thread per row: S from TMEM to registers, P back to TMEM
//     O += P V       tcgen05.mma, P from TMEM, V from shared memory
// With two buffers the products of one tile run under the softmax of the next.  (With one buffer of 128 keys a slot's tile was
// a chain of softmax, PV and QK of 4000 cycles in which every unit idled half the time.)
// A row block of up to 256 rows shares every key tile between the slots (slot s = rows 128 s ...).  One of up to 128
// rows gives each slot every other key tile, and the two (O, m, l) are joined at the end.
//
// The cache needs no re-layout: a cached row's 16-byte words are permuted by XOR with slot mod 8, which is what the
// 128-byte swizzle of the tensor core expects of rows of 128 bytes.  So K (K-major) and V (MN-major) tiles are copied by plain TMA
// boxes of 16 rows x 128 bytes, one per page and 64 dimensions.  A page that is missing or bad is copied from
// beyond the tensor's end, which TMA fills with zeros: no traffic, and no stale shared memory in the product.
//
// The running maximum is only raised when a row's new maximum exceeds it by 2^8: P stays below 2^8, exact in the same
// relative sense, and O is rescaled only where a row's scores climb: where they stay within 2^8 of those of its first tile, as with the normal
// inputs of the timings here, not at all.
//
// Measured, 32/8 heads of 128, in a replayed graph and, in brackets, called in a loop (where the clock is lower: the power limit).  Narrow, 32
// sequences with a window of 4096 and trees of 26: 105 to 114 us (117 to 125), 553 MB, 5.0 TB/s (4.6); bound by the bytes in
// flight (the tensor pipe is 35 % busy).  Wide, 16 sequences of 32k keys and trees of 64 (550 GFLOP on 2.2 GB): 537 to 576 us (620 to 640), 0.96 to
// 1.02 PFLOP/s (0.89), about 60 % of what a library matrix product reaches.  There the chain bounds it: with N = 64 keys an MMA takes 48 cycles (64 with N = 128, which shared
// memory sets), so 128 keys of both slots want 2400 cycles of the tensor core, and the issue waits for the softmax on top; with the
// softmax skipped the same loop takes 450 us.  Tried and slower: tiles of 128 keys with one buffer (559 against 547), an issuer per
// buffer (565 against 536), no turns at the exponentials (584), a third of the exponentials as a polynomial (645).
#pragma once

#include <cuda.h>

#include "opw_tree_kernels.cuh"

namespace opw_tree {

constexpr int kMmaThreads = 384;              // two softmax warpgroups; in the third two producers and two MMA issuers
constexpr int kMmaKeys = 64;                  // keys per tile
constexpr int kTilePages = kMmaKeys / 16;
constexpr int kBadRing = 32;
constexpr float kRaise = 8.f;                 // log2 of how far a row's maximum may run ahead of the one in use

// kWide: row blocks of 256 rows, for trees of more than 128.  Without it a block has 128, both slots read one query tile, and the
// shared memory of the other goes to V: a V tile waits for its softmax where a K tile is used at once, and with
// four tiles of either a CTA had too few bytes in flight (64 trees of 8 at 1k to 4k keys: 138 us, with six of V 130 us).
template <int D, bool kWide>
struct MmaTree {
  static constexpr int kHalves = D / 64;
  static constexpr int kRows = kWide ? 256 : 128;
  static constexpr uint32_t kHalfBytes = kMmaKeys * 128;      // 64 dimensions of a K or V tile
  static constexpr uint32_t kPiece = kHalves * kHalfBytes;    // a K or V tile
  static constexpr uint32_t kQHalf = 128 * 128, kQTile = kHalves * kQHalf;   // a query tile: 128 rows
  // ring depths, even: in alternate mode the tile that had a place before is then the same slot's
  static constexpr int kStagesK = D == 128 ? 4 : 8, kStagesV = D == 128 ? (kWide ? 4 : 6) : (kWide ? 8 : 12);
  static constexpr int kPieces = kStagesK + kStagesV, kQTiles = kWide ? 2 : 1;
  static size_t smem(int batch) { return 1024 + (size_t)kPieces * kPiece + kQTiles * kQTile + (size_t)(batch + 1) * 8; }
};

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, int c1, int c3, int c4, uint32_t bar, uint64_t pol) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5, %6}], "
      "[%7], %8;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(c1), "r"(0), "r"(c3), "r"(c4), "r"(bar), "l"(pol)
      : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
// two fp32 at a time
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D[tmem] (+)= A * B, M = 128, K = 16; A in shared memory or in TMEM
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
      "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.eq.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a),
      "l"(b), "r"(idesc)
      : "memory");
}
#define OPW_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define OPW_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 (16) consecutive 32-bit columns of this thread's TMEM lane
__device__ __forceinline__ void tm_ld32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
      "%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : OPW_R8(r, 0), OPW_R8(r, 8), OPW_R8(r, 16), OPW_R8(r, 24)
      : "r"(addr));
}
__device__ __forceinline__ void tm_ld16(uint32_t addr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : OPW_R8(r, 0), OPW_R8(r, 8)
               : "r"(addr));
}
__device__ __forceinline__ void tm_st32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
      "%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::OPW_I8(r, 0),
      OPW_I8(r, 8), OPW_I8(r, 16), OPW_I8(r, 24), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::OPW_I8(r, 0), OPW_I8(r, 8),
      "r"(addr)
      : "memory");
}
#undef OPW_R8
#undef OPW_I8
__device__ __forceinline__ void tm_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void named_arrive(int id, int threads) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void named_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle (layout type 2, version 1); offsets in 16-byte units.  K-major (Q, K): 8-row groups
// 1024 bytes apart, leading offset unused.  MN-major (V): 64-element blocks along the dimensions kHalfBytes apart
// (leading), groups of eight keys 1024 bytes apart (stride).
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr, uint32_t block_bytes) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(block_bytes >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// kind::f16: fp32 accumulator, A and B bf16, A K-major, B K-major or MN-major (bit 16), N, M = 128
__device__ __forceinline__ uint32_t idesc_of(int n, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}

__device__ __forceinline__ bool mbar_wait_or_dead(uint32_t bar, uint32_t parity, volatile int* dead, uint32_t* status) {
  const uint64_t t0 = global_timer_ns();
#pragma unroll 1
  while (!*dead) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (global_timer_ns() - t0 > kWaitLimitNs) {
      *dead = 1;
      atomicOr(status, kErrTimeout);
    }
  }
  return false;
}

// The row blocks of a worker's share, one after the other; every role walks the same list.
struct Segment {
  int b, g, rb, rows;          // rows of the block that exist
  int32_t t0, n;               // first key tile and number of tiles
  bool first, last;            // the block's first / last tile is among them
  bool shared;                 // both slots on every tile (more than 128 rows), or alternate tiles
  Span sp;
};
template <int kRows>
__device__ __forceinline__ Segment segment_at(const TreeParams& p, const int64_t* cum, int64_t u, int64_t u1) {
  Segment s;
  s.b = find_sequence(cum, p.batch, u);
  s.sp = span_of(p, s.b, kRows);
  const int32_t cnt = tiles_of(s.sp, kMmaKeys);
  const int64_t rem = u - cum[s.b];
  const int32_t ri = (int32_t)(rem / cnt);
  s.t0 = (int32_t)(rem - (int64_t)ri * cnt);
  s.g = ri / s.sp.blocks;
  s.rb = ri - s.g * s.sp.blocks;
  s.rows = min(s.sp.tree * p.G - s.rb * kRows, kRows);
  s.n = (int32_t)min((int64_t)(cnt - s.t0), u1 - u);
  s.first = s.t0 == 0;
  s.last = s.t0 + s.n == cnt;
  s.shared = kRows > 128 && s.rows > 128;
  return s;
}
template <int D, bool kWide>
__global__ void __launch_bounds__(kMmaThreads, 1) tree_mma_kernel(const __grid_constant__ CUtensorMap map, const TreeParams p) {
  using C = MmaTree<D, kWide>;
  constexpr uint32_t NK = C::kStagesK, NV = C::kStagesV;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[NK + NV], empty_bar[NK + NV], s_bar[2][2], p_bar[2][2], o_bar[2][2], seg_bar, end_bar[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int bad_s[kBadRing];                     // pages of a tile that are bad: bit per page; by tile, the last few
  __shared__ uint32_t odd_s[2][4];                    // keys of a tile with values that are not finite, by warp
  __shared__ float ml_s[2][2][128];                   // m, l of the two slots, to be joined
  __shared__ float zero_s;
  __shared__ volatile int dead_s;                     // a wait ran out: nobody waits any more

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t q_smem = base, ring = base + C::kQTiles * C::kQTile, ring_v = ring + NK * C::kPiece;
  int64_t* cum = reinterpret_cast<int64_t*>(smem_raw + (base - raw) + (size_t)C::kPieces * C::kPiece + C::kQTiles * C::kQTile);

  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory");
    for (int i = 0; i < C::kPieces; ++i) {             // K's stages, then V's
      mbar_init(smem_u32(&full_bar[i]), 1);
      mbar_init(smem_u32(&empty_bar[i]), 2);          // an arrival from each slot, or two from the one that has the tile
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&s_bar[0][0] + i), 1);
      mbar_init(smem_u32(&p_bar[0][0] + i), 4);       // a lane of each warp
      mbar_init(smem_u32(&o_bar[0][0] + i), 1);
    }
    mbar_init(smem_u32(&seg_bar), 256 + 2);           // the softmax threads and both MMA issuers (at the issuers' loop)
    mbar_init(smem_u32(&end_bar[0]), 1);
    mbar_init(smem_u32(&end_bar[1]), 1);
    dead_s = 0;
    zero_s = 0.f;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_before();
  scan_units(p, cum, C::kRows, kMmaKeys);             // begins and ends with a barrier of the block
  tc_after();
  constexpr uint32_t tmem = 0;                        // all 512 columns are this block's: they begin at column 0
  const int64_t U = cum[p.batch];
  const int64_t workers = workers_for(U, gridDim.x, kMmaKeys);
  const bool spare = blockIdx.x >= workers;           // fewer units than blocks
  const int64_t u0 = spare ? U : worker_begin(U, blockIdx.x, workers), u1 = spare ? U : worker_begin(U, blockIdx.x + 1, workers);
  // The combine kernel may queue up behind the first blocks that finish: its blocks do not fit beside one of these (registers), and
  // where they wait they have their index work behind them.  (Released at the end instead, in a replayed graph: chain of 4
  // 12.2 us, this way 11.8; 32 x window 4096 133 to 145 us, this way 111 to 113; call by call there is no difference.)
  pdl_launch_dependents();
  pdl_wait();                                         // up to here only this step's lengths were read
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i <= p.batch; i += kMmaThreads) p.cum[i] = cum[i];

  // Bounded wait; after the first that ran out, every wait of the block returns at once and the roles walk on through the
  // same control flow (which depends on lengths only), so that no named barrier is left short.
  auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
    const uint32_t a = smem_u32(bar);
    return mbar_try_wait(a, parity) || mbar_wait_or_dead(a, parity, &dead_s, p.status);
  };

  // Registers: 384 threads are launched with 168 each (64512); a softmax thread holds a row's 64 scores of a tile
  // beside what it keeps and wants more, the third warpgroup needs little: 256 x 200 + 128 x 104 = 64512.
  if (warp >= 8) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
  if (warp == 8 || warp == 11) {
    // ---- producers: warp 8 copies the K tiles, warp 11 the V tiles ----
    const int kv = warp == 8 ? 0 : 1;
    const uint32_t stages = kv == 0 ? NK : NV, stage0 = kv == 0 ? 0 : NK;
    const uint64_t policy = l2_evict_first_policy();
    const int32_t nowhere = (int32_t)(p.num_pages * p.Hkv);   // one past the tensor's last tile: zeros
    uint32_t issued = 0;
    bool ok = true;
    for (int64_t u = u0; u < u1 && ok;) {
      const Segment s = segment_at<C::kRows>(p, cum, u, u1);
      const int32_t page0 = s.sp.lo / kPage + s.t0 * kTilePages + (lane & (kTilePages - 1));
      auto fetch = [&](int t) -> int32_t {            // this lane's page of tile t: raw id, or -2 where there is none
        const int32_t lp = page0 + t * kTilePages;
        return t < s.n && (int64_t)lp * kPage < s.sp.n ? __ldg(p.page_table + (int64_t)s.b * p.max_pages + lp) : -2;
      };
      int32_t id = fetch(0), next = fetch(1);
      for (int t = 0; t < s.n; ++t) {
        const int32_t after = fetch(t + 2);
        const bool good = id >= 0 && id < p.num_pages;
        const uint32_t bad = __ballot_sync(0xffffffffu, !good && id != -2) & ((1u << kTilePages) - 1u);
        const int32_t tile = good ? (int32_t)((int64_t)id * p.Hkv + s.g) : nowhere;
        int32_t pages[kTilePages];                     // one thread issues: a lane each would issue one after the other, slowly
#pragma unroll
        for (int i = 0; i < kTilePages; ++i) pages[i] = __shfl_sync(0xffffffffu, tile, i);
        const uint32_t round = issued / stages, st = stage0 + issued - round * stages;
        if (round > 0) ok = ok && wait(&empty_bar[st], (round - 1) & 1u);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (elect_one()) {
          const uint32_t bar = smem_u32(&full_bar[st]), dst = ring + st * C::kPiece;
          if (kv == 0) {
            bad_s[issued % kBadRing] = (int)bad;       // (rewritten long after every row has looked: the ring of K is shorter)
            if (bad) atomicOr(p.status, kErrBadPage);
          }
          mbar_expect_tx(bar, C::kPiece);
#pragma unroll
          for (int i = 0; i < kTilePages; ++i)
#pragma unroll
            for (int h = 0; h < C::kHalves; ++h)
              tma_load_5d(dst + (uint32_t)h * C::kHalfBytes + (uint32_t)i * 2048u, &map, h, kv, pages[i], bar, policy);
        }
        __syncwarp();
        ++issued;
        id = next;
        next = after;
      }
      u += s.n;
    }
    // every copy lands before the block's shared memory is given up
    for (uint32_t i = issued > stages ? issued - stages : 0; i < issued; ++i)
      for (int k = 0; k < 1 << 16; ++k)
        if (mbar_try_wait(smem_u32(&full_bar[stage0 + i % stages]), (i / stages) & 1u)) break;
  } else {
    // ---- MMA issuers, a warp per slot: one's waits and bookkeeping hide under the other's products ----
    const int x = __shfl_sync(0xffffffffu, warp, 0) - 9;
    const uint32_t s_tm = x * 128, o_tm = 256 + x * 128;
    constexpr uint32_t q_half = C::kQHalf >> 4, k_half = C::kHalfBytes >> 4;
    const uint32_t id_s = idesc_of(kMmaKeys, false), id_o = idesc_of(D, true);
    uint32_t tiles = 0, mine = 0, n_seg = 0;         // tiles of all segments before; of this slot's; segments
    // The slot's n-th tile uses buffer n % 2, and phase n / 2 of that buffer's barriers.  This loop is the kernel's
    // pulse: a wait costs about 100 cycles here even when it need not wait, so there are four per tile and nothing else.
    const bool el = elect_one();
    const uint64_t q = desc_k(q_smem + (kWide ? x * C::kQTile : 0u)), k0 = desc_k(ring), v0 = desc_mn(ring_v, C::kHalfBytes);
    const uint32_t sb = smem_u32(&s_bar[x][0]), ob = smem_u32(&o_bar[x][0]), pb = smem_u32(&p_bar[x][0]);
    const uint32_t kf = smem_u32(&full_bar[0]), vf = smem_u32(&full_bar[NK]), ve = smem_u32(&empty_bar[NK]);
    auto wait_at = [&](uint32_t bar, uint32_t parity) {
      return mbar_try_wait(bar, parity) || mbar_wait_or_dead(bar, parity, &dead_s, p.status);
    };
    auto scores = [&](uint32_t tile, uint32_t n) -> bool {   // the slot's n-th tile, number `tile` of the worker
      const uint32_t st = tile % NK;
      if (!wait_at(kf + 8 * st, (tile / NK) & 1u)) return false;
      const uint64_t k = k0 + (uint64_t)(st * (C::kPiece >> 4));
      const uint32_t d = s_tm + 64 * (n & 1u);
      if (el) {
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
          mma_ss(d, q + (uint64_t)((j >> 2) * q_half + 2 * (j & 3)), k + (uint64_t)((j >> 2) * k_half + 2 * (j & 3)), id_s,
                 (uint32_t)(j != 0));
        tc_commit(sb + 8 * (n & 1u));
      }
      return true;
    };
    for (int64_t u = u0; u < u1;) {
      const Segment s = segment_at<C::kRows>(p, cum, u, u1);
      const uint32_t step = s.shared ? 1u : 2u, end = tiles + (uint32_t)s.n;
      uint32_t t = s.shared ? tiles : tiles + x;
      // An issuer arrives for a segment itself, and only once it has seen the one before: its waits go by parity, and a slot without
      // a tile in a segment (one tile, alternating slots) would otherwise let its softmax threads and the other slot complete the
      // barrier twice while this warp has not looked once.
      __syncwarp();
      if (el) mbar_arrive(smem_u32(&seg_bar));
      if (!wait(&seg_bar, n_seg++ & 1u)) break;
      tc_after();
      if (t < end && !scores(t, mine)) break;
      if (t + step < end && !scores(t + step, mine + 1)) break;
      bool ok = true;
      for (; t < end; t += step, ++mine) {
        const uint32_t st = t % NV, buf = mine & 1u, phase = (mine >> 1) & 1u;
        __syncwarp();                                // no lane's wait falls two phases behind the elected one
        ok = wait_at(vf + 8 * st, (t / NV) & 1u) && wait_at(pb + 8 * buf, phase);
        if (!ok) break;
        tc_after();
        if (el) {
          const uint64_t v = v0 + (uint64_t)(st * (C::kPiece >> 4));
          const uint32_t pt = s_tm + 64 * buf;
#pragma unroll
          for (int k = 0; k < kMmaKeys / 16; ++k) mma_ts(o_tm, pt + 8 * k, v + (uint64_t)(128 * k), id_o);
          tc_commit(ob + 8 * buf);
        }
        ok = wait_at(ob + 8 * buf, phase);           // P lies where the next scores of this buffer go
        if (!ok) break;
        if (el) mbar_arrive_n(ve + 8 * st, step);   // (two arrivals free a tile: one slot's of each, or both of one)
        if (t + 2 * step < end) {
          ok = scores(t + 2 * step, mine + 2);
          if (!ok) break;
        }
      }
      if (!ok) break;
      tiles = end;
      u += s.n;
    }
    __syncwarp();
    if (el) {                                        // nothing is in flight when the TMEM is given back
      tc_commit(smem_u32(&end_bar[x]));
      for (int k = 0; k < 1 << 16; ++k)
        if (mbar_try_wait(smem_u32(&end_bar[x]), 0)) break;
    }
    __syncwarp();
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // ---- softmax: thread = one row of slot x ----
    const int x = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t o_addr = lane_addr + 256 + x * 128;
    uint32_t mine = 0;                                 // tiles of this slot so far
    // (the products of the slot's n-th tile are in O)
    auto wait_products = [&](uint32_t n) { (void)wait(&o_bar[x][n & 1u], (n >> 1) & 1u); };
    uint32_t tiles = 0;                                // of all segments before
    bool on_first = true;
    for (int64_t u = u0; u < u1;) {
      const Segment s = segment_at<C::kRows>(p, cum, u, u1);
      const Span& sp = s.sp;
      const int r = s.shared ? x * 128 + row : row;    // row of the block
      const bool live = r < s.rows;
      const int R = s.rb * C::kRows + r, node = R / p.G;
      auto global_row = [&](int rr) {
        const int RR = s.rb * C::kRows + rr, nn = RR / p.G;
        return ((int64_t)s.b * p.nodes + nn) * p.Hq + (int64_t)s.g * p.G + (RR - nn * p.G);
      };
      // queries to shared memory, in the layout of a K-major swizzled operand; rows that are not there: zeros
      const uint32_t qs = q_smem + (kWide ? (uint32_t)x * C::kQTile : 0u);
      constexpr int kLoaders = kWide ? 128 : 256;      // of a query tile: its slot's threads, or all
#pragma unroll 4
      for (int i = kWide ? row : (int)threadIdx.x; i < 128 * (D / 8); i += kLoaders) {
        const int qr = i / (D / 8), c = i % (D / 8), rr = s.shared ? x * 128 + qr : qr;
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (rr < s.rows) w = *(reinterpret_cast<const uint4*>(p.q + global_row(rr) * D) + c);
        const uint32_t a = qs + (uint32_t)(c >> 3) * C::kQHalf + (uint32_t)qr * 128u + (uint32_t)(((c & 7) ^ (qr & 7)) << 4);
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
      }
      fence_proxy_async();
      {
        uint32_t z[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) z[i] = 0u;
#pragma unroll
        for (int c = 0; c < D; c += 32) tm_st32(o_addr + c, z);
        tm_wait_st();
      }
      tc_before();
      mbar_arrive(smem_u32(&seg_bar));

      auto view_of_row = [&]() -> RowView {            // asked for at masked tiles only
        if (!live) return {0ull, 0, 0, 0};
        return row_view(p, s.b, sp, node);
      };
      const int32_t border = window_border(p, s.b, sp, lane);
      float m = -INFINITY, l = 0.f;
      const uint64_t scale2 = pack2(p.scale_log2e, p.scale_log2e);
      const bool idle = (warp & 3) * 32 + (s.shared ? x * 128 : 0) >= s.rows;   // none of the warp's rows exists
      // The slots take turns at the exponentials (barriers 4 and 5: slot 0's, slot 1's turn).  Left alone they fall into
      // step, wait for the MUFU together and then leave it idle together.
      const int tiles0 = s.shared ? s.n : (s.n + 1) / 2, tiles1 = s.shared ? s.n : s.n / 2;
      int turn = 0;
      auto my_turn = [&]() { named_sync(4 + x, 256); };
      auto next_turn = [&]() {
        ++turn;
        if (x == 0 ? turn <= tiles1 : turn < tiles0) named_arrive(5 - x, 256);
      };
      if (x == 1) named_arrive(4, 256);                // slot 0 begins
      for (int t = s.shared ? 0 : x; t < s.n; t += s.shared ? 1 : 2) {
        const int32_t key0 = sp.lo / kPage * kPage + (s.t0 + t) * kMmaKeys;
        const bool edge = key0 + kMmaKeys > sp.ctx || key0 < border;
        const uint32_t buf = mine & 1u, s_addr = lane_addr + x * 128 + 64 * buf;
        (void)wait(&s_bar[x][buf], (mine >> 1) & 1u);
        tc_after();
        if (row == 0) {                                // K has been read
          mbar_arrive_n(smem_u32(&empty_bar[(tiles + t) % NK]), s.shared ? 1u : 2u);
        }
        if (edge) {
          // Values of keys that some row may not see.  The tile's warpgroup (slot 0's where they share it) clears the rows nobody
          // may read and looks for values that are not finite, a thread per key.  The V tile's barrier may only be asked
          // once the scores are there: they are issued after the tile that had its place in the ring before was read, so
          // that a completed phase of this parity is the one meant.
          const uint32_t st = (tiles + t) % NV;
          const int id = s.shared ? 1 : 2 + x, threads = s.shared ? 256 : 128;
          const uint32_t tile = ring_v + st * C::kPiece;
          const bool mine_v = !s.shared || x == 0;
          const int ox = s.shared ? 0 : x;
          // thread = 64 dimensions of a key: warps 0 and 1 the first, 2 and 3 the second (head_dim 128)
          const int vk = row & 63, vh = row >> 6;
          const uint32_t v = tile + (uint32_t)vh * C::kHalfBytes + (uint32_t)vk * 128u;
          (void)wait(&full_bar[NK + st], ((tiles + t) / NV) & 1u);
          named_sync(id, threads);
          if (mine_v) {
            const int32_t key = key0 + vk;
            const bool gone = key >= sp.n || key < sp.lo;
            bool found = false;
            if (vh < C::kHalves) {
#pragma unroll 2
              for (int c = 0; c < 8; ++c) {
                const uint32_t a = v + (uint32_t)(((c + lane) & 7) << 4);
                if (gone) {
                  asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(a), "r"(0u) : "memory");
                } else {
                  uint4 w;
                  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(a));
                  found |= any_not_finite(w);
                }
              }
            }
            const uint32_t bal = __ballot_sync(0xffffffffu, found);
            if (lane == 0) odd_s[ox][warp & 3] = bal;
            fence_proxy_async();
          }
          named_sync(id, threads);
          const volatile uint32_t* odd = odd_s[ox];
          const uint32_t odd0 = odd[0] | odd[2], odd1 = odd[1] | odd[3];   // keys 0..31, 32..63
          if (odd0 | odd1) {                           // rare: they leave the tile and are added to the rows that see them
            if (mine > 0) wait_products(mine - 1);
            tc_after();
            const RowView view = view_of_row();
            const uint32_t add0 = odd0 & visible_word(view, key0), add1 = odd1 & visible_word(view, key0 + 32);
#pragma unroll 1
            for (int c0 = 0; c0 < D; c0 += 16) {
              uint32_t o[16];
              tm_ld16(o_addr + c0, o);
              tm_wait_ld();
#pragma unroll 1
              for (int j = 0; j < kMmaKeys; ++j) {
                if (!(((j < 32 ? add0 : add1) >> (j & 31)) & 1u)) continue;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const int d = c0 + e;
                  const float val = bf16_at(tile + (uint32_t)(d >> 6) * C::kHalfBytes + (uint32_t)j * 128u +
                                            (uint32_t)((((d & 63) >> 3) ^ (j & 7)) << 4) + (uint32_t)(d & 7) * 2u);
                  if (!isfinite(val)) o[e] = __float_as_uint(__uint_as_float(o[e]) + val);
                }
              }
              __syncwarp();
              tm_st16(o_addr + c0, o);
            }
            tm_wait_st();
            named_sync(id, threads);                   // everybody has read them
            if (mine_v && vh < C::kHalves && (((vk < 32 ? odd0 : odd1) >> (vk & 31)) & 1u)) {
#pragma unroll 1
              for (int d = 0; d < 64; ++d) {
                const uint32_t a = v + (uint32_t)(d * 2);
                if (!isfinite(bf16_at(a))) asm volatile("st.shared.u16 [%0], %1;" ::"r"(a), "h"((uint16_t)0) : "memory");
              }
            }
            fence_proxy_async();
            named_sync(id, threads);
          }
        }
        if (idle) {                                    // P stays what it is: these rows of O are never read
          tc_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&p_bar[x][buf]));
          my_turn();
          next_turn();
          ++mine;
          continue;
        }
        const int bad = *(volatile int*)&bad_s[(tiles + t) % kBadRing];
        uint32_t seen0 = ~0u, seen1 = ~0u;
        if (edge || bad) {
          const RowView view = view_of_row();
          auto gone = [&](int page) { return ((bad >> page) & 1 ? 0xffffu : 0u) | ((bad >> (page + 1)) & 1 ? 0xffff0000u : 0u); };
          seen0 = visible_word(view, key0) & ~gone(0);
          seen1 = visible_word(view, key0 + 32) & ~gone(2);
        }
        uint32_t sv[kMmaKeys];
        tm_ld32(s_addr, sv);
        tm_ld32(s_addr + 32, sv + 32);
        tm_wait_ld();
        if (edge || bad) {
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            if (!((seen0 >> j) & 1u)) sv[j] = 0xff800000u;             // -inf
            if (!((seen1 >> j) & 1u)) sv[32 + j] = 0xff800000u;
          }
        }
        float tops[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) tops[e] = fmaxf(__uint_as_float(sv[e]), __uint_as_float(sv[4 + e]));
#pragma unroll
        for (int j = 8; j < kMmaKeys; j += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e) tops[e] = fmaxf(tops[e], fmaxf(__uint_as_float(sv[j + e]), __uint_as_float(sv[j + 4 + e])));
        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * p.scale_log2e;
        const bool raise = top > m + kRaise || (m == -INFINITY && top > -INFINITY);
        if (__any_sync(0xffffffffu, raise)) {
          const bool shrink = raise && m != -INFINITY; // (with m = -inf, O and l are 0 or not finite: they stay)
          const float a = shrink ? fast_exp2(m - top) : 1.f;
          if (__any_sync(0xffffffffu, shrink)) {
            wait_products(mine - 1);
            tc_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              tm_ld16(o_addr + c, o);
              tm_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a);
              tm_st16(o_addr + c, o);
            }
          }
          l *= a;
          if (raise) m = top;
        }
        my_turn();
        // (the zero, from shared memory behind the barrier, keeps the exponentials from moving above it)
        const float off1 = (m == -INFINITY ? 0.f : -m) + *(volatile float*)&zero_s;
        const uint64_t off = pack2(off1, off1);
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int c = 0; c < kMmaKeys; c += 32) {
          uint32_t pk[16];
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            float e0, e1;
            unpack2(fma2(pack2(__uint_as_float(sv[c + j]), __uint_as_float(sv[c + j + 1])), scale2, off), e0, e1);
            e0 = fast_exp2(e0);
            e1 = fast_exp2(e1);
            sum[(j >> 1) & 1] = add2(sum[(j >> 1) & 1], pack2(e0, e1));
            pk[j >> 1] = pack_bf16(e0, e1);            // rounded for the product only, the sum keeps 32 bits
          }
          tm_st16(s_addr + c / 2, pk);
        }
        next_turn();
        tm_wait_st();
        tc_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&p_bar[x][buf]));
        float a0, a1;
        unpack2(add2(sum[0], sum[1]), a0, a1);
        l += a0 + a1;
        ++mine;
      }
      tiles += (uint32_t)s.n;

      // ---- the block, or this worker's part of it, is done ----
      if (mine > 1) wait_products(mine - 2);
      if (mine > 0) wait_products(mine - 1);
      float scale0 = 1.f, scale1 = 0.f;                // of this slot's and the other's accumulator
      int c0 = 0, c1 = D;
      if (!s.shared) {
        ml_s[x][0][row] = m;
        ml_s[x][1][row] = l;
        tc_before();
        named_sync(1, 256);                            // either slot has waited for its own products
        const float mo = ml_s[x ^ 1][0][row], lo = ml_s[x ^ 1][1][row], top = fmaxf(m, mo);
        scale0 = m == -INFINITY ? (l == l ? 0.f : l) : fast_exp2(m - top);
        scale1 = mo == -INFINITY ? (lo == lo ? 0.f : lo) : fast_exp2(mo - top);
        l = (m == -INFINITY ? l : l * scale0) + (mo == -INFINITY ? lo : lo * scale1);
        m = top;
        c0 = x * (D / 2);
        c1 = c0 + D / 2;
      }
      tc_after();
      const bool complete = s.first && s.last;
      const float inv = !complete ? 1.f : l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
      float* pb = p.partials + (2 * (int64_t)blockIdx.x + (on_first ? 0 : 1)) * (int64_t)(C::kRows * (D + 2));
      const int64_t grow = live ? global_row(r) : 0;
#pragma unroll 1
      for (int c = c0; c < c1; c += 32) {
        uint32_t o[32];
        tm_ld32(o_addr + c, o);
        tm_wait_ld();
        if (!s.shared) {
          uint32_t o2[32];
          tm_ld32(lane_addr + 256 + (x ^ 1) * 128 + c, o2);
          tm_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e)
            o[e] = __float_as_uint(__uint_as_float(o[e]) * scale0 + __uint_as_float(o2[e]) * scale1);
        }
        if (live && complete) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint4 w;
            w.x = pack_bf16(__uint_as_float(o[e]) * inv, __uint_as_float(o[e + 1]) * inv);
            w.y = pack_bf16(__uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv);
            w.z = pack_bf16(__uint_as_float(o[e + 4]) * inv, __uint_as_float(o[e + 5]) * inv);
            w.w = pack_bf16(__uint_as_float(o[e + 6]) * inv, __uint_as_float(o[e + 7]) * inv);
            *reinterpret_cast<uint4*>(p.out + grow * D + c + e) = w;
          }
        } else if (live) {
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<uint4*>(pb + r * D + c + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
        __syncwarp();
      }
      if (live && (s.shared || x == 0)) {
        if (!complete) {
          pb[C::kRows * D + r] = m;
          pb[C::kRows * (D + 1) + r] = l;
        } else if (p.lse) {
          p.lse[grow] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : l == 0.f ? -INFINITY : l;
        }
      }
      if (!s.shared) {
        tc_before();
        named_sync(1, 256);                            // the other slot has read this one's accumulator
        tc_after();
      }
      on_first = false;
      u += s.n;
    }
  }
  tc_before();
  __syncthreads();
  if (warp == 9) {
    tc_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

}  // namespace opw_tree
