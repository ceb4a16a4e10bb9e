// Attention of many rows over a paged cache on the 5th-generation tensor cores (chunks of new tokens, prefill).
//
// o = sum_j softmax_j(scale q . k_j) v_j over tiles of 256 rows (two halves, A and B, of 128) and 128 keys.  Each half:
//   S = q_hi K^T + q_lo K^T        q = (hi + lo) 2^-e in binary16, a row's largest entry in [2^14, 2^15)
//   p = 2^(scale log2(e) S - m)    m the row's running maximum, l the running total, both fp32
//   O = O 2^(m_old - m) + p_hi V + p_lo V
// The stored keys and values are exact in binary16, so two products instead of one give fp32 accuracy, and the kernel
// is bound by the tensor pipe: 4 products of 128 x 128 x dim a half and tile.  Two halves, so that the products of one
// run while the softmax of the other does; they share the tiles of K and V in shared memory.
//   warp 0      MMA issuer.
//   warps 1-3   producer: K and V tiles from the pages in the 128-byte-swizzled layout that the MMAs read, by TMA (a
//               box a page; warp 1), or, int8, through registers, widened.  Values of tiles at an edge of what the
//               rows see are looked over: stale ones become zeros.
//   warps 4-11  softmax of half A, 16 rows a warp and four threads a row (so that a half's softmax takes half as long as
//               its products, which the other half's wait for); also q's split, the sums' rescaling and the output.
//   warps 12-19 the same of half B.
// Tensor memory: S of A and of B (128 columns each) and O of A and of B (dim columns each).  p overwrites S in place: a
// chunk of 32 scores becomes 16 columns of p_hi and 16 of p_lo, the A operand of the second product.
// p is held as 2^9 p: the low half keeps an absolute 2^-34 of the row's largest.  The running maximum is raised only
// where it would let p pass 2^5, so that O is seldom rescaled.  O is folded into an fp32 sum in the workspace with
// round-to-nearest every kChain tiles, since the tensor core truncates as it accumulates (an unbroken chain's bias grows
// with its length).
// Divided tiles are joined by a second, small launch over all SMs.
// Every wait is bounded; on expiry the status word is raised and the block leaves with its copies and MMAs done.

#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "attention.cuh"
#include "noise.cuh"  // packed fp32 pairs
#include "ptx.cuh"

namespace spl {
namespace {

constexpr int kThreads = 20 * 32, kProducers = 3;
constexpr int kRows = 256, kKeys = 128, kStages = 3;
constexpr int kChain = 8;        // key tiles of an accumulation chain of O (1024 keys)
constexpr float kShift = 9.0f;  // p is held as 2^kShift p
constexpr float kLazy = 5.0f;    // and may reach 2^(kShift + kLazy), times a scale below 2, before the maximum is raised
constexpr int kMinExp = -100, kMaxExp = 126;

// Barriers by index: kFull, kEmpty a stage; kScale the scales of K of two steps; kRaw the copies of V's edge tiles; the
// others a half each, their phases counting its own key tiles (kQ: its pieces); kPieceFull, kPieceFree a piece's place.
enum {
  kFull = 0, kEmpty = 3, kScale = 6, kQ = 8, kSFull = 10, kPFull = 12, kPv = 14, kDrain = 16, kRaw = 17,
  kPieceFull = 18, kPieceFree = 20, kBars = 22
};

// A block's piece of a tile, as warp 1 hands it to the others (two in shared memory, in turn).
struct Piece {
  int tiles;           // key tiles, 0 after the last piece
  int j0;              // first key of the first
  int key_lo, key_hi;  // keys that some row sees
  int all_lo, all_hi;  // keys that every row sees
  int b, h;            // sequence, key head
  int row0, n, len;    // the sequence's first row, rows and length
  int r0, rows;        // rows of the tile among the sequence's rows of the key head
  int first;           // the first tile's index among the whole tile's
  int whole;           // the piece is the whole tile
  int last_block;      // the block that has the whole tile's end
};
constexpr int kPieces = 2;

// D columns of binary16 in panels of 64 (128 bytes, 128-byte swizzle): a panel of R rows is R x 128 bytes.
template <int D>
struct Layout {
  static constexpr int PANELS = D / 64;
  static constexpr uint32_t PANEL = 128 * 128;             // 128 rows
  static constexpr uint32_t TILE = PANELS * PANEL;         // q_hi or q_lo of a half; a K or V tile
  static constexpr uint32_t Q = 0, KV = 4 * TILE;          // [A hi, A lo, B hi, B lo], stages
  static constexpr uint32_t AUX = KV + kStages * TILE;
  // aux: scales of K and of V of two tiles, bits of bad values of two tiles, largest scales of two tiles, barriers
  static constexpr uint32_t KS = AUX, VS = KS + 2 * kKeys * 4, BAD = VS + 2 * kKeys * 4, VMAX = BAD + 2 * 16;
  static constexpr uint32_t BARS = VMAX + 2 * 16, MISC = BARS + 8 * kBars, PIECES = MISC + 16;
  static constexpr uint32_t BYTES = PIECES + kPieces * sizeof(Piece);
  static constexpr uint32_t SMEM = BYTES;                  // the base is aligned (checked by the kernel)
  static_assert(SMEM <= 232448, "227 KB of dynamic shared memory per block");
  static_assert(kMaxSeqs * 8 <= 4 * TILE + kStages * TILE, "the prefix sums fit where the tiles go");
  static constexpr uint32_t S = 0, O = 256;                // tensor memory columns (+ 128 and + D for half B)
  static constexpr uint32_t IDESC_S = make_idesc(0, 128, kKeys);
  static constexpr uint32_t IDESC_O = make_idesc(0, 128, D) | (1u << 16);  // B: the values, dims contiguous
};
constexpr uint32_t kTmemCols = 512;

// A workspace slot: sums as [dim / 4][256 rows][4], then the rows' maxima and totals.
template <int D>
constexpr int64_t slot_floats() {
  return (int64_t)kRows * (D + kSlotStats);
}

// A divided tile that begins in a block's run, for the join.
struct Divided {
  int last_block;  // 0: none (a divided tile never ends in block 0)
  int head, row0, n, r0, rows;
};

__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                       uint32_t accumulate, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(hi), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                       uint32_t accumulate, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
      "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(hi), "r"(leader)
      : "memory");
}
// Descriptor low word of a tile whose rows are the K dimension (values): 64-dim panels PANEL bytes apart (leading
// byte offset), groups of 8 keys 1024 bytes apart (stride byte offset, in the high word).
__device__ __forceinline__ uint32_t sdesc_lo_mn(uint32_t saddr) {
  return ((saddr & 0x3FFFFu) >> 4) | ((128u * 128u >> 4) << 16);
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ bool f16_special2(uint32_t h) {
  return (h & 0x7c00u) == 0x7c00u || (h & 0x7c000000u) == 0x7c000000u;
}

using Run = AttnRun<kRows, kKeys, kThreads>;

template <int D, bool I8>
struct Kernel {
  using L = Layout<D>;
  const AttnArgs& a;
  const CUtensorMap &map_k, &map_v;  // F16: the stored vectors as [slots, D]
  uint32_t smem;                     // shared address of the aligned base
  uint32_t tmem;
  volatile int* abort;
  Piece* pieces;

  __device__ uint32_t bar(int i) const { return smem + L::BARS + 8u * i; }
  __device__ bool wait(int i, uint32_t parity) const {
    return __all_sync(0xffffffffu, mbar_wait(bar(i), parity, kWaitNs, abort));
  }
  __device__ void give_up() const {
    *abort = 1;
    atomicOr(a.batch.status, kStatusTimeout);
  }
  // Whether some row of the tile sees only a part of the 128 keys from j0 on.
  static __device__ bool edge_of(const Piece& x, int j0) { return j0 < x.all_lo || j0 + kKeys > x.all_hi; }
  // The k-th piece, when it is there; a warp that has done with it says so (it may not read it afterwards).
  __device__ const Piece* piece(int k, bool& ok) const {
    ok = ok && wait(kPieceFull + k % kPieces, (uint32_t)(k / kPieces) & 1u);
    return pieces + k % kPieces;
  }
  __device__ void piece_done(int k) const {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar(kPieceFree + k % kPieces));
  }
  // Warp 1: the k-th piece of the run (or its end) for all.
  __device__ bool hand_out(const Run& run, int k) const {
    if (k >= kPieces && !wait(kPieceFree + k % kPieces, (uint32_t)(k / kPieces - 1) & 1u)) return false;
    if ((threadIdx.x & 31) == 0) {
      Piece& y = pieces[k % kPieces];
      y.tiles = 0;
      if (run.busy()) {
        const AttnTile& x = run.x;
        y = {run.last() - run.first, (x.unit0 + run.first) * kKeys, x.key_lo, x.key_hi, x.all_lo, x.all_hi, x.b, x.h,
             (int)x.s.row0, x.s.n, x.s.len, x.r0, x.rows, run.first, run.whole() ? 1 : 0, run.last_block()};
      }
      mbar_arrive(bar(kPieceFull + k % kPieces));
    }
    __syncwarp();
    return true;
  }

  // ---------------------------------------------------------------- producer
  // Values of an edge tile, a lane a key: those that no row sees become zeros; an infinity or NaN in one that only
  // some rows see becomes 0 and is marked.
  __device__ void look_over(const Piece& x, int j0, uint32_t base, int step) const {
    const int lane = threadIdx.x & 31;
    for (int word = (threadIdx.x >> 5) - 1; word < kKeys / 32; word += kProducers) {
      const int key = 32 * word + lane, j = j0 + key;
      const bool seen = j >= x.key_lo && j < x.key_hi;
      bool bad = false;
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        const uint32_t at = base + (c >> 3) * L::PANEL + key * 128 + (((c & 7) ^ (key & 7)) << 4);
        const uint4 v = ld_shared16(at);
        const bool special = f16_special2(v.x) || f16_special2(v.y) || f16_special2(v.z) || f16_special2(v.w);
        bad |= special;
        if (special || !seen) st_shared16(at, make_uint4(0u, 0u, 0u, 0u));
      }
      const unsigned marks = __ballot_sync(0xffffffffu, bad && seen);
      if (lane == 0)
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(smem + L::BAD + 16u * (step & 1) + 4u * word), "r"(marks)
                     : "memory");
    }
    fence_proxy_async_smem();
    __syncwarp();
  }
  static __device__ __forceinline__ void mbar_arrive_more(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
  }
  __device__ void producer(Run& run) const {
    const int i = threadIdx.x - 32, warp = i >> 5, lane = i & 31;
    const uint64_t policy = l2_evict_last();  // other tiles of rows read the same keys
    const int heads = a.cache.heads, shift = a.cache.page_shift, in_page = (1 << shift) - 1;
    int tile = 0, step = 0;  // tiles issued, pairs of them
    bool ok = true;
    // F16: barriers of the copies in flight (a bit a stage: kRaw instead of kFull) and phases, for leaving early
    uint32_t raw_phase = 0u;
    for (int k = 0; ok; ++k) {
      if (warp == 0) {
        ok = hand_out(run, k);
        if (run.busy()) run.next();
      }
      const Piece* place = piece(k, ok);
      if (!ok) break;
      const Piece x = *place;
      if (warp > 0) piece_done(k);
      if (x.tiles == 0) break;
      // page of the keys 16 lane .. of the u-th tile, -1 where no row sees any of them (lanes 0-7)
      auto pages_of = [&](int u) {
        const int j = x.j0 + u * kKeys + 16 * lane;
        if (lane >= kKeys / 16 || u >= x.tiles || j >= x.key_hi || j + 16 <= x.key_lo) return -1;
        return paged_page(a.cache, a.batch, x.b, j);
      };
      int page = pages_of(0);
      if constexpr (!I8) {
        // Boxes of a page's tokens, at most 128, a lane each; where no row sees any key of it the box lies past the
        // pool's end and the copy fills it with zeros.
        const int box = min(kKeys, 1 << shift), boxes = kKeys / box;
        for (int u = 0; ok && u < x.tiles; ++u, ++step) {
          const int j0 = x.j0 + u * kKeys;
          const int pg = __shfl_sync(0xffffffffu, page, (lane * box / 16) & 7);
          const int row = pg >= 0 ? (int)((((int64_t)pg * heads + x.h) << shift) + ((j0 + lane * box) & in_page))
                                  : (int)((int64_t)a.cache.pages * heads << shift);
          const bool edge = edge_of(x, j0);
          for (int which = 0; ok && which < 2; ++which, ++tile) {
            const int stage = tile % kStages;
            if (warp == 0) {
              if (tile >= kStages) ok = wait(kEmpty + stage, (uint32_t)(tile / kStages - 1) & 1u);
              if (!ok) break;
              const bool raw = which && edge;  // values that are looked over before they are handed on
              if (lane == 0) {
                mbar_expect_tx(bar(raw ? kRaw : kFull + stage), L::TILE);
                if (!raw) mbar_arrive_more(bar(kFull + stage), kProducers - 1);
              }
              __syncwarp();
              if (lane < boxes) {
                const uint32_t dst = smem + L::KV + (uint32_t)stage * L::TILE + (uint32_t)(lane * box) * 128u;
#pragma unroll
                for (int p = 0; p < L::PANELS; ++p)
                  tma_load_2d(dst + p * L::PANEL, which ? &map_v : &map_k, bar(raw ? kRaw : kFull + stage), 64 * p, row,
                              policy);
              }
              __syncwarp();
            }
            if (which && edge) {
              ok = wait(kRaw, raw_phase);
              if (!ok) break;
              raw_phase ^= 1u;
              look_over(x, j0, smem + L::KV + (uint32_t)stage * L::TILE, step);
              if (lane == 0) mbar_arrive(bar(kFull + stage));
            }
          }
          if (!ok) break;
          page = pages_of(u + 1);
        }
      } else {
        constexpr int PARTS = D / 16, KEY_STEP = 32 * kProducers / PARTS, PER = (kKeys + KEY_STEP - 1) / KEY_STEP;
        uint4 regs[PER];  // the next tile's 16-byte chunks, on their way
        float scale[2];
        auto load = [&](int u, int which) {
          const int j0 = x.j0 + u * kKeys;
          const char* src = static_cast<const char*>(which ? a.cache.v : a.cache.k);
          const int part = i % PARTS, key0 = i / PARTS;
#pragma unroll
          for (int k = 0; k < PER; ++k) {
            const int key = key0 + KEY_STEP * k, j = j0 + key;
            const int pg = __shfl_sync(0xffffffffu, page, (key >> 4) & 7);
            const bool there = key < kKeys && pg >= 0 && j >= x.key_lo && j < x.key_hi;
            const int64_t slot = there ? ((((int64_t)pg * heads + x.h) << shift) + (j & in_page)) : 0;
            regs[k] = there ? __ldg(reinterpret_cast<const uint4*>(src + slot * D + part * 16))
                            : make_uint4(0u, 0u, 0u, 0u);
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int key = i + 32 * kProducers * k, j = j0 + key;
            const int pg = __shfl_sync(0xffffffffu, page, (key >> 4) & 7);
            const bool there = key < kKeys && pg >= 0 && j >= x.key_lo && j < x.key_hi;
            const int64_t slot = there ? ((((int64_t)pg * heads + x.h) << shift) + (j & in_page)) : 0;
            scale[k] = there ? __ldg((which ? a.cache.v_scale : a.cache.k_scale) + slot) : 0.f;
          }
        };
        auto put = [&](int which) {
          const int stage = tile % kStages;
          if (tile >= kStages) ok = wait(kEmpty + stage, (uint32_t)(tile / kStages - 1) & 1u);
          if (!ok) return;
          const uint32_t base = smem + L::KV + (uint32_t)stage * L::TILE;
          const int part = i % PARTS, key0 = i / PARTS;  // two chunks of 8 values
          const uint32_t panel = base + (uint32_t)(part >> 2) * L::PANEL;
#pragma unroll
          for (int k = 0; k < PER; ++k) {
            const int key = key0 + KEY_STEP * k;
            if (key >= kKeys) break;
            const uint4 c = regs[k];
            const uint32_t w[4] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u, c.z ^ 0x80808080u, c.w ^ 0x80808080u};
            const int c0 = (2 * part) & 7;
            st_shared16(panel + key * 128 + ((c0 ^ (key & 7)) << 4),
                        make_uint4(i8_pair(w[0], 0x4140u), i8_pair(w[0], 0x4342u), i8_pair(w[1], 0x4140u),
                                   i8_pair(w[1], 0x4342u)));
            st_shared16(panel + key * 128 + (((c0 + 1) ^ (key & 7)) << 4),
                        make_uint4(i8_pair(w[2], 0x4140u), i8_pair(w[2], 0x4342u), i8_pair(w[3], 0x4140u),
                                   i8_pair(w[3], 0x4342u)));
          }
          const uint32_t sc = smem + (which ? L::VS : L::KS) + (uint32_t)(step & 1) * (kKeys * 4) + 4u * i;
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(sc), "f"(scale[0]) : "memory");
          if (i < kKeys - 32 * kProducers)
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(sc + 4u * 32 * kProducers), "f"(scale[1]) : "memory");
          if (which) {
            float top = fmaxf(scale[0], scale[1]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (lane == 0)
              asm volatile("st.shared.f32 [%0], %1;" ::"r"(smem + L::VMAX + 16u * (step & 1) + 4u * warp), "f"(top)
                           : "memory");
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(kFull + stage));
            if (!which) mbar_arrive(bar(kScale + (step & 1)));
          }
          ++tile;
        };
        load(0, 0);
        for (int u = 0; ok && u < x.tiles; ++u, ++step) {
          put(0);
          load(u, 1);
          page = pages_of(u + 1);
          if (ok) put(1);
          if (u + 1 < x.tiles) load(u + 1, 0);
        }
      }
    }
    if constexpr (!I8) {  // no copy in flight when the block leaves early
      if (!ok && warp == 0)
        for (int t = max(0, tile - kStages); t <= tile; ++t)
          mbar_wait(bar(kFull + t % kStages), (uint32_t)(t / kStages) & 1u, kDrainNs, nullptr);
    }
    if (!ok && lane == 0) give_up();
  }

  // ---------------------------------------------------------------- MMA issuer
  __device__ void issue_s(int half, int tile, uint32_t leader) const {
    const uint32_t q = sdesc_lo(smem + L::Q + (uint32_t)half * 2 * L::TILE);
    const uint32_t k = sdesc_lo(smem + L::KV + (uint32_t)(tile % kStages) * L::TILE);
    const uint32_t d = tmem + L::S + 128u * half;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const uint32_t off = ((uint32_t)(s / 4) * L::PANEL + (uint32_t)(s % 4) * 32u) >> 4;
      mma_ss(d, q + off, k + off, kSdescHi128, L::IDESC_S, s > 0 ? 1u : 0u, leader);
      mma_ss(d, q + off + (L::TILE >> 4), k + off, kSdescHi128, L::IDESC_S, 1u, leader);
    }
  }
  __device__ void issue_pv(int half, int tile, bool fresh, uint32_t leader) const {
    const uint32_t v = sdesc_lo_mn(smem + L::KV + (uint32_t)(tile % kStages) * L::TILE);
    const uint32_t p = tmem + L::S + 128u * half, d = tmem + L::O + (uint32_t)D * half;
#pragma unroll
    for (int s = 0; s < kKeys / 16; ++s) {
      const uint32_t at = p + 32u * (s / 2) + 8u * (s % 2), off = (uint32_t)(s * 16 * 128) >> 4;
      mma_ts(d, at, v + off, kSdescHi128, L::IDESC_O, fresh && s == 0 ? 0u : 1u, leader);
      mma_ts(d, at + 16u, v + off, kSdescHi128, L::IDESC_O, 1u, leader);
    }
  }
  __device__ void issuer() const {
    const uint32_t leader = elect_one();
    bool ok = true;
    int tile = 0;
    uint32_t p_phase = 0u, q_phase = 0u;  // a bit each half
    auto commit = [&](int i) {
      if (leader) mma_commit(bar(i));
      __syncwarp();
    };
    auto full = [&](int t) {
      ok = ok && wait(kFull + t % kStages, (uint32_t)(t / kStages) & 1u);
      tc_fence_after();
    };
    // The loops' bounds come through shuffles: the compiler then knows them, and all that the descriptors are made of,
    // to be the same in every lane.
    for (int k = 0; ok; ++k) {
      const Piece* x = piece(k, ok);
      if (!ok) break;
      const int halves = __shfl_sync(0xffffffffu, x->rows > 128 ? 2 : 1, 0);
      const int n = __shfl_sync(0xffffffffu, x->tiles, 0);
      piece_done(k);
      if (n == 0) break;
      full(tile);
      for (int h = 0; ok && h < halves; ++h) {
        ok = wait(kQ + h, q_phase >> h & 1u);
        if (!ok) break;
        q_phase ^= 1u << h;
        tc_fence_after();
        issue_s(h, tile, leader);
        commit(kSFull + h);
      }
      if (!ok) break;
      commit(kEmpty + tile % kStages);
      for (int j = 0; ok && j < n; ++j, tile += 2) {
        for (int h = 0; ok && h < halves; ++h) {
          ok = wait(kPFull + h, p_phase >> h & 1u);
          if (ok && h == 0) full(tile + 1);
          if (!ok) break;
          p_phase ^= 1u << h;
          tc_fence_after();
          issue_pv(h, tile + 1, j % kChain == 0, leader);
          commit(kPv + h);
          if (h == halves - 1) commit(kEmpty + (tile + 1) % kStages);
          if (j + 1 < n) {
            if (h == 0) full(tile + 2);
            if (!ok) break;
            issue_s(h, tile + 2, leader);
            commit(kSFull + h);
            if (h == halves - 1) commit(kEmpty + (tile + 2) % kStages);
          }
        }
      }
    }
    if (!ok && leader) give_up();
    commit(kDrain);  // every MMA done before tensor and shared memory are given back
    mbar_wait(bar(kDrain), 0u, kDrainNs, nullptr);
  }

  // ---------------------------------------------------------------- softmax of one half
  // A warp has 16 rows of its half, a thread (g, t) = (lane / 4, lane % 4) of rows g and g + 8 the columns 8 b + 2 t + {0, 1}.

  // q's rows as hi + lo into shared memory; the scales of the thread's two rows.
  __device__ void split_q(const Piece& x, int half, int row0, float (&row_scale)[2]) const {
    const int lane = threadIdx.x & 31;
    constexpr int LANES = D / 4, PER = 32 / LANES, BATCH = 8;  // lanes of a row, rows at a time
    const int sub = lane / LANES, at = lane % LANES;
    const float sign = a.scale_log2 < 0.f ? -1.f : 1.f;  // the scale's sign goes into q
    float mine = 0.f;                                    // scale of row `lane` of the 16
    const uint32_t hi = smem + L::Q + (uint32_t)half * 2 * L::TILE + (uint32_t)(at >> 4) * L::PANEL;
    int64_t own = -1;  // where row `lane` begins
    if (lane < 16 && 128 * half + row0 + lane < x.rows) {
      const int fr = x.r0 + 128 * half + row0 + lane, token = fr / a.group;
      own = (int64_t)(x.row0 + token) * a.ldq + (int64_t)(x.h * a.group + fr % a.group) * D;
    }
    for (int r0 = 0; r0 < 16; r0 += BATCH * PER) {
      float4 v[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int64_t from = __shfl_sync(0xffffffffu, own, r0 + i * PER + sub);
        v[i] = from >= 0 ? __ldg(reinterpret_cast<const float4*>(a.q + from) + at) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        float top = fmaxf(fmaxf(fabsf(v[i].x), fabsf(v[i].y)), fmaxf(fabsf(v[i].z), fabsf(v[i].w)));
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int e = fp16_row_exponent(top);
        const float up = sign * pow2f(e);
#pragma unroll
        for (int p = 0; p < PER; ++p) {
          const int ep = __shfl_sync(0xffffffffu, e, p * LANES);
          if (lane == r0 + i * PER + p) mine = fabsf(a.scale_log2) * pow2f(-ep);
        }
        uint32_t h0, l0, h1, l1;
        split_f16(v[i].x * up, v[i].y * up, h0, l0);
        split_f16(v[i].z * up, v[i].w * up, h1, l1);
        const int r = row0 + r0 + i * PER + sub;  // of the half
        const uint32_t addr = hi + (uint32_t)r * 128 + (((uint32_t)(at & 15) / 2 ^ (r & 7)) << 4) + 8u * (at & 1);
        asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(addr), "r"(h0), "r"(h1) : "memory");
        asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(addr + L::TILE), "r"(l0), "r"(l1) : "memory");
      }
    }
    row_scale[0] = __shfl_sync(0xffffffffu, mine, lane >> 2);
    row_scale[1] = __shfl_sync(0xffffffffu, mine, (lane >> 2) + 8);
  }

  // A key tile's scores in tensor memory, and what they meet: the scales of the keys and values (int8), the marks of bad
  // values, the keys [lo, hi) that the thread's rows see, the rows' own scales.
  struct Scores {
    uint32_t ts, ks, vs, bad;
    int lo[2], hi[2];
    float row_scale[2];
  };
  static __device__ __forceinline__ void mul2(uint32_t& a, uint32_t& b, uint32_t x, uint32_t y) {
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tmul.rn.f32x2 p, p, q;\n\t"
        "mov.b64 {%0, %1}, p;\n\t}"
        : "+r"(a), "+r"(b)
        : "r"(x), "r"(y));
  }
  static __device__ __forceinline__ uint2 ld_shared8(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
    return v;
  }
  static __device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
  }
  static __device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
  }
  // The scores of keys 64 c .. 64 c + 63: times the keys' scales, the hidden ones -inf, the bad ones NaN.
  template <bool EDGE>
  static __device__ __forceinline__ void prepare(const Scores& x, int c, uint32_t (&s)[32]) {
    const int t = threadIdx.x & 3;
    if constexpr (I8) {
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const uint2 w = ld_shared8(x.ks + 256u * c + 32u * b + 8u * t);
        mul2(s[4 * b], s[4 * b + 1], w.x, w.y);
        mul2(s[4 * b + 2], s[4 * b + 3], w.x, w.y);
      }
    }
    if constexpr (EDGE) {
      if constexpr (!I8) {
        const uint2 bad = ld_shared8(x.bad + 8u * c);
        if (bad.x | bad.y) {
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            const uint32_t m = (b < 4 ? bad.x : bad.y) >> (8 * (b & 3) + 2 * t);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (m >> (i & 1) & 1u) s[4 * b + i] = 0x7fc00000u;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int r = i >> 1 & 1, j = 8 * (i >> 2) + (i & 1);  // of the thread's keys, from 64 c + 2 t on
        if (j < x.lo[r] - 64 * c - 2 * t || j >= x.hi[r] - 64 * c - 2 * t) s[i] = 0xff800000u;
      }
    }
  }
  // Scores to probabilities, in place in tensor memory.  Where a row's scores pass its maximum by more than kLazy it is
  // raised, and what was made with the old one is rescaled.  p = 2^(row_scale s + base); of a chunk of 32 columns the
  // high halves (times the values' scales) take the first 16, the low ones the others.  The scores of 64 keys are in
  // registers at a time, the first for the second time: all 128 beside p would be more than there are.
  template <bool EDGE, class Rescale>
  static __device__ __forceinline__ bool make_p(const Scores& x, float (&m)[2], float (&l)[2], const float (&down)[2],
                                                Rescale rescale_o) {
    const int t = threadIdx.x & 3;
    uint32_t s[2][32];
    tmem_ld_16x64(x.ts, s[0]);
    tmem_ld_16x64(x.ts + 64u, s[1]);
    tmem_ld_wait(s[0]);
    tmem_ld_wait(s[1]);
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      prepare<EDGE>(x, c, s[c]);
      float u[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < 32; i += 2)
        u[i >> 1 & 1] = max3(u[i >> 1 & 1], __uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1]));
      top[0] = fmaxf(top[0], u[0]);
      top[1] = fmaxf(top[1], u[1]);
    }
    bool raise[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      top[r] = quad_max(top[r]);
      top[r] = top[r] == -INFINITY ? top[r] : top[r] * x.row_scale[r];
      raise[r] = m[r] == -INFINITY ? top[r] > -INFINITY : top[r] > m[r] + kLazy;
    }
    if (__any_sync(0xffffffffu, raise[0] || raise[1])) {
      float f[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        f[r] = !raise[r] ? 1.f : (m[r] == -INFINITY ? 0.f : exp2_approx(m[r] - top[r]));
        l[r] *= f[r];
        if (raise[r]) m[r] = top[r];
      }
      if (!rescale_o(f[0], f[1])) return false;
    }
    unsigned long long scale2[2], base2[2], sum[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float base = kShift - (m[r] == -INFINITY ? 0.f : m[r]);
      scale2[r] = p2(x.row_scale[r], x.row_scale[r]);
      base2[r] = p2(base, base);
      sum[r] = p2(0.f, 0.f);
    }
    const unsigned long long minus1 = p2(-1.f, -1.f), zero2 = p2(-0.f, -0.f);
    auto put = [&](int c, uint32_t (&s)[32]) {
#pragma unroll
      for (int b0 = 0; b0 < 8; b0 += 4) {
        uint32_t hi[8], lo[8];
#pragma unroll
        for (int b = b0; b < b0 + 4; ++b) {
          uint2 w = make_uint2(0u, 0u);
          if constexpr (I8) w = ld_shared8(x.vs + 256u * c + 32u * b + 8u * t);
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float s0 = __uint_as_float(s[4 * b + 2 * r]), s1 = __uint_as_float(s[4 * b + 2 * r + 1]);
            float t0, t1;
            up2(fma2(p2(s0, s1), scale2[r], base2[r]), t0, t1);
            if constexpr (EDGE) {  // -inf times a scale of 0
              t0 = s0 == -INFINITY ? s0 : t0;
              t1 = s1 == -INFINITY ? s1 : t1;
            }
            unsigned long long p = p2(exp2_approx(t0), exp2_approx(t1));
            sum[r] = add2(sum[r], p);
            if constexpr (I8) {
              p = fma2(p, fma2(p2(__uint_as_float(w.x), __uint_as_float(w.y)), p2(down[r], down[r]), zero2), zero2);
              if constexpr (EDGE) {  // a hidden value's scale may be anything
                float a, b;
                up2(p, a, b);
                p = p2(s0 == -INFINITY ? 0.f : a, s1 == -INFINITY ? 0.f : b);
              }
            }
            float p0, p1, r0, r1;
            up2(p, p0, p1);
            const uint32_t h16 = pack_f16(p0, p1);
            const float2 h = unpack_f16(h16);
            up2(fma2(p2(h.x, h.y), minus1, p), r0, r1);
            hi[2 * (b - b0) + r] = h16;
            lo[2 * (b - b0) + r] = pack_f16(r0, r1);
          }
        }
        tmem_st_16x16(x.ts + 64u * c + 8u * b0, hi);
        tmem_st_16x16(x.ts + 64u * c + 8u * b0 + 16u, lo);
      }
    };
    put(1, s[1]);
    tmem_ld_16x64(x.ts, s[0]);
    tmem_ld_wait(s[0]);
    prepare<EDGE>(x, 0, s[0]);
    put(0, s[0]);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float p0, p1;
      up2(sum[r], p0, p1);
      l[r] += p0 + p1;
    }
    tmem_st_wait();
    return true;
  }

  __device__ void softmax(int half, Divided* divided) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int row0 = 32 * (warp & 3) + 16 * ((warp - 4) >> 2 & 1);  // the warp's rows of the half (its tensor memory lanes)
    const uint32_t lanes = (uint32_t)row0 << 16;
    const uint32_t ts = tmem + lanes + L::S + 128u * half, to = tmem + lanes + L::O + (uint32_t)D * half;
    bool ok = true;
    int step = 0;        // tiles of K so far
    uint32_t phase = 0;  // of this half's barriers: they complete once a key tile of a piece that has the half
    for (int k = 0; ok; ++k) {
      const Piece* place = piece(k, ok);
      if (!ok) break;
      const Piece& x = *place;
      const int n = x.tiles;
      if (n == 0) break;
      const bool whole = x.whole != 0;
      float* slot = a.slots + ((int64_t)blockIdx.x * 2 + (x.first == 0 ? 1 : 0)) * slot_floats<D>();
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      if (x.rows > 128 * half) {
        Scores sc;
        split_q(x, half, row0, sc.row_scale);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kQ + half));
        const int own0 = 128 * half + row0 + g;  // the thread's rows of the tile: own0, own0 + 8
        int ev[2] = {kMinExp, kMinExp}, ev_slot[2] = {kMinExp, kMinExp};
        float m_slot[2] = {-INFINITY, -INFINITY};
        bool has_slot = false;
        // O, plus the slot's sums (if any) brought into its units: into the slot, or at the end of a whole tile out.
        auto fold = [&](bool final) {
          const bool out = final && whole;
          float keep[2], f[2];
          float* dst[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            keep[r] = m_slot[r] == -INFINITY ? 1.f
                                             : exp2_approx(m_slot[r] - m[r]) * (I8 ? exp2_int(ev_slot[r] - ev[r]) : 1.f);
            const float unit = final && I8 ? exp2_int(ev[r]) : 1.f;
            f[r] = out ? (l[r] == 0.f ? 0.f : 1.0f / l[r]) * unit : unit;
            const int fr = x.r0 + own0 + 8 * r;
            dst[r] = own0 + 8 * r < x.rows ? a.out + (int64_t)(x.row0 + fr / a.group) * a.ldo +
                                                 (int64_t)(x.h * a.group + fr % a.group) * D + 2 * t
                                           : nullptr;
          }
          const bool add = !final && has_slot && __all_sync(0xffffffffu, keep[0] == 1.f && keep[1] == 1.f);
          // dims 8 b + 2 t, + 1 of a row in the slot
          auto at = [&](int b, int r) { return slot + ((2 * b + (t >> 1)) * kRows + own0 + 8 * r) * 4 + 2 * (t & 1); };
#pragma unroll 1
          for (int c = 0; c < D / 64; ++c) {
            uint32_t v[32];
            tmem_ld_16x64(to + 64u * c, v);
            tmem_ld_wait(v);
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
              float2 s[8];
              if (has_slot && !add) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  s[i] = __ldcg(reinterpret_cast<const float2*>(at(8 * c + h + (i >> 1), i & 1)));
              }
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int b = h + (i >> 1), r = i & 1;
                float2 w = make_float2(__uint_as_float(v[4 * b + 2 * r]), __uint_as_float(v[4 * b + 2 * r + 1]));
                if (add) {  // the units have not changed: added where it lies, without waiting
                  asm volatile("red.relaxed.gpu.global.add.v2.f32 [%0], {%1,%2};" ::"l"(at(8 * c + b, r)), "f"(w.x),
                               "f"(w.y)
                               : "memory");
                  continue;
                }
                if (has_slot) w = make_float2(fmaf(s[i].x, keep[r], w.x), fmaf(s[i].y, keep[r], w.y));
                w = make_float2(w.x * f[r], w.y * f[r]);
                if (!out) *reinterpret_cast<float2*>(at(8 * c + b, r)) = w;
                else if (dst[r]) *reinterpret_cast<float2*>(dst[r] + 64 * c + 8 * b) = w;
              }
            }
          }
          has_slot = true;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            m_slot[r] = m[r];
            ev_slot[r] = ev[r];
          }
        };
        for (int j = 0; j < n; ++j, ++step, phase ^= 1u) {
          const int j0 = x.j0 + j * kKeys;
          const bool edge = edge_of(x, j0);
          ok = wait(kSFull + half, phase);
          if (!ok) break;
          tc_fence_after();
          // The scales, or the marks, of this step's tiles.  A stage of V is not filled again before this half's p is
          // there; one of K may be, so its scales have barriers of their own.
          if (I8) ok = wait(kScale + (step & 1), (uint32_t)(step >> 1) & 1u);
          if (ok && (I8 || edge)) {
            const int tv = 2 * step + 1;
            ok = wait(kFull + tv % kStages, (uint32_t)(tv / kStages) & 1u);
          }
          if (!ok) break;
          sc.ts = ts;
          sc.ks = smem + L::KS + (uint32_t)(step & 1) * (kKeys * 4);
          sc.vs = smem + L::VS + (uint32_t)(step & 1) * (kKeys * 4);
          sc.bad = smem + L::BAD + 16u * (step & 1);
          if (edge) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {  // (rows past the last see all: nothing reads them)
              int lo = j0, hi = j0 + kKeys;
              if (own0 + 8 * r < x.rows)
                row_keys({0, x.n, x.len}, a.window, (x.r0 + own0 + 8 * r) / a.group, lo, hi);
              sc.lo[r] = lo - j0;
              sc.hi[r] = hi - j0;
            }
          }
          const bool fresh = j % kChain == 0;
          if (fresh && j > 0) {  // a chain is complete: O into the slot
            ok = wait(kPv + half, phase ^ 1u);
            if (!ok) break;
            tc_fence_after();
            fold(false);
          }
          auto rescale_o = [&](float f0, float f1) {
            if (fresh || !__any_sync(0xffffffffu, f0 != 1.f || f1 != 1.f)) return true;  // (or O starts anew)
            if (!wait(kPv + half, phase ^ 1u)) return false;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 64; ++c) {
              uint32_t v[32];
              tmem_ld_16x64(to + 64u * c, v);
              tmem_ld_wait(v);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * (i & 2 ? f1 : f0));
              tmem_st_16x64(to + 64u * c, v);
            }
            return true;
          };
          float down[2] = {1.f, 1.f};
          if constexpr (I8) {  // the largest value scale that a row sees sets its sums' units
            float big[2] = {0.f, 0.f};
            if (edge) {
              for (int i = 2 * t; i < kKeys; i += 8) {
                const uint2 w = ld_shared8(sc.vs + 4u * i);
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                  if (i >= sc.lo[r] && i < sc.hi[r]) big[r] = fmaxf(big[r], __uint_as_float(w.x));
                  if (i + 1 >= sc.lo[r] && i + 1 < sc.hi[r]) big[r] = fmaxf(big[r], __uint_as_float(w.y));
                }
              }
              big[0] = quad_max(big[0]);
              big[1] = quad_max(big[1]);
            } else {
              const uint4 w = ld_shared16(smem + L::VMAX + 16u * (step & 1));
              big[0] = big[1] = max3(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z));
            }
            float f[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int e = max(ev[r], min(kMaxExp, ((__float_as_int(big[r]) >> 23) & 255) - 127));
              f[r] = exp2_int(ev[r] - e);
              ev[r] = e;
              down[r] = exp2_int(-e);
            }
            ok = rescale_o(f[0], f[1]);
            if (!ok) break;
          }
          ok = edge ? make_p<true>(sc, m, l, down, rescale_o) : make_p<false>(sc, m, l, down, rescale_o);
          if (!ok) break;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(kPFull + half));
        }
        if (ok) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
          }
          ok = wait(kPv + half, phase ^ 1u);
        }
        if (ok) {
          tc_fence_after();
          fold(true);
          tc_fence_before();
          if (!whole && t == 0) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              slot[(int64_t)kRows * D + own0 + 8 * r] = m[r];
              slot[(int64_t)kRows * D + kRows + own0 + 8 * r] = l[r];
            }
          }
        }
      } else {
        step += n;
      }
      if (ok && !whole && x.first == 0 && warp == 4 && lane == 0)
        *divided = {x.last_block, x.h, x.row0, x.n, x.r0, x.rows};
      piece_done(k);
    }
    if (!ok && lane == 0) give_up();
  }
};

template <int D, bool I8>
__global__ void __launch_bounds__(kThreads, 1)
attention_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v, Divided* divided) {
  using L = Layout<D>;
  extern __shared__ __align__(1024) uint8_t base[];
  const uint32_t smem = smem_u32(base);
  volatile int* abort = reinterpret_cast<volatile int*>(base + L::MISC);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base + L::MISC + 8);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  if (threadIdx.x == 0) divided[blockIdx.x].last_block = 0;
  if (smem & 1023u) {  // the swizzled tiles need it; never taken where the declared alignment holds
    if (threadIdx.x == 0) atomicOr(a.batch.status, kStatusTimeout);
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem + L::BARS + 8u * (kFull + s), kProducers);  // a warp each
      mbar_init(smem + L::BARS + 8u * (kEmpty + s), 1);  // the MMAs
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(smem + L::BARS + 8u * (kScale + h), kProducers);
      mbar_init(smem + L::BARS + 8u * (kQ + h), 8);      // a softmax warp each
      mbar_init(smem + L::BARS + 8u * (kSFull + h), 1);
      mbar_init(smem + L::BARS + 8u * (kPFull + h), 8);
      mbar_init(smem + L::BARS + 8u * (kPv + h), 1);
    }
    mbar_init(smem + L::BARS + 8u * kDrain, 1);
    mbar_init(smem + L::BARS + 8u * kRaw, 1);
    for (int i = 0; i < kPieces; ++i) {
      mbar_init(smem + L::BARS + 8u * (kPieceFull + i), 1);
      mbar_init(smem + L::BARS + 8u * (kPieceFree + i), kThreads / 32 - 1);  // every warp but warp 1
    }
    *abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async_smem();
  }
  if (warp == 0) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
  Run run(a, reinterpret_cast<int64_t*>(base));  // the prefix sums lie where the tiles will
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const Kernel<D, I8> k{a, map_k, map_v, smem, __shfl_sync(0xffffffffu, *tmem_slot, 0), abort,
                         reinterpret_cast<Piece*>(base + L::PIECES)};
  if (warp == 0) k.issuer();
  else if (warp < 4) k.producer(run);
  else k.softmax((warp - 4) >> 3, divided + blockIdx.x);
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(k.tmem, kTmemCols);
  }
}

// The pieces of the divided tiles, joined in the order of their blocks: blockIdx.x the block in whose run the tile
// begins, blockIdx.y a part of its (row, dims).  A warp takes 32 rows and 4 dims of each.
constexpr int kJoinParts = 8, kJoinThreads = 256;
template <int D>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const AttnArgs a, const Divided* divided) {
  const Divided x = divided[blockIdx.x];
  const int c0 = blockIdx.x, c1 = x.last_block;
  if (c1 <= c0) return;
  const int lane = threadIdx.x & 31;
  const int warps = kJoinParts * (kJoinThreads / 32), first = blockIdx.y * (kJoinThreads / 32) + (threadIdx.x >> 5);
  for (int task = first; task < (x.rows + 31) / 32 * (D / 4); task += warps) {
    const int row = task / (D / 4) * 32 + lane, d4 = task % (D / 4);
    if (row >= x.rows) continue;
    auto slot = [&](int c) { return a.slots + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * slot_floats<D>(); };
    float m = -INFINITY;
    for (int c = c0; c <= c1; ++c) m = fmaxf(m, __ldg(slot(c) + (int64_t)kRows * D + row));
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll 4
    for (int c = c0; c <= c1; ++c) {
      const float* s = slot(c);
      const float mc = __ldg(s + (int64_t)kRows * D + row), lc = __ldg(s + (int64_t)kRows * D + kRows + row);
      const float4 p = __ldg(reinterpret_cast<const float4*>(s) + d4 * kRows + row);
      const float w = mc == -INFINITY ? 1.f : exp2_approx(mc - m);  // without keys: zeros, or NaN
      v = make_float4(fmaf(p.x, w, v.x), fmaf(p.y, w, v.y), fmaf(p.z, w, v.z), fmaf(p.w, w, v.w));
      l = fmaf(lc, w, l);
    }
    const float f = l == 0.f ? 0.f : 1.0f / l;
    const int fr = x.r0 + row;
    *reinterpret_cast<float4*>(a.out + (int64_t)(x.row0 + fr / a.group) * a.ldo +
                               (int64_t)(x.head * a.group + fr % a.group) * D + 4 * d4) =
        make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
  }
}

template <int D, bool I8>
spl_status launch(const AttnArgs& a, int blocks, cudaStream_t stream) {
  constexpr uint32_t smem = Layout<D>::SMEM;
  if (cudaFuncSetAttribute(attention_tc_kernel<D, I8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) !=
      cudaSuccess)
    return SPL_ECUDA;
  Divided* divided = reinterpret_cast<Divided*>(a.slots + (int64_t)blocks * 2 * slot_floats<D>());
  CUtensorMap map_k = {}, map_v = {};
  if (!I8) {
    const int64_t slots = (int64_t)a.cache.pages * a.cache.heads << a.cache.page_shift;
    const int box = std::min(kKeys, 1 << a.cache.page_shift);
    if (slots > INT32_MAX - kKeys) return SPL_ESHAPE;  // rows of a copy's coordinates
    if (!tma_panel_map(&map_k, a.cache.k, slots, D, box) || !tma_panel_map(&map_v, a.cache.v, slots, D, box))
      return SPL_ECUDA;
  }
  attention_tc_kernel<D, I8><<<blocks, kThreads, smem, stream>>>(a, map_k, map_v, divided);
  const spl_status st = launch_status();
  if (st != SPL_OK) return st;
  attention_join_kernel<D><<<dim3(blocks, kJoinParts), kJoinThreads, 0, stream>>>(a, divided);
  return launch_status();
}

}  // namespace

size_t attention_tc_bytes(int head_dim, int blocks) {
  const int64_t floats = head_dim == 128 ? slot_floats<128>() : slot_floats<64>();
  return (size_t)blocks * (2 * floats * sizeof(float) + sizeof(Divided));
}

spl_status run_attention_tc(const AttnArgs& a, int head_dim, bool i8, int blocks, cudaStream_t stream) {
  if (head_dim == 128) return i8 ? launch<128, true>(a, blocks, stream) : launch<128, false>(a, blocks, stream);
  return i8 ? launch<64, true>(a, blocks, stream) : launch<64, false>(a, blocks, stream);
}

}  // namespace spl
