// Attention of many rows over a paged cache on the 5th-generation tensor cores (chunks of new tokens, prefill).
//
// o = sum_j softmax_j(scale q . k_j) v_j over tiles of 128 rows and 128 keys:
//   S = q_hi K^T + q_lo K^T        q = (hi + lo) 2^-e in binary16, a row's largest entry in [2^14, 2^15)
//   p = 2^(scale log2(e) S - m)    m the row's running maximum, l the running total, both fp32
//   O = O 2^(m_old - m) + p_hi V + p_lo V
// The stored keys and values are exact in binary16, so two products instead of one give fp32 accuracy, and the kernel
// is bound by the tensor pipe: 4 products of 128 x 128 x dim a tile.  S of the next tile is made before O of this one,
// so that the softmax of a tile runs beside the products of its neighbours.  Roles:
//   warp 0       MMA issuer.
//   warp 1       hands out the block's pieces of tiles and loads K and V tiles from the pages, by TMA: binary16 in the
//                128-byte-swizzled layout that the MMAs read, a box a page; int8 as it is stored, beside.
//   warps 2-7    int8: widen the tiles to binary16, in that layout.  binary16: look over the values of tiles at an edge of
//                what the rows see (stale ones become zeros).
//   warps 8-11   the sums: O, out of tensor memory, a thread a row, into the workspace or the output.
//   warps 12-19  softmax, 16 rows a warp and four threads a row; also q's split.
// Tensor memory: two places of S and two of O.  p overwrites S: a chunk of 32 scores becomes 16 columns of p_hi and 16 of
// p_lo, the A operand of the second product.  p is held as 2^9 p: the low half keeps an absolute 2^-33 of the row's
// largest.  The running maximum is raised only where it would let p pass 2^5, so that O is seldom rescaled.  The tensor
// core truncates as it accumulates, and an unbroken chain's bias grows with its length: after kChain tiles O goes on in
// its other place while the sums' warps add the first to an fp32 sum in the workspace, rounding to nearest.
// Divided tiles are joined by a second, small launch over all SMs.  Keys on pages outside the pool are hidden: in place of
// a copy there are zeros (int8: what was there), and their scores are overwritten with -inf.
// Every wait is bounded; on expiry the status word is raised and the block leaves with its copies and MMAs done.
// Measured with 32 query heads on 8 of 128 dims, 2048 rows over 12049 keys: binary16 469 us, 0.9 of the instructions'
// 2560 clocks a tile (S takes 96 an instruction, both its operands being in shared memory, O 64); int8 696 us, bound by
// the widening and shared memory; 64 dims 397 and 653 us, bound by the softmax.  24 heads on 8, 512 rows over themselves
// 21 us: some 14 us of one tile's latency, launches and the join.

#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "attention.cuh"
#include "noise.cuh"  // packed fp32 pairs
#include "ptx.cuh"

namespace spl {
namespace {

constexpr int kHelpers = 6, kSoftmax = 8;  // warps
constexpr int kThreads = 32 * (2 + kHelpers + 4 + kSoftmax);
constexpr int kRows = 128, kKeys = 128;
constexpr int kChain = 4;        // key tiles of an accumulation chain of O (512 keys)
constexpr float kShift = 9.0f;   // p is held as 2^kShift p
constexpr float kLazy = 5.0f;    // and may reach 2^(kShift + kLazy), times a scale below 2, before the maximum is raised
constexpr int kMinExp = -100, kMaxExp = 126;
constexpr int kSteps = 4;        // key tiles whose scales or marks have a place (see the barriers of the producer)

// Barriers by index: kFull, kEmpty a stage; kRawFull, kRawEmpty a stage of int8 tiles as stored; kScale a place of K's
// scales; kQ a piece's q; kSFull, kPFull a place of S and the p in it (whose waiter may be a tile behind); kPv a tile's
// product with V; kOFull, kOFree, kMFull a place of O: its chain is complete, has been added up, its rows' maxima are
// there; kEdge the copies of V's edge tiles; kPieceFull, kPieceFree a piece's place.
enum {
  kFull = 0, kEmpty = 5, kScale = 10, kQ = 14, kSFull = 15, kPFull = 17, kPv = 19, kOFull = 20, kOFree = 22, kMFull = 24,
  kDrain = 26, kEdge = 27, kPieceFull = 28, kPieceFree = 30, kRawFull = 32, kRawEmpty = 35, kBars = 38
};

// A block's piece of a tile, as warp 1 hands it to the others (two in shared memory, in turn).
struct alignas(16) Piece {
  int tiles;           // key tiles, 0 after the last piece
  int j0;              // first key of the first
  int key_lo, key_hi;  // keys that some row sees
  int all_lo, all_hi;  // keys that every row sees
  int b, h;            // sequence, key head
  int row0, len, pos0; // the sequence's first row, length and first row's position
  int r0, rows;        // rows of the tile among the sequence's rows of the key head
  int first;           // the first tile's index among the whole tile's
  int whole;           // the piece is the whole tile
  int last_block;      // the block that has the whole tile's end
  int plain_hi;        // all_hi, or where the first key tile with a page outside the pool begins, as soon as it is met
};
constexpr int kPieces = 2;

// D columns of binary16 in panels of 64 (128 bytes, 128-byte swizzle): a panel of 128 rows is 16 KB.
template <int D, bool I8>
struct Layout {
  static constexpr int STAGES = I8 ? 3 : 5, RAW_STAGES = 3;
  static constexpr int PANELS = D / 64;
  static constexpr uint32_t PANEL = 128 * 128;
  static constexpr uint32_t TILE = PANELS * PANEL;         // q_hi or q_lo; a K or V tile
  static constexpr uint32_t Q = 0, KV = 2 * TILE;          // [q_hi, q_lo], stages
  // int8 tiles as stored, their scales and the mask of the blocks of 16 keys that were copied
  static constexpr uint32_t RAW = KV + STAGES * TILE, RAW_SCALE = kKeys * D, RAW_MASK = RAW_SCALE + kKeys * 4;
  static constexpr uint32_t RAW_STAGE = RAW_MASK + 16;
  static constexpr uint32_t AUX = RAW + (I8 ? RAW_STAGES * RAW_STAGE : 0);
  // rows' maxima and totals of two chains (int8: and exponents); int8: scales of K and V, largest of V's a warp; binary16:
  // marks of bad values; each for kSteps tiles
  static constexpr uint32_t M = AUX, LT = M + 2 * kRows * 4, EV = LT + 2 * kRows * 4, KS = EV + (I8 ? 2 * kRows * 4 : 0);
  static constexpr uint32_t VS = KS + (I8 ? kSteps * kKeys * 4 : 0), VMAX = VS + (I8 ? kSteps * kKeys * 4 : 0);
  static constexpr uint32_t BAD = VMAX + (I8 ? kSteps * 32 : 0), BARS = BAD + (I8 ? 0 : kSteps * 16);
  static constexpr uint32_t PIECES = BARS + 8 * kBars, MISC = PIECES + kPieces * sizeof(Piece);
  // boxes of a tile whose page is outside the pool; 16 bytes of no marks
  static constexpr uint32_t GONE = MISC + 16, ZERO = GONE + 4 * kSteps, SMEM = ZERO + 16;
  static_assert(BARS % 8 == 0 && PIECES % 16 == 0 && SMEM <= 232448, "227 KB of dynamic shared memory per block");
  static_assert(kMaxSeqs * kPrefixBytes + 8192 <= AUX, "the prefix sums fit where the tiles go");
  static constexpr uint32_t S = 0, O = 256;                // tensor memory columns (+ 128 and + D for the other place)
  static constexpr uint32_t IDESC_S = make_idesc(0, 128, kKeys);
  static constexpr uint32_t IDESC_O = make_idesc(0, 128, D) | (1u << 16);  // B: the values, dims contiguous
};
constexpr uint32_t kTmemCols = 512;

// A workspace slot: sums as [dim / 4][128 rows][4], then the rows' maxima and totals, and (int8) the exponents of the sums'
// units, which the totals do not share.
constexpr int kTcStats = kSlotStats + 1;
template <int D>
constexpr int64_t slot_floats() {
  return (int64_t)kRows * (D + kTcStats);
}

// A divided tile that begins in a block's run, for the join.
struct Divided {
  int last_block;  // 0: none (a divided tile never ends in block 0)
  int head, row0, r0, rows;
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
__device__ __forceinline__ void st_shared4(uint32_t addr, uint32_t v) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ void st_global32(float* p, float4 a, float4 b) {
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(a.x), "f"(a.y), "f"(a.z), "f"(a.w),
               "f"(b.x), "f"(b.y), "f"(b.z), "f"(b.w)
               : "memory");
}

template <int D, bool I8, bool TREE>
struct Kernel {
  using Run = AttnRun<kRows, kKeys, kThreads, TREE>;
  using L = Layout<D, I8>;
  static constexpr int STAGES = L::STAGES;
  const AttnArgs& a;
  const CUtensorMap &map_k, &map_v;  // F16: the stored vectors as [slots, D]
  uint32_t smem;                     // shared address of the aligned base
  uint32_t tmem;
  volatile int* abort;
  Piece* pieces;

  __device__ uint32_t bar(int i) const { return smem + L::BARS + 8u * i; }
  __device__ bool wait(int i, uint32_t parity, unsigned long long ns = kWaitNs) const {
    return __all_sync(0xffffffffu, mbar_wait_soon(bar(i), parity, ns, abort));
  }
  // For a warp that may wait while others work on all of `tiles` key tiles (1.4 to 2.4 us each).
  static __device__ unsigned long long wait_ns(int tiles) { return kWaitNs + 20000ull * (unsigned)tiles; }
  // One arrival for the warp, after all its lanes' work.
  __device__ void arrive(int i) const {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar(i));
  }
  __device__ void give_up() const {
    *abort = 1;
    atomicOr(a.batch.status, kStatusTimeout);
  }
  // Whether some row of the tile sees only a part of the 128 keys from j0 on.
  static __device__ bool edge_of(const Piece& x, int j0) { return j0 < x.all_lo || j0 + kKeys > x.all_hi; }
  // The k-th piece, when it is there; a warp that has done with it says so (it may not read it afterwards).
  __device__ const Piece* piece(int k, bool& ok, unsigned long long ns = kWaitNs) const {
    ok = ok && wait(kPieceFull + k % kPieces, (uint32_t)(k / kPieces) & 1u, ns);
    return pieces + k % kPieces;
  }
  __device__ void piece_done(int k) const { arrive(kPieceFree + k % kPieces); }
  // Warp 1: the k-th piece of the run (or its end) for all.
  __device__ bool hand_out(const Run& run, int k) const {
    if (k >= kPieces && !wait(kPieceFree + k % kPieces, (uint32_t)(k / kPieces - 1) & 1u)) return false;
    if ((threadIdx.x & 31) == 0) {
      Piece& y = pieces[k % kPieces];
      y.tiles = 0;
      if (run.busy()) {
        const AttnTile& x = run.x;
        y = {run.last() - run.first, (x.unit0 + run.first) * kKeys, x.key_lo, x.key_hi, x.all_lo, x.all_hi, x.b, x.h,
             x.s.row0, x.s.len, x.s.pos0, x.r0, x.rows, run.first, run.whole() ? 1 : 0, run.last_block(), x.all_hi};
      }
      mbar_arrive(bar(kPieceFull + k % kPieces));
    }
    __syncwarp();
    return true;
  }

  // ---------------------------------------------------------------- loads
  // A piece's tiles are loaded in the order in which the MMAs take them: K0, K1, V0, K2, V1, ..., V(n-1).  Scales and marks
  // of a tile lie in one of kSteps places: the place of step s is written again for step s + 4, whose tile goes into a
  // stage that was freed by an MMA issued after p of step s had arrived, so its softmax has read them.

  // The u-th of that order's 2 n tiles: true for V, and the step within the piece.
  static __device__ bool in_order(int i, int n, int& u) {
    const bool v = i == 2 * n - 1 || (i > 0 && (i & 1) == 0);
    u = i == 0 ? 0 : (v ? (i == 2 * n - 1 ? n - 1 : i / 2 - 1) : (i + 1) / 2);
    return v;
  }
  // The page of the first 16 keys from j on that some row sees of the `size` from there (in one page), kUnseen if there is
  // none, kGone if its id is outside the pool.
  static constexpr int kUnseen = -1, kGone = -2;
  __device__ int page_of(const Piece& x, int j, int size) const {
    const int from = max(j, x.key_lo & ~15);
    if (from >= min(j + size, x.key_hi)) return kUnseen;
    const int page = paged_page(a.cache, a.batch, x.b, from);
    return page >= 0 ? page : kGone;
  }
  static __device__ __forceinline__ void mbar_arrive_more(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
  }

  struct Loads {                                 // so far, of the whole run
    int tile = 0, step = 0;                      // tiles of K and V, of K
    int edge_tile = -STAGES, edge_phase = 0;     // V's last edge tile; the parity of the next one's copy
  };

  // Warp 1.
  __device__ void loader(Run& run) const {
    bool ok = true;
    Loads y;
    for (int k = 0; ok; ++k) {
      ok = hand_out(run, k);
      if (run.busy()) run.next();
      const Piece* place = piece(k, ok);
      if (!ok) break;
      const Piece x = *place;  // (in registers)
      const int n = x.tiles;
      if (n == 0) break;
      ok = I8 ? load_i8(x, pieces + k % kPieces, y) : load_f16(x, pieces + k % kPieces, y);
      y.step += n;
      piece_done(k);
    }
    if (!ok) {
      if ((threadIdx.x & 31) == 0) give_up();
      // no copy in flight when the block leaves
      constexpr int first = I8 ? kRawFull : kFull, stages = I8 ? L::RAW_STAGES : STAGES;
      for (int t = max(0, y.tile - stages); t <= y.tile; ++t)
        mbar_wait(bar(first + t % stages), (uint32_t)(t / stages) & 1u, kDrainNs, nullptr);
    }
  }
  // The first slots of a piece's boxes (a page's tokens, at most 128), those of kAhead tiles in a lane each, kUnseen where no
  // row sees any key of them, or kGone; those of the next kAhead tiles are looked up meanwhile.
  static constexpr int kAhead = 4;
  struct Boxes {
    const Kernel& k;
    const Piece& x;
    int box, per_tile, shift;
    uint64_t policy = l2_evict_last();  // other tiles of rows read the same keys
    int64_t now, next;
    __device__ Boxes(const Kernel& kernel, const Piece& piece) : k(kernel), x(piece) {
      shift = k.a.cache.page_shift;
      box = min(kKeys, 1 << shift);
      per_tile = kKeys / box;
      now = look_up(0);
      next = look_up(kAhead);
    }
    __device__ int64_t look_up(int u0) const {
      const int lane = threadIdx.x & 31, u = u0 + lane / per_tile, j = x.j0 + u * kKeys + lane % per_tile * box;
      const int page = lane < kAhead * per_tile && u < x.tiles ? k.page_of(x, j, box) : kUnseen;
      return page >= 0 ? ((((int64_t)page * k.a.cache.heads + x.h) << shift) + (j & ((1 << shift) - 1))) : page;
    }
    // The slot of the lane's box of tile u, which is in the window.
    __device__ int64_t of(int u) const {
      const int lane = threadIdx.x & 31, at = u % kAhead * per_tile + lane;
      const int64_t a = __shfl_sync(0xffffffffu, now, at & 31), b = __shfl_sync(0xffffffffu, next, at & 31);
      return lane >= per_tile ? kUnseen : (u >= base + kAhead ? b : a);
    }
    int base = 0;
    __device__ void advance() {  // past the last tile of the window's first half
      base += kAhead;
      now = next;
      next = look_up(base + kAhead);
    }
  };
  __device__ bool load_f16(const Piece& x, Piece* place, Loads& y) const {
    const int lane = threadIdx.x & 31, n = x.tiles;
    Boxes boxes(*this, x);
    const int none = (int)((int64_t)a.cache.pages * a.cache.heads << boxes.shift);  // past the pool: filled with zeros
    bool ok = true;
    for (int i = 0; ok && i < 2 * n; ++i, ++y.tile) {
      int u;
      const bool v = in_order(i, n, u), edge = v && edge_of(x, x.j0 + u * kKeys);
      const int stage = y.tile % STAGES, to = edge ? kEdge : kFull + stage;
      // No second copy on kEdge while a warp may still wait for the first (those that freed its stage do not).
      if (edge && y.tile - y.edge_tile < STAGES)
        ok = wait(kFull + y.edge_tile % STAGES, (uint32_t)(y.edge_tile / STAGES) & 1u);
      if (edge) y.edge_tile = y.tile;
      if (ok && y.tile >= STAGES) ok = wait(kEmpty + stage, (uint32_t)(y.tile / STAGES - 1) & 1u);
      if (!ok) break;
      if (lane == 0) mbar_expect_tx(bar(to), L::TILE);
      const int64_t slot = boxes.of(u);
      if (lane < boxes.per_tile) {
        const uint32_t dst = smem + L::KV + (uint32_t)stage * L::TILE + (uint32_t)(lane * boxes.box) * 128u;
#pragma unroll
        for (int p = 0; p < L::PANELS; ++p)
          tma_load_2d(dst + p * L::PANEL, v ? &map_v : &map_k, bar(to), 64 * p, slot >= 0 ? (int)slot : none, boxes.policy);
      }
      if (!v) mark_gone(place, smem + L::GONE + 4u * ((y.step + u) % kSteps), slot, x.j0 + u * kKeys);
      if (lane == 0 && !edge) mbar_arrive_more(bar(to), kHelpers - 1);
      __syncwarp();
      if (v && u % kAhead == kAhead - 1) boxes.advance();
    }
    return ok;
  }
  __device__ bool load_i8(const Piece& x, Piece* place, Loads& y) const {
    const int lane = threadIdx.x & 31, n = x.tiles;
    Boxes boxes(*this, x);
    bool ok = true;
    for (int i = 0; ok && i < 2 * n; ++i, ++y.tile) {
      int u;
      const bool v = in_order(i, n, u);
      const int stage = y.tile % L::RAW_STAGES;
      if (y.tile >= L::RAW_STAGES) ok = wait(kRawEmpty + stage, (uint32_t)(y.tile / L::RAW_STAGES - 1) & 1u);
      if (!ok) break;
      const int64_t slot = boxes.of(u);
      const uint32_t raw = smem + L::RAW + (uint32_t)stage * L::RAW_STAGE, full = bar(kRawFull + stage);
      const uint32_t mask = __ballot_sync(0xffffffffu, slot >= 0);  // of boxes
      if (!v) mark_gone(place, raw + L::RAW_MASK + 4u, slot, x.j0 + u * kKeys);
      if (lane == 0) {
        st_shared4(raw + L::RAW_MASK, mask);
        mbar_expect_tx(full, (uint32_t)(__popc(mask) * boxes.box * (D + 4)));
      }
      __syncwarp();
      if (slot >= 0) {
        bulk_load(raw + (uint32_t)(lane * boxes.box) * D, static_cast<const char*>(v ? a.cache.v : a.cache.k) + slot * D,
                  (uint32_t)boxes.box * D, full, boxes.policy);
        bulk_load(raw + L::RAW_SCALE + (uint32_t)(lane * boxes.box) * 4u, (v ? a.cache.v_scale : a.cache.k_scale) + slot,
                  (uint32_t)boxes.box * 4u, full, boxes.policy);
      }
      __syncwarp();
      if (v && u % kAhead == kAhead - 1) boxes.advance();
    }
    return ok;
  }

  // Warps 2-7.
  __device__ void helper() const {
    bool ok = true;
    Loads y;
    int last = 0;  // tiles of the piece before: binary16 has nothing to do with most of them
    for (int k = 0; ok; ++k) {
      const Piece* place = piece(k, ok, wait_ns(last));
      if (!ok) break;
      const Piece& x = *place;
      const int n = x.tiles;
      if (n == 0) break;
      for (int i = 0; ok && i < 2 * n; ++i, ++y.tile) {
        int u;
        const bool v = in_order(i, n, u);
        if constexpr (I8) {
          ok = widen(y.tile, y.step + u, v);
        } else if (v && edge_of(x, x.j0 + u * kKeys)) {
          ok = wait(kEdge, (uint32_t)y.edge_phase, wait_ns(n));
          if (!ok) break;
          y.edge_phase ^= 1;
          look_over(x, x.j0 + u * kKeys, smem + L::KV + (uint32_t)(y.tile % STAGES) * L::TILE, y.step + u);
          arrive(kFull + y.tile % STAGES);
        }
      }
      y.step += n;
      last = n;
      piece_done(k);
    }
    if (!ok && (threadIdx.x & 31) == 0) give_up();
  }
  // Values of an edge tile, a lane a key: those that no row sees become zeros; an infinity or NaN in one that only
  // some rows see becomes 0 and is marked.
  __device__ void look_over(const Piece& x, int j0, uint32_t base, int step) const {
    const int lane = threadIdx.x & 31, word = (threadIdx.x >> 5) - 2;
    if (word < kKeys / 32) {
      const int key = 32 * word + lane, j = j0 + key;
      const bool seen = j >= x.key_lo && j < x.key_hi;
      bool bad = false;
#pragma unroll 8
      for (int c = 0; c < D / 8; ++c) {
        const uint32_t at = base + (c >> 3) * L::PANEL + key * 128 + (((c & 7) ^ (key & 7)) << 4);
        const uint4 v = ld_shared16(at);
        const bool special = f16_special(v.x) || f16_special(v.y) || f16_special(v.z) || f16_special(v.w);
        bad |= special;
        if (special || !seen) st_shared16(at, make_uint4(0u, 0u, 0u, 0u));
      }
      const unsigned marks = __ballot_sync(0xffffffffu, bad && seen);
      if (lane == 0)
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(smem + L::BAD + 16u * (step % kSteps) + 4u * word), "r"(marks)
                     : "memory");
      fence_proxy_async_smem();
    }
  }
  // A tile of int8 to binary16 in the MMAs' layout, and its scales (of keys that were not copied K's 1, V's 0).  A thread has
  // the same 16 dims of every KEY_STEP-th key; all its loads run side by side.
  __device__ bool widen(int tile, int step, bool v) const {
    constexpr int PARTS = D / 16, KEY_STEP = 32 * kHelpers / PARTS, PER = (kKeys + KEY_STEP - 1) / KEY_STEP;
    const int i = threadIdx.x - 64, lane = i & 31, stage = tile % STAGES, raw_stage = tile % L::RAW_STAGES;
    const uint32_t raw = smem + L::RAW + (uint32_t)raw_stage * L::RAW_STAGE;
    const int part = i % PARTS, key0 = i / PARTS, c0 = (2 * part) & 7;  // two chunks of 8 values
    const uint32_t panel = smem + L::KV + (uint32_t)stage * L::TILE + (uint32_t)(part >> 2) * L::PANEL;
    if (!wait(kRawFull + raw_stage, (uint32_t)(tile / L::RAW_STAGES) & 1u)) return false;
    uint4 q[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (key0 + KEY_STEP * k < kKeys) q[k] = ld_shared16(raw + (uint32_t)(key0 + KEY_STEP * k) * D + 16u * part);
    float scale = 0.f;
    uint32_t mask = 0u, gone = 0u;
    if (i < kKeys) {
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(gone) : "r"(raw + L::RAW_MASK + 4u));
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(mask) : "r"(raw + L::RAW_MASK));
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(scale) : "r"(raw + L::RAW_SCALE + 4u * i));
      if (!(mask >> (i >> a.cache.page_shift) & 1u)) scale = v ? 0.f : 1.f;  // (a hidden score stays -inf)
    }
    arrive(kRawEmpty + raw_stage);
    if (tile >= STAGES && !wait(kEmpty + stage, (uint32_t)(tile / STAGES - 1) & 1u)) return false;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int key = key0 + KEY_STEP * k;
      if (key >= kKeys) break;
      const uint32_t w[4] = {q[k].x ^ 0x80808080u, q[k].y ^ 0x80808080u, q[k].z ^ 0x80808080u, q[k].w ^ 0x80808080u};
      const uint32_t row = panel + key * 128;
      st_shared16(row + ((c0 ^ (key & 7)) << 4), make_uint4(i8_pair(w[0], 0x4140u), i8_pair(w[0], 0x4342u),
                                                            i8_pair(w[1], 0x4140u), i8_pair(w[1], 0x4342u)));
      st_shared16(row + (((c0 + 1) ^ (key & 7)) << 4), make_uint4(i8_pair(w[2], 0x4140u), i8_pair(w[2], 0x4342u),
                                                                  i8_pair(w[3], 0x4140u), i8_pair(w[3], 0x4342u)));
    }
    if (i < kKeys) {
      asm volatile("st.shared.f32 [%0], %1;" ::"r"(smem + (v ? L::VS : L::KS) + (uint32_t)(step % kSteps) * (kKeys * 4) +
                                                   4u * i),
                   "f"(scale)
                   : "memory");
      if (v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) scale = fmaxf(scale, __shfl_xor_sync(0xffffffffu, scale, o));
        if (lane == 0)
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(smem + L::VMAX + 32u * (step % kSteps) + 4u * (i >> 5)),
                       "f"(scale)
                       : "memory");
      }
    }
    if (!v && i == 0) st_shared4(smem + L::GONE + 4u * (step % kSteps), gone);
    fence_proxy_async_smem();
    arrive(kFull + stage);
    if (!v && lane == 0) mbar_arrive(bar(kScale + step % kSteps));
    return true;
  }

  // ---------------------------------------------------------------- MMA issuer
  __device__ void issue_s(int place, int tile, uint32_t leader) const {
    const uint32_t q = sdesc_lo(smem + L::Q);
    const uint32_t k = sdesc_lo(smem + L::KV + (uint32_t)(tile % STAGES) * L::TILE);
    const uint32_t d = tmem + L::S + 128u * place;
    // The low halves first: each product truncates its sum, which is still small for them.
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const int s = i % (D / 16);
      const uint32_t off = ((uint32_t)(s / 4) * L::PANEL + (uint32_t)(s % 4) * 32u) >> 4;
      mma_ss(d, q + off + (i < D / 16 ? L::TILE >> 4 : 0u), k + off, kSdescHi128, L::IDESC_S, i > 0 ? 1u : 0u, leader);
    }
  }
  __device__ void issue_pv(int place, int o, int tile, bool fresh, uint32_t leader) const {
    const uint32_t v = sdesc_lo_mn(smem + L::KV + (uint32_t)(tile % STAGES) * L::TILE);
    const uint32_t p = tmem + L::S + 128u * place, d = tmem + L::O + (uint32_t)D * o;
#pragma unroll
    for (int i = 0; i < kKeys / 8; ++i) {
      const int s = i % (kKeys / 16);
      const uint32_t at = p + 32u * (s / 2) + 8u * (s % 2) + (i < kKeys / 16 ? 16u : 0u);
      mma_ts(d, at, v + ((uint32_t)(s * 16 * 128) >> 4), kSdescHi128, L::IDESC_O, fresh && i == 0 ? 0u : 1u, leader);
    }
  }
  __device__ void issuer() const {
    const uint32_t leader = elect_one();
    bool ok = true;
    int tile = 0, step = 0, chain = 0;
    auto commit = [&](int i) {
      if (leader) mma_commit(bar(i));
      __syncwarp();
    };
    auto full = [&](int t) {
      ok = ok && wait(kFull + t % STAGES, (uint32_t)(t / STAGES) & 1u);
      tc_fence_after();
    };
    // Loop bounds come through shuffles: the compiler then knows them, and all that the descriptors are made of, to be
    // the same in every lane.
    for (int k = 0; ok; ++k) {
      const Piece* x = piece(k, ok);
      if (!ok) break;
      const int n = __shfl_sync(0xffffffffu, x->tiles, 0);
      piece_done(k);
      if (n == 0) break;
      ok = wait(kQ, (uint32_t)k & 1u);
      full(tile);
      if (!ok) break;
      issue_s(step & 1, tile, leader);
      if (leader) mbar_arrive(bar(kSFull + (step & 1)));
      commit(kSFull + (step & 1));
      commit(kEmpty + tile % STAGES);
      ++tile;
      for (int j = 0; j < n; ++j, ++step) {
        if (j + 1 < n) {
          full(tile);
          if (!ok) break;
          issue_s((step + 1) & 1, tile, leader);
          if (leader) mbar_arrive(bar(kSFull + ((step + 1) & 1)));
          commit(kSFull + ((step + 1) & 1));
          commit(kEmpty + tile % STAGES);
          ++tile;
        }
        const bool fresh = j % kChain == 0;
        if (fresh && chain >= 2) ok = wait(kOFree + (chain & 1), (uint32_t)(chain / 2 - 1) & 1u);
        ok = ok && wait(kPFull + (step & 1), (uint32_t)(step >> 1) & 1u);
        full(tile);
        if (!ok) break;
        issue_pv(step & 1, chain & 1, tile, fresh, leader);
        commit(kPv);
        commit(kEmpty + tile % STAGES);
        ++tile;
        if (j % kChain == kChain - 1 || j == n - 1) {
          commit(kOFull + (chain & 1));
          ++chain;
        }
      }
    }
    if (!ok && leader) give_up();
    commit(kDrain);  // every MMA done before tensor and shared memory are given back
    mbar_wait(bar(kDrain), 0u, kDrainNs, nullptr);
  }

  // ---------------------------------------------------------------- the sums
  // O of a chain, a thread a row, plus the sums so far: into the slot, or at the end of a whole tile out.
  __device__ void sums(Divided* divided) const {
    const int own = 32 * ((threadIdx.x >> 5) & 3) + (threadIdx.x & 31);
    const uint32_t lanes = (uint32_t)(own & 96) << 16;
    const bool wide = a.ldo % 8 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
    bool ok = true;
    int chain = 0;
    for (int k = 0; ok; ++k) {
      const Piece* place = piece(k, ok);
      if (!ok) break;
      const Piece& x = *place;
      const int n = x.tiles;
      if (n == 0) break;
      float* slot = a.slots + ((int64_t)blockIdx.x * 2 + (x.first == 0 ? 1 : 0)) * slot_floats<D>();
      float4* slot4 = reinterpret_cast<float4*>(slot) + own;  // + 128 for each four dims
      const int chains = (n + kChain - 1) / kChain;
      float m_slot = -INFINITY;
      int ev_slot = kMinExp;
      for (int c = 0; c < chains; ++c, ++chain) {
        const int o = chain & 1;
        const uint32_t parity = (uint32_t)(chain >> 1) & 1u;
        ok = wait(kMFull + o, parity) && wait(kOFull + o, parity);
        if (!ok) break;
        tc_fence_after();
        const bool last = c == chains - 1, out = last && x.whole != 0;
        float m, l = 0.f;
        int ev = 0;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(m) : "r"(smem + L::M + 4u * (o * kRows + own)));
        if (last) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(l) : "r"(smem + L::LT + 4u * (o * kRows + own)));
        if constexpr (I8) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(ev) : "r"(smem + L::EV + 4u * (o * kRows + own)));
        const float keep = m_slot == -INFINITY ? 1.f : exp2_approx(m_slot - m) * (I8 ? exp2_int(ev_slot - ev) : 1.f);
        const float f = !out ? 1.f : (l == 0.f ? 0.f : 1.0f / l) * (I8 ? exp2_int(ev) : 1.f);
        const bool mine = own < x.rows;  // the others' sums are nobody's
        if (__any_sync(0xffffffffu, mine)) {
          // The units have not changed: added where it lies, without waiting.  Else the slot's values are on their way
          // while those before them are worked on.
          const bool add = !out && c > 0 && __all_sync(0xffffffffu, keep == 1.f || !mine), fetch = c > 0 && !add && mine;
          float* dst = a.out;
          if (out && mine) {
            const int fr = x.r0 + own;
            dst += (int64_t)(x.row0 + fr / a.group) * a.ldo + (int64_t)(x.h * a.group + fr % a.group) * D;
          }
          const uint32_t from = tmem + lanes + L::O + (uint32_t)D * o;
          const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
          float4 next[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) next[i] = fetch ? __ldcg(slot4 + i * kRows) : zero;
#pragma unroll 1
          for (int d = 0; d < D; d += 16) {
            float v[16];
            tmem_ld_32x16(from + d, v);
            float4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[i] = make_float4(fmaf(next[i].x, keep, v[4 * i]), fmaf(next[i].y, keep, v[4 * i + 1]),
                                 fmaf(next[i].z, keep, v[4 * i + 2]), fmaf(next[i].w, keep, v[4 * i + 3]));
              next[i] = fetch && d + 16 < D ? __ldcg(slot4 + ((d + 16) / 4 + i) * kRows) : zero;
            }
            if (!mine) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float4* at = slot4 + (d / 4 + i) * kRows;
              if (add)
                asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1,%2,%3,%4};" ::"l"(at), "f"(w[i].x), "f"(w[i].y),
                             "f"(w[i].z), "f"(w[i].w)
                             : "memory");
              else if (!out)
                *at = w[i];
              else
                w[i] = make_float4(w[i].x * f, w[i].y * f, w[i].z * f, w[i].w * f);
            }
            if (out && wide) {  // whole 32-byte sectors
              st_global32(dst + d, w[0], w[1]);
              st_global32(dst + d + 8, w[2], w[3]);
            } else if (out) {
#pragma unroll
              for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(dst + d + 4 * i) = w[i];
            }
          }
        }
        tc_fence_before();
        arrive(kOFree + o);
        if (last && !out) {
          slot[kRows * D + own] = m;
          slot[kRows * D + kRows + own] = l;
          if constexpr (I8) slot[kRows * D + 2 * kRows + own] = (float)ev;
        }
        m_slot = m;
        ev_slot = ev;
      }
      if (ok && x.whole == 0 && x.first == 0 && own == 0)
        *divided = {x.last_block, x.h, x.row0, x.r0, x.rows};
      piece_done(k);
    }
    if (!ok && (threadIdx.x & 31) == 0) give_up();
  }

  // ---------------------------------------------------------------- softmax
  // A warp has 16 rows, a thread (g, t) = (lane / 4, lane % 4) of rows g and g + 8 the columns 8 b + 2 t + {0, 1}.

  // q's rows as hi + lo into shared memory; the scales of the thread's two rows.
  __device__ void split_q(const Piece& x, int row0, float (&row_scale)[2]) const {
    const int lane = threadIdx.x & 31;
    constexpr int LANES = D / 4, PER = 32 / LANES, BATCH = 16 / PER;  // lanes of a row, rows at a time
    const int sub = lane / LANES, at = lane % LANES;
    const float sign = a.scale_log2 < 0.f ? -1.f : 1.f;  // the scale's sign goes into q
    float mine = 0.f;                                    // scale of row `lane` of the 16
    const uint32_t hi = smem + L::Q + (uint32_t)(at >> 4) * L::PANEL;
    int64_t own = -1;  // where row `lane` begins
    if (lane < 16 && row0 + lane < x.rows) {
      const int fr = x.r0 + row0 + lane, token = fr / a.group;
      own = (int64_t)(x.row0 + token) * a.ldq + (int64_t)(x.h * a.group + fr % a.group) * D;
    }
    float4 v[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int64_t from = __shfl_sync(0xffffffffu, own, i * PER + sub);
      v[i] = from >= 0 ? __ldg(reinterpret_cast<const float4*>(a.q + from) + at) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      float top = fmaxf(fmaxf(fabsf(v[i].x), fabsf(v[i].y)), fmaxf(fabsf(v[i].z), fabsf(v[i].w)));
      if constexpr (LANES == 32) {  // (of positive numbers the larger has the larger bits)
        top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(top, 0.f))));
      } else {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      }
      const int e = fp16_row_exponent(top);
      const float up = sign * pow2f(e);
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int ep = __shfl_sync(0xffffffffu, e, p * LANES);
        if (lane == i * PER + p) mine = fabsf(a.scale_log2) * pow2f(-ep);
      }
      uint32_t h0, l0, h1, l1;
      split_f16(v[i].x * up, v[i].y * up, h0, l0);
      split_f16(v[i].z * up, v[i].w * up, h1, l1);
      const int r = row0 + i * PER + sub;  // of the tile
      const uint32_t addr = hi + (uint32_t)r * 128 + (((uint32_t)(at & 15) / 2 ^ (r & 7)) << 4) + 8u * (at & 1);
      asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(addr), "r"(h0), "r"(h1) : "memory");
      asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(addr + L::TILE), "r"(l0), "r"(l1) : "memory");
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
    // Trees: the rows' masks (of rows past the last none: they see all), the first of their bits' keys as the tile counts
    // them, words; lo and hi limit them.
    const uint32_t* seen[2];
    bool there[2];
    int pos0;
    int64_t words;
    // Which of the tile's 32 keys from j on row r sees.
    __device__ uint32_t sees(int r, int j) const {
      return there[r] ? tree_keys(seen[r], words, pos0, lo[r], hi[r], j) : ~0u;
    }
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
  // The scores of keys 32 c .. 32 c + 31: times the keys' scales, the hidden ones -inf, the bad ones NaN.
  template <bool EDGE>
  static __device__ __forceinline__ void prepare(const Scores& x, int c, uint32_t (&s)[16]) {
    const int t = threadIdx.x & 3;
    if constexpr (I8) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const uint2 w = ld_shared8(x.ks + 128u * c + 32u * b + 8u * t);
        mul2(s[4 * b], s[4 * b + 1], w.x, w.y);
        mul2(s[4 * b + 2], s[4 * b + 3], w.x, w.y);
      }
    }
    if constexpr (EDGE) {
      if constexpr (!I8) {
        uint32_t bad;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(bad) : "r"(x.bad + 4u * c));
        if (bad) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (bad >> (8 * (i >> 2) + 2 * t + (i & 1)) & 1u) s[i] = 0x7fc00000u;
        }
      }
      if constexpr (TREE) {
        const uint32_t sees[2] = {x.sees(0, 32 * c) >> (2 * t), x.sees(1, 32 * c) >> (2 * t)};
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!(sees[i >> 1 & 1] >> (8 * (i >> 2) + (i & 1)) & 1u)) s[i] = 0xff800000u;
        return;
      }
      // of the thread's keys, 8 b + {0, 1} from 32 c + 2 t on, a row sees [lo, hi)
      const int lo[2] = {x.lo[0] - 32 * c - 2 * t, x.lo[1] - 32 * c - 2 * t};
      const int hi[2] = {x.hi[0] - 32 * c - 2 * t, x.hi[1] - 32 * c - 2 * t};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int j = 8 * (i >> 2) + (i & 1), r = i >> 1 & 1;
        if (j < lo[r] || j >= hi[r]) s[i] = 0xff800000u;
      }
    }
  }
  // Warp 1, before its last arrival for a K tile: the tile's boxes whose pages are outside the pool, for the softmax.  That
  // reads them only where plain_hi sends it (at every tile they took 1 to 2.5% of its time).
  __device__ void mark_gone(Piece* place, uint32_t at, int64_t slot, int j0) const {
    const uint32_t gone = __ballot_sync(0xffffffffu, slot == kGone);
    if ((threadIdx.x & 31) == 0) {
      st_shared4(at, gone);
      if (gone) place->plain_hi = min(place->plain_hi, j0);
    }
  }
  // The scores of those boxes become -inf where they lie.
  __device__ void hide(uint32_t ts, uint32_t gone) const {
    const int shift = min(a.cache.page_shift, 7);
#pragma unroll 1
    for (int j = 0; j < kKeys; j += 16)
      if (gone >> (j >> shift) & 1u) tmem_fill_16x16(ts + (uint32_t)j, 0xff800000u);
    tmem_st_wait();
  }
  // Over the chunks of 32 scores, the load of one beside the work on the one before it.  The loops are kept short: the
  // roles' code together does not fit the instruction caches when this is unrolled over the whole tile.
  template <class Take>
  static __device__ __forceinline__ void over_chunks(uint32_t ts, Take take) {
    uint32_t s[2][16];
    tmem_ld_16x32(ts, s[0]);
#pragma unroll 1
    for (int c = 0; c < 4; c += 2) {
      tmem_ld_wait(s[0]);
      tmem_ld_16x32(ts + 32u * (c + 1), s[1]);
      take(c, s[0]);
      tmem_ld_wait(s[1]);
      if (c == 0) tmem_ld_16x32(ts + 64u, s[0]);
      take(c + 1, s[1]);
    }
  }
  // Scores to probabilities, in place in tensor memory.  Where a row's scores pass its maximum by more than kLazy it is
  // raised, and what was made with the old one is rescaled.  p = 2^(row_scale s + base), held in binary16 as hi + lo (times
  // the values' scales); of a chunk of 32 columns the high halves take the first 16, the low ones the others.  The high
  // half is p cut to 11 bits.
  template <bool EDGE, class Rescale>
  static __device__ __forceinline__ bool make_p(const Scores& x, float (&m)[2], float (&l)[2], const float (&down)[2],
                                                Rescale rescale_o) {
    const int t = threadIdx.x & 3;
    float top[2] = {-INFINITY, -INFINITY};
    over_chunks(x.ts, [&](int c, uint32_t (&s)[16]) {
      prepare<EDGE>(x, c, s);
#pragma unroll
      for (int i = 0; i < 16; i += 2)
        top[i >> 1 & 1] = max3(top[i >> 1 & 1], __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
    });
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
    over_chunks(x.ts, [&](int c, uint32_t (&s)[16]) {
      prepare<EDGE>(x, c, s);
      uint32_t hi[8], lo[8];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        uint2 w = make_uint2(0u, 0u);
        if constexpr (I8) w = ld_shared8(x.vs + 128u * c + 32u * b + 8u * t);
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
              float p0, p1;
              up2(p, p0, p1);
              p = p2(s0 == -INFINITY ? 0.f : p0, s1 == -INFINITY ? 0.f : p1);
            }
          }
          float p0, p1, r0, r1;
          up2(p, p0, p1);
          const float h0 = __uint_as_float(__float_as_uint(p0) & 0xffffe000u);
          const float h1 = __uint_as_float(__float_as_uint(p1) & 0xffffe000u);
          up2(fma2(p2(h0, h1), minus1, p), r0, r1);
          hi[2 * b + r] = pack_f16(h0, h1);
          lo[2 * b + r] = pack_f16(r0, r1);
        }
      }
      tmem_st_16x16(x.ts + 32u * c, hi);
      tmem_st_16x16(x.ts + 32u * c + 16u, lo);
    });
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float p0, p1;
      up2(sum[r], p0, p1);
      l[r] += p0 + p1;
    }
    tmem_st_wait();
    return true;
  }

  __device__ void softmax() const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int row0 = 32 * (warp & 3) + 16 * (warp >> 2 & 1);  // the warp's rows (its tensor memory lanes)
    const uint32_t lanes = (uint32_t)row0 << 16;
    bool ok = true;
    int step = 0, tile0 = 0, chain = 0;  // tiles of K, of K and V before the piece, chains of O so far
    for (int k = 0; ok; ++k) {
      const Piece* place = piece(k, ok);
      if (!ok) break;
      const Piece& x = *place;
      const int n = x.tiles;
      if (n == 0) break;
      Scores sc;
      split_q(x, row0, sc.row_scale);
      fence_proxy_async_smem();
      arrive(kQ);
      const int own0 = row0 + g;  // the thread's rows of the tile: own0, own0 + 8
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      int ev[2] = {kMinExp, kMinExp};
      for (int j = 0; j < n; ++j, ++step) {
        const int j0 = x.j0 + j * kKeys, s4 = step % kSteps;
        const bool fresh = j % kChain == 0;
        ok = wait(kSFull + (step & 1), (uint32_t)(step >> 1) & 1u);
        if (ok && I8) ok = wait(kScale + s4, (uint32_t)(step / kSteps) & 1u);
        const bool edge = j0 < x.all_lo || j0 + kKeys > x.plain_hi;
        if (ok && (I8 || edge)) {  // V's scales, or marks
          const int tv = tile0 + (j < n - 1 ? 2 * j + 2 : 2 * j + 1);
          ok = wait(kFull + tv % STAGES, (uint32_t)(tv / STAGES) & 1u);
        }
        if (!ok) break;
        tc_fence_after();
        sc.ts = tmem + lanes + L::S + 128u * (step & 1);
        sc.ks = smem + L::KS + (uint32_t)s4 * (kKeys * 4);
        sc.vs = smem + L::VS + (uint32_t)s4 * (kKeys * 4);
        if (edge) {
          sc.bad = smem + (edge_of(x, j0) ? L::BAD + 16u * s4 : L::ZERO);
          uint32_t gone;
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(gone) : "r"(smem + L::GONE + 4u * s4));
          if (gone) hide(sc.ts, gone);
#pragma unroll
          for (int r = 0; r < 2; ++r) {  // (rows past the last see all: nothing reads them)
            int lo = j0, hi = j0 + kKeys;
            const int token = (x.r0 + own0 + 8 * r) / a.group;
            if constexpr (TREE) {
              sc.there[r] = own0 + 8 * r < x.rows;
              if (sc.there[r]) {
                sc.seen[r] = a.seen + (x.row0 + token) * a.words;
                lo = tree_lo(sc.seen[r], a.words, a.window, x.pos0, x.len);
                hi = x.len;
              }
            } else if (own0 + 8 * r < x.rows) {
              row_keys({0, 0, x.len, x.pos0}, a.window, token, lo, hi);
            }
            sc.lo[r] = lo - j0;
            sc.hi[r] = hi - j0;
          }
          if constexpr (TREE) {
            sc.pos0 = x.pos0 - j0;
            sc.words = a.words;
          }
        }
        auto rescale_o = [&](float f0, float f1) {
          if (fresh || !__any_sync(0xffffffffu, f0 != 1.f || f1 != 1.f)) return true;  // (or O starts anew)
          if (!wait(kPv, (uint32_t)(step - 1) & 1u)) return false;
          tc_fence_after();
          const uint32_t to = tmem + lanes + L::O + (uint32_t)D * (chain & 1);
#pragma unroll 1
          for (int c = 0; c < D / 64; ++c) {
            uint32_t v[32];
            tmem_ld_16x64(to + 64u * c, v);
            tmem_ld_wait(v);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * (i & 2 ? f1 : f0));
            tmem_st_16x64(to + 64u * c, v);
          }
          tmem_st_wait();  // (a second rescaling in the same tile reads what this one wrote)
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
                if constexpr (TREE) {
                  const uint32_t sees = sc.sees(r, i & ~31) >> (i & 31);
                  if (sees & 1u) big[r] = fmaxf(big[r], __uint_as_float(w.x));
                  if (sees & 2u) big[r] = fmaxf(big[r], __uint_as_float(w.y));
                } else {
                  if (i >= sc.lo[r] && i < sc.hi[r]) big[r] = fmaxf(big[r], __uint_as_float(w.x));
                  if (i + 1 >= sc.lo[r] && i + 1 < sc.hi[r]) big[r] = fmaxf(big[r], __uint_as_float(w.y));
                }
              }
            }
            big[0] = quad_max(big[0]);
            big[1] = quad_max(big[1]);
          } else {
            const uint4 w = ld_shared16(smem + L::VMAX + 32u * s4);
            big[0] = big[1] = fmaxf(max3(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z)),
                                    __uint_as_float(w.w));
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
        arrive(kPFull + (step & 1));
        const bool last = j == n - 1;
        if (j % kChain == kChain - 1 || last) {  // the chain's units for the sums, in the place of the one before last
          const int o = chain & 1;
          if (last) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
              l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
            }
          }
          if (chain >= 2) ok = wait(kOFree + o, (uint32_t)(chain / 2 - 1) & 1u);
          if (!ok) break;
          if (t == 0) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const uint32_t at = 4u * (o * kRows + own0 + 8 * r);
              asm volatile("st.shared.f32 [%0], %1;" ::"r"(smem + L::M + at), "f"(m[r]) : "memory");
              if (last) asm volatile("st.shared.f32 [%0], %1;" ::"r"(smem + L::LT + at), "f"(l[r]) : "memory");
              if constexpr (I8) asm volatile("st.shared.b32 [%0], %1;" ::"r"(smem + L::EV + at), "r"(ev[r]) : "memory");
            }
          }
          arrive(kMFull + o);
          ++chain;
        }
      }
      tile0 += 2 * n;
      piece_done(k);
    }
    if (!ok && lane == 0) give_up();
  }
};

template <int D, bool I8, bool TREE>
__global__ void __launch_bounds__(kThreads, 1)
attention_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v, Divided* divided) {
  using L = Layout<D, I8>;
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
    auto init = [&](int i, int count) { mbar_init(smem + L::BARS + 8u * i, count); };
    for (int s = 0; s < L::STAGES; ++s) {
      init(kFull + s, kHelpers);
      init(kEmpty + s, 1);
    }
    for (int s = 0; s < kSteps; ++s) init(kScale + s, kHelpers);
    init(kQ, kSoftmax);
    init(kPv, 1);
    for (int i = 0; i < 2; ++i) {
      init(kSFull + i, 2);  // the products, and the issuer for what it has seen of K's tile
      init(kPFull + i, kSoftmax);
      init(kOFull + i, 1);
      init(kOFree + i, 4);
      init(kMFull + i, kSoftmax);
      init(kPieceFull + i, 1);
      init(kPieceFree + i, kThreads / 32);
    }
    init(kDrain, 1);
    init(kEdge, 1);
    for (int s = 0; s < L::RAW_STAGES; ++s) {
      init(kRawFull + s, 1);
      init(kRawEmpty + s, kHelpers);
    }
    *abort = 0;
    *reinterpret_cast<uint4*>(base + L::ZERO) = make_uint4(0u, 0u, 0u, 0u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async_smem();
  }
  if (warp == 0) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
  typename Kernel<D, I8, TREE>::Run run(a, reinterpret_cast<int64_t*>(base));  // the prefix sums lie where the tiles will
  fence_proxy_async_smem();                      // and are read and written before the copies overwrite them
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // the join may be launched: it waits for this kernel's end
  const Kernel<D, I8, TREE> k{a, map_k, map_v, smem, __shfl_sync(0xffffffffu, *tmem_slot, 0), abort,
                        reinterpret_cast<Piece*>(base + L::PIECES)};
  // 96 registers a thread at the start; 3 x 72 + 2 x 128 <= 5 x 96
  if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0) k.issuer();
    else if (warp == 1) k.loader(run);
    else if (warp < 8) k.helper();
    else k.sums(divided + blockIdx.x);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 128;");
    k.softmax();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(k.tmem, kTmemCols);
  }
}

// The pieces of the divided tiles, joined in the order of their blocks: blockIdx.x the block in whose run the tile
// begins, blockIdx.y a part of its (row, dims).  A warp takes 4 rows of 32 dims at a time.
constexpr int kJoinParts = 8, kJoinThreads = 256;
template <int D, bool I8>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const AttnArgs a, const Divided* divided) {
  pdl_wait();  // launched while the pieces are made
  const Divided x = divided[blockIdx.x];
  const int c0 = blockIdx.x, c1 = x.last_block;
  if (c1 <= c0) return;
  const int lane = threadIdx.x & 31;
  const int warps = kJoinParts * (kJoinThreads / 32), first = blockIdx.y * (kJoinThreads / 32) + (threadIdx.x >> 5);
  for (int task = first; task < (x.rows + 3) / 4 * (D / 32); task += warps) {  // 4 rows of 32 dims a warp
    const int row = task / (D / 32) * 4 + (lane & 3), d4 = task % (D / 32) * 8 + (lane >> 2);
    if (row >= x.rows) continue;
    auto slot = [&](int c) { return a.slots + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * slot_floats<D>(); };
    float m = -INFINITY, ev = kMinExp;
    for (int c = c0; c <= c1; ++c) {
      m = fmaxf(m, __ldcg(slot(c) + kRows * D + row));
      if constexpr (I8) ev = fmaxf(ev, __ldcg(slot(c) + kRows * D + 2 * kRows + row));
    }
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll 4
    for (int c = c0; c <= c1; ++c) {
      const float* s = slot(c);
      const float mc = __ldcg(s + kRows * D + row), lc = __ldcg(s + kRows * D + kRows + row);
      const float4 p = __ldcg(reinterpret_cast<const float4*>(s) + d4 * kRows + row);
      float w = mc == -INFINITY ? 1.f : exp2_approx(mc - m);  // without keys: zeros, or NaN
      l = fmaf(lc, w, l);
      if constexpr (I8) w *= exp2_int((int)(__ldcg(s + kRows * D + 2 * kRows + row) - ev));
      v = make_float4(fmaf(p.x, w, v.x), fmaf(p.y, w, v.y), fmaf(p.z, w, v.z), fmaf(p.w, w, v.w));
    }
    const float f = (l == 0.f ? 0.f : 1.0f / l) * (I8 ? exp2_int((int)ev) : 1.f);
    const int fr = x.r0 + row;
    *reinterpret_cast<float4*>(a.out + (int64_t)(x.row0 + fr / a.group) * a.ldo +
                               (int64_t)(x.head * a.group + fr % a.group) * D + 4 * d4) =
        make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
  }
}

template <int D, bool I8, bool TREE>
spl_status launch(const AttnArgs& a, int blocks, cudaStream_t stream) {
  constexpr uint32_t smem = Layout<D, I8>::SMEM;
  static bool done[kMaxDevices] = {false};
  if (!allow_shared(reinterpret_cast<const void*>(attention_tc_kernel<D, I8, TREE>), smem, done)) return SPL_ECUDA;
  Divided* divided = reinterpret_cast<Divided*>(a.slots + (int64_t)blocks * 2 * slot_floats<D>());
  CUtensorMap map_k = {}, map_v = {};
  if (!I8) {
    const int64_t slots = (int64_t)a.cache.pages * a.cache.heads << a.cache.page_shift;
    const int box = std::min(kKeys, 1 << a.cache.page_shift);
    if (!tma_panel_map(&map_k, a.cache.k, slots, D, box) || !tma_panel_map(&map_v, a.cache.v, slots, D, box))
      return SPL_ECUDA;
  }
  attention_tc_kernel<D, I8, TREE><<<blocks, kThreads, smem, stream>>>(a, map_k, map_v, divided);
  const spl_status st = launch_status();
  if (st != SPL_OK) return st;
  return launch_pdl(attention_join_kernel<D, I8>, dim3(blocks, kJoinParts), dim3(kJoinThreads), 0, stream, a,
                    static_cast<const Divided*>(divided));
}

}  // namespace

size_t attention_tc_bytes(int head_dim, int blocks) {
  const int64_t floats = head_dim == 128 ? slot_floats<128>() : slot_floats<64>();
  return (size_t)blocks * (2 * floats * sizeof(float) + sizeof(Divided));
}

template <bool TREE>
static spl_status pick(const AttnArgs& a, int head_dim, bool i8, int blocks, cudaStream_t stream) {
  if (head_dim == 128) return i8 ? launch<128, true, TREE>(a, blocks, stream) : launch<128, false, TREE>(a, blocks, stream);
  return i8 ? launch<64, true, TREE>(a, blocks, stream) : launch<64, false, TREE>(a, blocks, stream);
}
spl_status run_attention_tc(const AttnArgs& a, int head_dim, bool i8, bool tree, int blocks, cudaStream_t stream) {
  return tree ? pick<true>(a, head_dim, i8, blocks, stream) : pick<false>(a, head_dim, i8, blocks, stream);
}

}  // namespace spl
