// The attention weight that stored tokens gather from many rows (chunks, prompts), on the 5th-generation tensor cores.
//
//   score_j <- decay score_j + sum_i 2^(s_ij - lse_i),   s_ij = scale log2(e) q_i . k_j,   lse_i = log2 sum_j 2^s_ij
// The sum over rows needs every row's lse first, so the scores are made twice, over tiles of 128 rows (a token's `group`
// query heads side by side) and 128 keys:
//   S = q_hi K^T + q_lo K^T    q = (hi + lo) 2^-e in binary16, split ahead; the stored values are exact in binary16
// A first pass keeps the rows' maxima and totals of each range of key tiles, a small kernel joins those, and a second pass
// adds up p for each key.  Both walk the same way, a tile of rows after another and its key tiles in turn, and differ in
// which operand is the MMA's A: S has the rows in tensor memory's lanes in the first pass, so that a thread has a row, and
// K q^T the keys in the second, so that a thread has a key and its sum: neither reduces across threads, and nothing is
// added by atomics, whose order would change the bits.  Roles:
//   warp 0       MMA issuer.
//   warp 1       hands out the block's pieces of work and loads tiles of q and (binary16) of K, by TMA, a box a page.
//   warp 2       second pass: the rows' scales and lse.
//   warp 3       first pass, binary16: looks for keys that are not finite.
//   warps 4-11   two groups: maxima and totals (the key tiles in turn), or sums (half of a tile's rows each).
//   warps 12-19  int8: two groups widen the key tiles to binary16 in turn.
// Tensor memory: four places of S.
// Measured with 32 query heads on 8, 2048 rows over 12049 keys, binary16: passes of 222 to 229 and 232 to 237 us, 19 us before
// them and 7 between; int8 303 and 303.  What sets the pace is the issuing warp: a tile's 16 products are 1024 clocks of the tensor pipe (0.71
// and 0.68 of the time), but of its 1320 it spends 680 in handing them over, 200 in a commit and an arrival, 150 in asking for the
// operands and the place, the rest between tiles, and the pipe runs dry.  So it asks at once and commits once: a key tile's stage is
// free when its scores are there.  The epilogues come next: without the products, 207 and 222 us.  They pay for what they execute
// and read, so tiles of which all is seen have code of their own, and in the second pass, where a column's scale and lse go to
// every thread (4 wavefronts for 16 bytes), q's exponents are in steps, for a tile mostly to have one scale (15 sequences of 32
// rows int8, second pass 54 -> 43 us).  These in all, over 600 to 6000 keys: 92 us, of which 10 to 13 a pass are a launch, the
// dependent loads of the first piece and the first tile.
// A piece of the second pass has all rows of its keys, unless heads and key tiles are too few for all SMs: then it has one of
// several parts of them, and the last to end adds the parts' sums up: 2048 rows of 14 heads on 2 of 64 dims over 12049 keys
// 354 -> 251 us (now 210); 2048 rows of 32 heads on 8 over themselves 142 -> 126 (now 118).
// Every wait is bounded; on expiry the status word is raised and the block leaves with its
// copies and MMAs done.

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include <cuda_fp16.h>

#include "noise.cuh"  // packed fp32 pairs
#include "ptx.cuh"
#include "weigh.cuh"

namespace spl {
namespace {

constexpr int kTile = 128;          // rows and keys
constexpr int kEpilogue = 8;        // warps
constexpr int kThreads = 32 * (4 + kEpilogue), kThreadsI8 = kThreads + 32 * 8;
constexpr int kQStages = 2, kS = 4;
constexpr int kMostTiles = 8;       // key tiles of a piece of the second pass (a thread has a sum of each)
constexpr int kMostRange = 16;      // key tiles of a piece of the first pass
constexpr int kPieces = 4;
constexpr int kMostChunks = 16;     // parts of the rows that a piece of the second pass may have
constexpr int kSumTiles = 2048;     // key tiles of all pieces together when it has a part

// What the blocks go by, made on the device: key tiles of a piece of each pass, pieces of each, and behind it the first
// pieces of the sequences, [seqs] for each pass.
struct WeighPlan {
  int range, tiles, chunks;  // and parts of the rows, of which a piece of the second has one
  int64_t pieces[2];
  unsigned long long taken[2];  // beyond every block's first
};

struct TcArgs {
  WeighCall w;
  uint16_t *q_hi, *q_lo;  // [heads][total][dim], total = rows group
  float2* rows;           // [heads][total]: scale, NaN of a row that is not finite; lse, before it NaN if a key that it sees is not
  float2* parts;          // [heads][total][splits][2]: maximum, total
  int splits;             // places of a row
  // rows in parts: a piece's sums, [item][group][its key tile][key], and behind each range's first how many are there, [warp]
  float* sums;
  unsigned* arrived;
  int64_t total;
  WeighPlan* plan;
  int64_t* first[2];
};

struct alignas(16) Piece {
  int b, h;
  int row0, n, len, pos0;
  int rt0, rt1;  // row tiles [rt0, rt1), of the first pass one
  int t0, t1;    // key tiles
  int split;     // the range's index among the sequence's
                 // second pass: the piece's number where rows are in parts, else -1
  int last;      // no piece: the end
};

// ---------------------------------------------------------------- before the passes
// Block 0: the plan.  The others: q's rows as hi + lo, a warp a row or two.
constexpr int kPrepThreads = 256;
template <int D>
__global__ void __launch_bounds__(kPrepThreads) weigh_prepare_kernel(const __grid_constant__ TcArgs a, int grid) {
  const WeighCall& w = a.w;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, seqs = w.batch.seqs;
  if (blockIdx.x == 0) {
    __shared__ unsigned long long sums[kMostRange + kMostTiles], scan[2][kPrepThreads];  // pieces of a head, by their length
    __shared__ int key_tiles[kMaxSeqs], row_tiles[kMaxSeqs], longest, tallest, chosen[2], chunks;
    if (threadIdx.x == 0) longest = tallest = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < seqs; b += kPrepThreads) {
      const PagedSeq s = paged_seq(w.batch, w.cache.page_shift, b);
      key_tiles[b] = (s.len + kTile - 1) / kTile;
      row_tiles[b] = (s.n * w.group + kTile - 1) / kTile;
      atomicMax(&longest, key_tiles[b]);
      atomicMax(&tallest, row_tiles[b]);
    }
    __syncthreads();
    for (int i = warp; i < kMostRange + kMostTiles; i += kPrepThreads / 32) {
      const bool first = i < kMostRange;
      const uint32_t n = (uint32_t)(first ? i : i - kMostRange) + 1u;
      unsigned long long sum = 0;
      for (int b = lane; b < seqs; b += 32)
        sum += (unsigned long long)(((uint32_t)key_tiles[b] + n - 1u) / n) * (first ? (uint32_t)row_tiles[b] : 1u);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) sums[i] = sum;
    }
    __syncthreads();
    // The lengths that give the fewest key tiles to any block; beginning a piece or, in the second pass, a row tile costs some too.
    if (warp == 0) {
      unsigned long long cost = ~0ull;
      const int n = lane + 1;
      if (n <= kMostRange && (longest + n - 1) / n <= a.splits) {
        const unsigned long long pieces = sums[lane] * w.cache.heads;
        cost = (pieces + grid - 1) / grid * (n + 2) * 32 + (31 - lane);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) cost = min(cost, __shfl_xor_sync(0xffffffffu, cost, o));
      if (lane == 0) chosen[0] = 32 - (int)(cost & 31);  // (of equal ones the longest)
    } else if (warp == 1) {
      // And where that leaves blocks without work, the rows in parts.
      static_assert(kMostTiles == 8, "three bits");
      unsigned long long cost = ~0ull;
      const int n = lane % kMostTiles + 1;
      const unsigned long long pieces = sums[kMostRange + n - 1] * w.cache.heads;
      for (int c = 1 + lane / kMostTiles; c <= kMostChunks && c <= max(1, tallest); c += 32 / kMostTiles) {
        if (c > 1 && pieces * c * n > kSumTiles) break;
        // (a part's sums leave and come back: some 4 tiles' time)
        const unsigned long long one = (unsigned long long)((tallest + c - 1) / c) * (n + 1) + (c > 1 ? 4 : 0);
        cost = min(cost, ((pieces * c + grid - 1) / grid * one) * 256 + (c - 1) * 8 + (kMostTiles - n));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) cost = min(cost, __shfl_xor_sync(0xffffffffu, cost, o));
      if (lane == 0) chosen[1] = kMostTiles - (int)(cost % 8), chunks = (int)(cost / 8 % 32) + 1;
    }
    __syncthreads();
    const int64_t items = (int64_t)sums[kMostRange + chosen[1] - 1] * w.cache.heads * chunks;
    if (threadIdx.x == 0) *a.plan = {chosen[0], chosen[1], chunks, {(int64_t)sums[chosen[0] - 1] * w.cache.heads, items}, {0, 0}};
    if (chunks > 1)
      for (int i = threadIdx.x; i < 4 * (int)items; i += kPrepThreads) a.arrived[i] = 0u;
    // Each sequence's first piece: sums before it, a run of sequences a thread.
    const int per = (seqs + kPrepThreads - 1) / kPrepThreads, b0 = min(seqs, per * (int)threadIdx.x), b1 = min(seqs, b0 + per);
    auto count = [&](int b, int pass) {
      const uint32_t n = (uint32_t)chosen[pass];
      return (unsigned long long)(((uint32_t)key_tiles[b] + n - 1u) / n) * (uint32_t)(pass == 0 ? row_tiles[b] : chunks) *
             (unsigned)w.cache.heads;
    };
    for (int pass = 0; pass < 2; ++pass) {
      unsigned long long own = 0;
      for (int b = b0; b < b1; ++b) own += count(b, pass);
      scan[pass][threadIdx.x] = own;
    }
    __syncthreads();
    if (warp < 2) {
      unsigned long long carry = 0;
#pragma unroll 1
      for (int i0 = 0; i0 < kPrepThreads && i0 < seqs; i0 += 32) {  // (a thread has a sequence or more)
        const unsigned long long own = scan[warp][i0 + lane];
        unsigned long long v = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned long long other = __shfl_up_sync(0xffffffffu, v, o);
          if (lane >= o) v += other;
        }
        scan[warp][i0 + lane] = carry + v - own;
        carry += __shfl_sync(0xffffffffu, v, 31);
      }
    }
    __syncthreads();
    for (int pass = 0; pass < 2; ++pass) {
      unsigned long long sum = scan[pass][threadIdx.x];
      for (int b = b0; b < b1; ++b) {
        a.first[pass][b] = (int64_t)sum;
        sum += count(b, pass);
      }
    }
    return;
  }
  constexpr int LANES = D / 4, PER = 32 / LANES;
  const int sub = lane / LANES, at = lane % LANES;
  const int64_t all = w.batch.rows * w.q_heads;
  for (int64_t i0 = ((int64_t)(blockIdx.x - 1) * (kPrepThreads / 32) + warp) * PER; i0 < all;
       i0 += (int64_t)(gridDim.x - 1) * (kPrepThreads / 32) * PER) {
    const int64_t i = i0 + sub;
    const bool there = i < all;
    const int64_t token = there ? i / w.q_heads : 0;
    const int head = there ? (int)(i % w.q_heads) : 0;
    float4 v = there ? __ldcs(reinterpret_cast<const float4*>(w.q + token * w.ldq + (int64_t)head * D) + at)
                     : make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = fabsf(v.x) + fabsf(v.y) + (fabsf(v.z) + fabsf(v.w));
    float top = fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w)));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    // A row that is not finite is zeros in the products, which then are finite wherever the key is, and NaN by its scale.
    const bool finite = top <= FLT_MAX && sum == sum;
    if (!finite) v = make_float4(0.f, 0.f, 0.f, 0.f), top = 0.f;
    // (in steps of 12, so that rows of like size have the same and the second pass one scale for a tile; the largest is then in
    // [2^3, 2^15), where the low half's smallest step, 2^-24, is still far below 2^-22 of it)
    const int e = top > 0.f ? (fp16_row_exponent(top) - 8 + 132) / 12 * 12 - 132 + 8 : 8;
    const float up = w.scale_log2 < 0.f ? -pow2f(e) : pow2f(e);  // the scale's sign goes into q
    uint32_t h0, l0, h1, l1;
    split_f16(v.x * up, v.y * up, h0, l0);
    split_f16(v.z * up, v.w * up, h1, l1);
    if (!there) continue;
    const int64_t row = (int64_t)(head / w.group) * a.total + token * w.group + head % w.group;
    reinterpret_cast<uint2*>(a.q_hi + row * D)[at] = make_uint2(h0, h1);
    reinterpret_cast<uint2*>(a.q_lo + row * D)[at] = make_uint2(l0, l1);
    if (at == 0) a.rows[row] = make_float2(finite ? fabsf(w.scale_log2) * pow2f(-e) : NAN, 0.f);
  }
}

// ---------------------------------------------------------------- the passes
template <int D, bool I8>
struct Layout {
  static constexpr int PANELS = D / 64, STAGES = D == 64 ? 4 : (I8 ? 2 : 3);
  // key tiles whose marks or scales have a place: the loader is at most STAGES ahead of the issuer, which is at most kS ahead of
  // the epilogue
  static constexpr int NOTES = D == 64 ? 16 : 8;
  static_assert(NOTES > STAGES + kS, "and one that is being written");
  // A tile's products are done, and its stage free, when its scores are there; their place's next phase is not before the stage is
  // used again.
  static_assert(STAGES <= kS, "one phase to wait for");
  static constexpr uint32_t PANEL = 128 * 128, TILE = PANELS * PANEL;
  static constexpr uint32_t Q = 0, K = kQStages * 2 * TILE;  // stages of [q_hi, q_lo]; of K
  // second pass: the rows' scales and lse of each stage of q; int8: the keys' scales; first pass: marks of keys without a page
  static constexpr uint32_t COL = K + STAGES * TILE, SCALE = COL + kQStages * kTile * 8;
  static constexpr uint32_t GONE = SCALE + (I8 ? NOTES * kTile * 4 : 0);
  static constexpr uint32_t ONE = GONE + NOTES * 16, BARS = ONE + 16;
  enum { kQFull = 0, kQEmpty = 2, kSFull = 4, kSFree = 8, kPieceFull = 12, kPieceFree = 16, kColFull = 20, kColEmpty = 22,
         kFirst = 24, kSecond = 25, kDrain = 26, kKFull = 27, kBars = (kKFull + STAGES + 1) / 2 * 2 };
  static constexpr uint32_t PIECES = BARS + 8 * kBars, MISC = PIECES + kPieces * sizeof(Piece);
  // int8, second pass: the slots and old scores of the threads' keys, [group][2][key tile][key]
  static constexpr uint32_t STASH = MISC + 16, SMEM = STASH + (I8 ? 2 * 2 * kMostTiles * kTile * 4 : 0);
  static_assert(PIECES % 16 == 0 && SMEM <= 232448, "227 KB of dynamic shared memory per block");
  static constexpr uint32_t IDESC = make_idesc(0, 128, 128);
};
constexpr uint32_t kTmemCols = 512;

__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                       uint32_t accumulate, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(hi), "r"(leader)
      : "memory");
}
// 32 lanes x 32 columns (thread t gets lane base + t); read after tmem_ld_wait.
__device__ __forceinline__ void tmem_ld_32x32_begin(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t ld_shared4(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ void st_shared4(uint32_t addr, uint32_t v) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
template <int D, bool I8, bool SUM>
struct Kernel {
  using L = Layout<D, I8>;
  const TcArgs& a;
  const CUtensorMap &map_hi, &map_lo, &map_k;
  uint32_t smem, tmem;
  volatile int* abort;
  Piece* pieces;

  __device__ uint32_t bar(int i) const { return smem + L::BARS + 8u * i; }
  __device__ bool wait(int i, uint32_t parity, unsigned long long ns = kWaitNs) const {
    return __all_sync(0xffffffffu, mbar_wait_soon(bar(i), parity, ns, abort));
  }
  // Whether the stage of key tile `key` may be written, whose last was the one STAGES before.
  __device__ bool stage_free(int key, unsigned long long ns = kWaitNs) const {
    const int last = key - L::STAGES;
    return last < 0 || wait(L::kSFull + last % kS, (uint32_t)(last / kS) & 1u, ns);
  }
  __device__ void arrive(int i) const {  // one for the warp, after all its lanes' work
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar(i));
  }
  __device__ void give_up() const {
    *abort = 1;
    atomicOr(a.w.batch.status, kStatusTimeout);
  }

  // ---------------------------------------------------------------- the walk
  // Of a row tile: its rows, the key tiles of the piece that it meets, and the keys that all its rows see.
  struct Span {
    int r0, rows, k0, k1, all_lo, all_hi;
  };
  __device__ Span span(const Piece& x, int rt) const {
    const int group = a.w.group;
    Span y;
    y.r0 = rt * kTile;
    y.rows = min(kTile, x.n * group - y.r0);
    const PagedSeq s = {x.row0, x.n, x.len, x.pos0};
    int lo, hi;
    row_keys(s, a.w.window, y.r0 / group, lo, y.all_hi);
    row_keys(s, a.w.window, (y.r0 + y.rows - 1) / group, y.all_lo, hi);
    y.k0 = max(x.t0, lo / kTile);
    y.k1 = hi > lo ? min(x.t1, (hi + kTile - 1) / kTile) : y.k0;
    return y;
  }
  // For every piece begin(piece), for each of its row tiles that meets key tiles tile(piece, span, its number), for each of
  // these step(piece, span, key tile, its number), end(piece); all return whether to go on.
  template <class Begin, class Rows, class Step, class RowsEnd, class End>
  __device__ bool walk(Begin begin, Rows rows, Step step, RowsEnd rows_end, End end) const {
    int tile = 0, key = 0;
    for (int k = 0;; ++k) {
      if (!wait(L::kPieceFull + k % kPieces, (uint32_t)(k / kPieces) & 1u)) return false;
      const Piece x = pieces[k % kPieces];
      arrive(L::kPieceFree + k % kPieces);
      if (x.last) return true;
      if (!begin(x)) return false;
      for (int rt = x.rt0; rt < x.rt1; ++rt) {
        const Span y = span(x, rt);
        if (y.k0 >= y.k1) continue;
        if (!rows(x, y, tile)) return false;
        for (int kt = y.k0; kt < y.k1; ++kt, ++key)
          if (!step(x, y, kt, key, tile)) return false;
        if (!rows_end(x, y, tile)) return false;
        ++tile;
      }
      if (!end(x)) return false;
    }
  }
  static constexpr auto nothing = [](auto&&...) { return true; };

  // The k-th piece of the block, by warp 1.
  __device__ bool hand_out(int k) const {
    const int lane = threadIdx.x & 31, seqs = a.w.batch.seqs, group = a.w.group;
    if (k >= kPieces && !wait(L::kPieceFree + k % kPieces, (uint32_t)(k / kPieces - 1) & 1u, kLoaderNs)) return false;
    // The next that nobody has: pieces differ in size, and which block has one does not matter to any result.
    unsigned long long taken = 0;
    if (k > 0 && lane == 0) taken = atomicAdd(&a.plan->taken[SUM], 1ull);
    const int64_t item = k == 0 ? (int64_t)blockIdx.x : (int64_t)gridDim.x + (int64_t)__shfl_sync(0xffffffffu, taken, 0);
    Piece x = {};
    x.last = 1;
    if (item < a.plan->pieces[SUM]) {
      const int64_t* first = a.first[SUM];
      int lo = 0, n = seqs;  // the last sequence that begins at or before it
      while (n > 1) {
        const int step = (n + 31) >> 5, i = lane * step;
        const unsigned below = __ballot_sync(0xffffffffu, i < n && first[lo + (i < n ? i : 0)] <= item);
        const int pick = below ? 31 - __clz(below) : 0;
        lo += pick * step;
        n = n - pick * step < step ? n - pick * step : step;
      }
      const PagedSeq s = paged_seq(a.w.batch, a.w.cache.page_shift, lo);
      const int per = SUM ? a.plan->tiles : a.plan->range;
      const int tiles = (s.len + kTile - 1) / kTile, rows = s.n * group, row_tiles = (rows + kTile - 1) / kTile;
      const int splits = (tiles + per - 1) / per;
      int64_t rest = item - first[lo];
      const int chunks = SUM ? a.plan->chunks : 1;
      const int64_t of_head = (int64_t)splits * (SUM ? chunks : row_tiles);
      x.b = lo;
      x.h = (int)quotient(rest, of_head);
      rest -= x.h * of_head;
      x.row0 = s.row0, x.n = s.n, x.len = s.len, x.pos0 = s.pos0;
      int split, chunk = 0;
      if constexpr (SUM) {
        split = (int)quotient(rest, chunks);
        chunk = (int)(rest - (int64_t)split * chunks);
        x.split = chunks > 1 ? (int)item : -1;
      } else {
        x.split = split = (int)(rest % splits);
      }
      x.t0 = split * per;
      x.t1 = min(tiles, x.t0 + per);
      if constexpr (SUM) {  // the tokens that may see a key of the range
        const int64_t i0 = max((int64_t)0, (int64_t)x.t0 * kTile - s.pos0);
        const int64_t i1 = a.w.window == INT32_MAX ? s.n : min((int64_t)s.n, (int64_t)x.t1 * kTile - s.pos0 + a.w.window);
        const int64_t rt0 = i0 < i1 ? i0 * group / kTile : 0, rt1 = i0 < i1 ? (i1 * group + kTile - 1) / kTile : 0;
        x.rt0 = chunks == 1 ? (int)rt0 : (int)(rt0 + (rt1 - rt0) * chunk / chunks);
        x.rt1 = chunks == 1 ? (int)rt1 : (int)(rt0 + (rt1 - rt0) * (chunk + 1) / chunks);
      } else {
        x.rt0 = (int)quotient(rest, splits);
        x.rt1 = x.rt0 + 1;
      }
      x.last = 0;
    }
    if (lane == 0) {
      pieces[k % kPieces] = x;
      mbar_arrive(bar(L::kPieceFull + k % kPieces));
    }
    __syncwarp();
    return true;
  }

  // ---------------------------------------------------------------- loads
  static constexpr int kUnseen = -1, kGone = -2;
  // The page of the keys from j on (all in one), kUnseen past the sequence's end, kGone if it is outside the pool.
  __device__ int page_of(const Piece& x, int j) const {
    if (j >= x.len) return kUnseen;
    const int page = paged_page(a.w.cache, a.w.batch, x.b, j);
    return page >= 0 ? page : kGone;
  }
  // Warp 1.  In the second pass it begins while the first one's last blocks and the join are at work, for which the others wait
  // without spinning: its own waits may last longer.
  static constexpr unsigned long long kLoaderNs = SUM ? 20 * kWaitNs : kWaitNs;
  __device__ void loader() const {
    const int lane = threadIdx.x & 31, shift = a.w.cache.page_shift;
    const int box = min(kTile, 1 << shift), boxes = kTile / box;
    const int none = (int)((int64_t)a.w.cache.pages * a.w.cache.heads << shift);  // past the pool: filled with zeros
    const uint64_t policy = l2_evict_last();  // other blocks read the same tiles
    int tiles = 0, keys = 0;  // loaded so far
    bool ok = true;
    for (int k = 0; ok; ++k) {
      ok = hand_out(k);
      if (!ok) break;
      const Piece x = pieces[k % kPieces];
      __syncwarp();
      arrive(L::kPieceFree + k % kPieces);
      if (x.last) break;
      for (int rt = x.rt0; ok && rt < x.rt1; ++rt) {
        const Span y = span(x, rt);
        if (y.k0 >= y.k1) continue;
        const int q = tiles % kQStages;
        if (tiles >= kQStages) ok = wait(L::kQEmpty + q, (uint32_t)(tiles / kQStages - 1) & 1u, kLoaderNs);
        if (!ok) break;
        if (lane == 0) {
          const uint32_t to = smem + L::Q + (uint32_t)q * 2u * L::TILE;
          const int row = (int)((int64_t)x.h * a.total + (int64_t)x.row0 * a.w.group + y.r0);
          mbar_expect_tx(bar(L::kQFull + q), 2u * L::TILE);
#pragma unroll
          for (int p = 0; p < L::PANELS; ++p) {
            tma_load_2d(to + p * L::PANEL, &map_hi, bar(L::kQFull + q), 64 * p, row, policy);
            tma_load_2d(to + L::TILE + p * L::PANEL, &map_lo, bar(L::kQFull + q), 64 * p, row, policy);
          }
        }
        __syncwarp();
        ++tiles;
        if constexpr (I8) continue;
        auto look_up = [&](int kt) {  // the lane's box of a key tile
          const int j = kt * kTile + lane * box;
          const int page = lane < boxes && kt < y.k1 ? page_of(x, j) : kUnseen;
          return page >= 0 ? ((((int64_t)page * a.w.cache.heads + x.h) << shift) + (j & ((1 << shift) - 1))) : (int64_t)page;
        };
        int64_t slot = look_up(y.k0);
        for (int kt = y.k0; ok && kt < y.k1; ++kt) {
          const int64_t next = look_up(kt + 1);
          const int stage = keys % L::STAGES;
          ok = stage_free(keys, kLoaderNs);
          if (!ok) break;
          const unsigned gone = __ballot_sync(0xffffffffu, slot == kGone);
          if (lane < 4) {  // a bit a key
            uint32_t word = 0;
            for (int i = 0; i < 32; i += 16)
              if (gone >> ((32 * lane + i) / box) & 1u) word |= 0xffffu << i;
            st_shared4(smem + L::GONE + 16u * (keys % L::NOTES) + 4u * lane, word);
          }
          __syncwarp();
          if (lane == 0) mbar_expect_tx(bar(L::kKFull + stage), L::TILE);
          __syncwarp();
          if (lane < boxes) {
            const uint32_t to = smem + L::K + (uint32_t)stage * L::TILE + (uint32_t)(lane * box) * 128u;
#pragma unroll
            for (int p = 0; p < L::PANELS; ++p)
              tma_load_2d(to + p * L::PANEL, &map_k, bar(L::kKFull + stage), 64 * p, slot >= 0 ? (int)slot : none, policy);
          }
          __syncwarp();
          slot = next;
          ++keys;
        }
      }
    }
    if (!ok) {
      if (lane == 0) give_up();
      // no copy in flight when the block leaves
      for (int t = max(0, tiles - kQStages); t < tiles; ++t)
        mbar_wait(bar(L::kQFull + t % kQStages), (uint32_t)(t / kQStages) & 1u, kDrainNs, nullptr);
      for (int t = max(0, keys - L::STAGES); t < keys; ++t)
        mbar_wait(bar(L::kKFull + t % L::STAGES), (uint32_t)(t / L::STAGES) & 1u, kDrainNs, nullptr);
    }
  }
  // Warp 2, second pass: scales and -lse of a tile's rows, of rows that are not there an lse that leaves nothing; and the scale,
  // if all have the same, else -1.
  __device__ void columns() const {
    const int lane = threadIdx.x & 31;
    const bool ok = walk(
        nothing,
        [&](const Piece& x, const Span& y, int tile) {
          const int q = tile % kQStages;
          if (tile >= kQStages && !wait(L::kColEmpty + q, (uint32_t)(tile / kQStages - 1) & 1u)) return false;
          const float2* rows = a.rows + (int64_t)x.h * a.total + (int64_t)x.row0 * a.w.group + y.r0;
          const float one = rows[0].x;
          float2 v[4];
          bool fast = true;
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // (rows behind the tile's own are in its products all the same, finite ones)
            const bool there = 4 * lane + i < y.rows;
            v[i] = there ? rows[4 * lane + i] : make_float2(0.f, INFINITY);
            fast = fast && (!there || v[i].x == one);
          }
          const uint32_t to = smem + L::COL + 1024u * q + 16u * lane;
          st_shared16(to, make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[1].x), __float_as_uint(v[2].x),
                                     __float_as_uint(v[3].x)));
          st_shared16(to + 512u, make_uint4(__float_as_uint(-v[0].y), __float_as_uint(-v[1].y), __float_as_uint(-v[2].y),
                                            __float_as_uint(-v[3].y)));
          fast = __all_sync(0xffffffffu, fast);
          if (lane == 0) st_shared4(smem + L::ONE + 4u * q, __float_as_uint(fast ? one : -1.f));
          arrive(L::kColFull + q);
          return true;
        },
        nothing, nothing, nothing);
    if (!ok && lane == 0) give_up();
  }
  // The slot of key j, or the reason that it has none.
  __device__ int slot_of(const Piece& x, int j) const {
    const int page = page_of(x, j);
    return page >= 0 ? (int)paged_slot(a.w.cache, page, x.h, j) : page;
  }
  // Warps 12-19 (int8): every other key tile widened to binary16 in the MMAs' layout, a thread the same 16 dims of every
  // KEY_STEP-th key; marks of keys without a page and, in the first pass, the keys' scales.
  __device__ void widen() const {
    constexpr int PARTS = D / 16, KEY_STEP = 128 / PARTS, PER = kTile / KEY_STEP, KEYS = 32 / PARTS;
    static_assert(PER * KEYS == 32, "a warp's keys");
    const int i = threadIdx.x & 127, set = (threadIdx.x >> 7) - kThreads / 128, lane = i & 31;
    const int part = i % PARTS, key0 = i / PARTS, c0 = (2 * part) & 7;
    const int8_t* codes = static_cast<const int8_t*>(a.w.cache.k);
    // A tile's codes, on their way while the one before is widened (but not across pieces: the next one may be handed out
    // only after what is held here has been worked on).
    uint4 q[PER];
    float scale = 0.f;
    unsigned gone = 0;
    int held = -1;  // which tile
    auto finish = [&]() {
      if (held < 0) return true;
      const int stage = held % L::STAGES;
      if (!stage_free(held)) return false;
      const uint32_t panel = smem + L::K + (uint32_t)stage * L::TILE + (uint32_t)(part >> 2) * L::PANEL;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int at = key0 + KEY_STEP * k;
        const uint32_t v[4] = {q[k].x ^ 0x80808080u, q[k].y ^ 0x80808080u, q[k].z ^ 0x80808080u, q[k].w ^ 0x80808080u};
        const uint32_t row = panel + at * 128;
        // (the upper panel's threads begin with their second chunk: the eight threads of a key then meet no bank twice)
        const bool swap = part >= 4;
        const uint32_t w0 = swap ? v[2] : v[0], w1 = swap ? v[3] : v[1], w2 = swap ? v[0] : v[2], w3 = swap ? v[1] : v[3];
        const int first = swap ? c0 + 1 : c0;
        st_shared16(row + ((first ^ (at & 7)) << 4), make_uint4(i8_pair(w0, 0x4140u), i8_pair(w0, 0x4342u),
                                                                i8_pair(w1, 0x4140u), i8_pair(w1, 0x4342u)));
        st_shared16(row + (((first ^ 1) ^ (at & 7)) << 4), make_uint4(i8_pair(w2, 0x4140u), i8_pair(w2, 0x4342u),
                                                                      i8_pair(w3, 0x4140u), i8_pair(w3, 0x4342u)));
      }
      // (an infinite scale is NaN: its scores might be -inf, which is no weight)
      st_shared4(smem + L::SCALE + 4u * (held % L::NOTES * kTile + i), __float_as_uint(scale + (scale - scale)));
      if (lane == 0) st_shared4(smem + L::GONE + 16u * (held % L::NOTES) + 4u * (i >> 5), gone);
      fence_proxy_async_smem();
      arrive(L::kKFull + stage);
      held = -1;
      return true;
    };
    const bool ok = walk(
        nothing, nothing,
        [&](const Piece& x, const Span&, int kt, int key, int) {
          if ((key & 1) != set) return true;
          // The warp's 32 keys, a lane each, and (for its scale and mark) the thread's own.
          const int key_of_lane = lane % KEYS + KEYS * (i >> 5) + KEY_STEP * (lane / KEYS);
          const int mine = slot_of(x, kt * kTile + key_of_lane), own = slot_of(x, kt * kTile + i);
          if (!finish()) return false;
#pragma unroll
          for (int k = 0; k < PER; ++k) {
            const int slot = __shfl_sync(0xffffffffu, mine, k * KEYS + key0 % KEYS);
            q[k] = slot >= 0 ? __ldg(reinterpret_cast<const uint4*>(codes + (int64_t)slot * D) + part) : make_uint4(0u, 0u, 0u, 0u);
          }
          scale = own >= 0 ? __ldg(a.w.cache.k_scale + own) : 0.f;
          gone = __ballot_sync(0xffffffffu, own == kGone);
          held = key;
          return true;
        },
        nothing, [&](const Piece&) { return finish(); });
    if (!ok && lane == 0) give_up();
  }

  // ---------------------------------------------------------------- MMA issuer
  __device__ void issuer() const {
    const uint32_t leader = elect_one();
    auto commit = [&](int i) {
      if (leader) mma_commit(bar(i));
      __syncwarp();
    };
    const bool ok = walk(
        nothing,
        [&](const Piece&, const Span&, int tile) { return wait(L::kQFull + tile % kQStages, (uint32_t)(tile / kQStages) & 1u); },
        [&](const Piece&, const Span&, int, int key, int tile) {
          const int stage = key % L::STAGES, place = key % kS;
          const uint32_t k_parity = (uint32_t)(key / L::STAGES) & 1u, s_parity = (uint32_t)(key / kS - 1) & 1u;
          // (both asked at once: mostly neither is waited for, and the answers are what takes time)
          const bool there = mbar_try(bar(L::kKFull + stage), k_parity);
          const bool free = key < kS || mbar_try(bar(L::kSFree + place), s_parity);
          if (!__all_sync(0xffffffffu, there && free)) {
            if (!wait(L::kKFull + stage, k_parity)) return false;
            if (key >= kS && !wait(L::kSFree + place, s_parity)) return false;
          }
          tc_fence_after();
          const uint32_t q = sdesc_lo(smem + L::Q + (uint32_t)__shfl_sync(0xffffffffu, tile % kQStages, 0) * 2u * L::TILE);
          const uint32_t kd = sdesc_lo(smem + L::K + (uint32_t)__shfl_sync(0xffffffffu, stage, 0) * L::TILE);
          const uint32_t d = tmem + 128u * (uint32_t)__shfl_sync(0xffffffffu, place, 0);
          // The low halves first: each product truncates its sum, which is still small for them.
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            const int s = i % (D / 16);
            const uint32_t off = ((uint32_t)(s / 4) * L::PANEL + (uint32_t)(s % 4) * 32u) >> 4;
            const uint32_t qi = q + off + (i < D / 16 ? L::TILE >> 4 : 0u), ki = kd + off;
            mma_ss(d, SUM ? ki : qi, SUM ? qi : ki, kSdescHi128, L::IDESC, i > 0 ? 1u : 0u, leader);
          }
          if (leader) {
            mbar_arrive(bar(L::kSFull + place));
            mma_commit(bar(L::kSFull + place));
          }
          __syncwarp();
          return true;
        },
        [&](const Piece&, const Span&, int tile) {
          commit(L::kQEmpty + tile % kQStages);
          return true;
        },
        nothing);
    if (!ok && leader) give_up();
    commit(L::kDrain);  // every MMA done before tensor and shared memory are given back
    mbar_wait(bar(L::kDrain), 0u, kDrainNs, nullptr);
  }

  // Warp 3, first pass, binary16: an infinity of a key may be one of the same sign in both halves' products, and a score of -inf
  // would be a weight of 0, not NaN.  But then all rows' scores of the key are infinities or NaN (others are at most 2^39), so one
  // warp's 32 rows are enough, and a sum of each.  Of tiles of which the rows see all; the others' are looked at one by one above
  // their masks.  (Done by the epilogue's warps, for all keys or a quarter each: 486 to 490 us instead of 478 for the 2048 rows.)
  __device__ void infinities() const {
    const int lane = threadIdx.x & 31;
    const bool ok = walk(
        nothing, nothing,
        [&](const Piece& x, const Span& y, int kt, int key, int) {
          const int place = key % kS, j0 = kt * kTile;
          if (!wait(L::kSFull + place, (uint32_t)(key / kS) & 1u)) return false;
          tc_fence_after();
          const uint4 gone = ld_shared16(smem + L::GONE + 16u * (key % L::NOTES));
          const bool edge = j0 < y.all_lo || j0 + kTile > y.all_hi || (gone.x | gone.y | gone.z | gone.w) != 0;
          unsigned long long sum[2] = {p2(0.f, 0.f), p2(0.f, 0.f)};
          if (!edge) {
            over_chunks(tmem + (96u << 16) + 128u * place, [&](int, uint32_t (&r)[32]) {
#pragma unroll
              for (int k = 0; k < 32; k += 2)
                sum[k / 2 & 1] = add2(sum[k / 2 & 1], p2(__uint_as_float(r[k]), __uint_as_float(r[k + 1])));
            });
          }
          tc_fence_before();
          arrive(L::kSFree + place);
          float s0, s1;
          up2(add2(sum[0], sum[1]), s0, s1);
          if (__any_sync(0xffffffffu, !(fabsf(s0 + s1) <= FLT_MAX))) {
            float2* rows = a.rows + (int64_t)x.h * a.total + (int64_t)x.row0 * a.w.group + y.r0;
            for (int i = lane; i < y.rows; i += 32) rows[i].y = NAN;
          }
          return true;
        },
        nothing, nothing);
    if (!ok && lane == 0) give_up();
  }

  // ---------------------------------------------------------------- epilogue
  static __device__ __forceinline__ void mul2(uint32_t& a, uint32_t& b, uint32_t x, uint32_t y) {
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tmul.rn.f32x2 p, p, q;\n\t"
        "mov.b64 {%0, %1}, p;\n\t}"
        : "+r"(a), "+r"(b)
        : "r"(x), "r"(y));
  }
  static __device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
  }
  // The 128 scores of a thread's lane, 32 at a time, the load of some beside the work on those before.
  template <class Take>
  __device__ void over_chunks(uint32_t ts, Take take) const {
    uint32_t v[2][32];
    tmem_ld_32x32_begin(ts, v[0]);
#pragma unroll 1
    for (int c = 0; c < 4; c += 2) {
      tmem_ld_wait(v[0]);
      tmem_ld_32x32_begin(ts + 32u * (c + 1), v[1]);
      take(c, v[0]);
      tmem_ld_wait(v[1]);
      if (c == 0) tmem_ld_32x32_begin(ts + 64u, v[0]);
      take(c + 1, v[1]);
    }
  }
  // The slots of the thread's key of each of the piece's key tiles, -1 where there is none.
  __device__ void slots_of(const Piece& x, int own, int (&slot)[kMostTiles]) const {
    const int* table = a.w.batch.table + x.b * a.w.batch.max_pages;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kMostTiles; ++i) {  // (the pages first, so that the loads run side by side)
      const int kt = x.t0 + i, j = kt * kTile + own;
      slot[i] = kt < x.t1 && j < x.len ? __ldg(table + (j >> a.w.cache.page_shift)) : -1;
      bad |= kt < x.t1 && j < x.len && (unsigned)slot[i] >= (unsigned)a.w.cache.pages;
    }
    if (bad) atomicOr(a.w.batch.status, kStatusIndex);
#pragma unroll
    for (int i = 0; i < kMostTiles; ++i)
      slot[i] = (unsigned)slot[i] < (unsigned)a.w.cache.pages ? (int)paged_slot(a.w.cache, slot[i], x.h, (x.t0 + i) * kTile + own)
                                                               : -1;
  }
  // A part of the rows: the sums to the workspace, and of the warps that have sums of the same keys the last to arrive adds all
  // up, in the parts' order whichever it is.
  __device__ void join_parts(const Piece& x, int own, int set, const float (&sum)[kMostTiles]) const {
    const int lane = threadIdx.x & 31, per = a.plan->tiles * kTile, chunks = a.plan->chunks, first = x.split / chunks * chunks;
    float* to = a.sums + ((int64_t)x.split * 2 + set) * per + own;
#pragma unroll
    for (int i = 0; i < kMostTiles; ++i)
      if (i < x.t1 - x.t0) __stcg(to + i * kTile, sum[i]);
    __threadfence();
    __syncwarp();
    unsigned there = 0;
    if (lane == 0) there = atomicAdd(a.arrived + 4 * first + own / 32, 1u);
    there = __shfl_sync(0xffffffffu, there, 0);
    if ((int)there != 2 * chunks - 1) return;
    __threadfence();
    const float* from = a.sums + (int64_t)first * 2 * per + own;
    float all[kMostTiles] = {}, before[kMostTiles];
    int slot[kMostTiles];
    slots_of(x, own, slot);
#pragma unroll
    for (int i = 0; i < kMostTiles; ++i)
      before[i] = slot[i] >= 0 && (x.t0 + i) * kTile + own < x.pos0 ? a.w.score[slot[i]] * a.w.decay : 0.f;
#pragma unroll 2
    for (int c = 0; c < 2 * chunks; ++c, from += per)
#pragma unroll
      for (int i = 0; i < kMostTiles; ++i)
        if (i < x.t1 - x.t0) all[i] += __ldcg(from + i * kTile);
#pragma unroll
    for (int i = 0; i < kMostTiles; ++i)
      if (slot[i] >= 0) a.w.score[slot[i]] = before[i] + all[i];
  }
  __device__ void epilogue() const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, set = (warp - 4) >> 2;
    const int own = 32 * (warp & 3) + lane;
    const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    bool ok;
    if constexpr (!SUM) {
      float m = -INFINITY, l = 0.f, scale = 0.f;
      int lo = 0, hi = 0;
      ok = walk(
          nothing,
          [&](const Piece& x, const Span& y, int) {
            m = -INFINITY, l = 0.f, scale = FLT_MIN, lo = hi = 0;
            if (own < y.rows) {
              scale = a.rows[(int64_t)x.h * a.total + (int64_t)x.row0 * a.w.group + y.r0 + own].x;
              if (scale < FLT_MIN) scale = FLT_MIN;  // (not 0, by which -inf would not stay)
              row_keys({x.row0, x.n, x.len, x.pos0}, a.w.window, (y.r0 + own) / a.w.group, lo, hi);
            }
            return true;
          },
          [&](const Piece& x, const Span& y, int kt, int key, int) {
            if (((kt - x.t0) & 1) != set) return true;
            const int place = key % kS, j0 = kt * kTile;
            if (!wait(L::kSFull + place, (uint32_t)(key / kS) & 1u)) return false;
            tc_fence_after();
            const uint32_t note = smem + L::GONE + 16u * (key % L::NOTES);
            const uint4 gone = ld_shared16(note);
            const bool edge = j0 < y.all_lo || j0 + kTile > y.all_hi || (gone.x | gone.y | gone.z | gone.w) != 0;
            const unsigned long long scale2 = p2(scale, scale);
            over_chunks(lanes + 128u * place, [&](int c, uint32_t (&r)[32]) {
              if constexpr (I8) {
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                  const uint4 w = ld_shared16(smem + L::SCALE + 4u * (key % L::NOTES * kTile + 32 * c + k));
                  mul2(r[k], r[k + 1], w.x, w.y);
                  mul2(r[k + 2], r[k + 3], w.z, w.w);
                }
              }
              if (edge) {
                const uint32_t g = c == 0 ? gone.x : (c == 1 ? gone.y : (c == 2 ? gone.z : gone.w));
                const int from = lo - j0 - 32 * c, to = hi - j0 - 32 * c;
#pragma unroll
                for (int k = 0; k < 32; ++k) {  // (-inf: see infinities())
                  if (!I8 && r[k] == 0xff800000u) r[k] = 0x7fc00000u;
                  if (k < from || k >= to || (g >> k & 1u)) r[k] = 0xff800000u;
                }
              }
              float top[2] = {__uint_as_float(r[0]), __uint_as_float(r[1])};
#pragma unroll
              for (int k = 2; k < 32; k += 4) {
                top[0] = max3(top[0], __uint_as_float(r[k]), __uint_as_float(r[k + 1]));
                if (k + 3 < 32) top[1] = max3(top[1], __uint_as_float(r[k + 2]), __uint_as_float(r[k + 3]));
              }
              const float t = fmaxf(top[0], top[1]) * scale;
              if (t > m) {
                l *= exp2_approx(m - t);
                m = t;
              }
              const float base = m == -INFINITY ? 0.f : -m;
              const unsigned long long base2 = p2(base, base);
              unsigned long long sum[2] = {p2(0.f, 0.f), p2(0.f, 0.f)};
#pragma unroll
              for (int k = 0; k < 32; k += 2) {
                float t0, t1;
                up2(fma2(p2(__uint_as_float(r[k]), __uint_as_float(r[k + 1])), scale2, base2), t0, t1);
                sum[k / 2 & 1] = add2(sum[k / 2 & 1], p2(exp2_approx(t0), exp2_approx(t1)));
              }
              float s0, s1;
              up2(add2(sum[0], sum[1]), s0, s1);
              l += s0 + s1;
            });
            tc_fence_before();
            arrive(L::kSFree + place);
            return true;
          },
          [&](const Piece& x, const Span& y, int) {
            if (own < y.rows) {
              const int64_t row = (int64_t)x.h * a.total + (int64_t)x.row0 * a.w.group + y.r0 + own;
              a.parts[(row * a.splits + x.split) * 2 + set] = make_float2(m, l);
            }
            return true;
          },
          nothing);
    } else {
      // Each group has half of the columns of every key tile; the second group adds its sums to the first one's.
      float sum[kMostTiles], before[kMostTiles];
      int slot[kMostTiles];  // of the thread's key of each, -1 where there is none
      int number = 0;        // of pieces
      // (int8: not in registers meanwhile)
      const uint32_t stash = smem + L::STASH + 4u * (2 * kMostTiles * kTile * set + own);
      ok = walk(
          [&](const Piece& x) {
#pragma unroll
            for (int i = 0; i < kMostTiles; ++i) sum[i] = 0.f;
            if (x.split >= 0) return true;
            slots_of(x, own, slot);
#pragma unroll
            for (int i = 0; i < kMostTiles; ++i)
              before[i] = set == 0 && slot[i] >= 0 && (x.t0 + i) * kTile + own < x.pos0 ? a.w.score[slot[i]] : 0.f;
            if constexpr (I8) {
#pragma unroll
              for (int i = 0; i < kMostTiles; ++i) {
                st_shared4(stash + 4u * kTile * i, (uint32_t)slot[i]);
                st_shared4(stash + 4u * kTile * (kMostTiles + i), __float_as_uint(before[i]));
              }
            }
            return true;
          },
          [&](const Piece&, const Span&, int tile) {
            return wait(L::kColFull + tile % kQStages, (uint32_t)(tile / kQStages) & 1u);
          },
          [&](const Piece& x, const Span& y, int kt, int key, int tile) {
            const int place = key % kS, j0 = kt * kTile, which = kt - x.t0;
            if (!wait(L::kSFull + place, (uint32_t)(key / kS) & 1u)) return false;
            tc_fence_after();
            float one;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(one) : "r"(smem + L::ONE + 4u * (tile % kQStages)));
            const bool general = j0 < y.all_lo || j0 + kTile > y.all_hi || one < 0.f;
            int from = 0, to = kTile;  // columns that see the thread's key
            if (general) {
              const int64_t i0 = max((int64_t)0, (int64_t)j0 + own - x.pos0);
              const int64_t i1 =
                  a.w.window == INT32_MAX ? x.n : min((int64_t)x.n, (int64_t)j0 + own - x.pos0 + a.w.window);
              from = (int)min((int64_t)kTile, max((int64_t)0, i0 * a.w.group - y.r0));
              to = (int)min((int64_t)kTile, max((int64_t)0, i1 * a.w.group - y.r0));
            }
            float ks = 1.f;
            if constexpr (I8)
              asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ks) : "r"(smem + L::SCALE + 4u * (key % L::NOTES * kTile + own)));
            const uint32_t col = smem + L::COL + 1024u * (tile % kQStages) + 256u * set;
            unsigned long long p[2] = {p2(0.f, 0.f), p2(0.f, 0.f)};
            uint32_t v[2][32];
            tmem_ld_32x32_begin(lanes + 128u * place + 64u * set, v[0]);
            tmem_ld_32x32_begin(lanes + 128u * place + 64u * set + 32u, v[1]);
            tmem_ld_wait(v[0]);
            tmem_ld_wait(v[1]);
            tc_fence_before();
            arrive(L::kSFree + place);
            // Any rows, any scales; or all rows (what is not there has an infinite lse) and one scale, where the lse are all that
            // is read: the same bits.
            auto add = [&](auto any) {
              const float both = any ? ks : ks * one;
              const unsigned long long ks2 = p2(both, both), zero2 = p2(-0.f, -0.f);
#pragma unroll
              for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                  const uint4 e4 = ld_shared16(col + 512u + 128u * c + 4u * k);  // -lse of four rows
                  uint4 x4;
                  if constexpr (any) x4 = ld_shared16(col + 128u * c + 4u * k);
#pragma unroll
                  for (int u = 0; u < 4; u += 2) {
                    const unsigned long long s = p2(__uint_as_float(v[c][k + u]), __uint_as_float(v[c][k + u + 1]));
                    const unsigned long long e2 = u == 0 ? p2(__uint_as_float(e4.x), __uint_as_float(e4.y))
                                                         : p2(__uint_as_float(e4.z), __uint_as_float(e4.w));
                    unsigned long long by = ks2;
                    if constexpr (any) {
                      by = u == 0 ? p2(__uint_as_float(x4.x), __uint_as_float(x4.y))
                                  : p2(__uint_as_float(x4.z), __uint_as_float(x4.w));
                      if constexpr (I8) by = fma2(ks2, by, zero2);
                    }
                    float t0, t1;
                    up2(fma2(s, by, e2), t0, t1);
                    float p0 = exp2_approx(t0), p1 = exp2_approx(t1);
                    if constexpr (any) {
                      const int at = 64 * set + 32 * c + k + u;
                      p0 = at >= from && at < to ? p0 : 0.f;
                      p1 = at + 1 >= from && at + 1 < to ? p1 : 0.f;
                    }
                    p[u / 2] = add2(p[u / 2], p2(p0, p1));
                  }
                }
              }
            };
            if (general) add(std::true_type());
            else add(std::false_type());
            float s0, s1, s2, s3;
            up2(p[0], s0, s1);
            up2(p[1], s2, s3);
            const float all = (s0 + s1) + (s2 + s3);
#pragma unroll
            for (int i = 0; i < kMostTiles; ++i) sum[i] += i == which ? all : 0.f;
            return true;
          },
          [&](const Piece&, const Span&, int tile) {
            arrive(L::kColEmpty + tile % kQStages);
            return true;
          },
          [&](const Piece& x) {
            if (x.split >= 0) {
              join_parts(x, own, set, sum);
              return true;
            }
            if constexpr (I8) {
#pragma unroll
              for (int i = 0; i < kMostTiles; ++i) {
                slot[i] = (int)ld_shared4(stash + 4u * kTile * i);
                before[i] = __uint_as_float(ld_shared4(stash + 4u * kTile * (kMostTiles + i)));
              }
            }
            // A piece at a time: neither group's barrier gets a phase ahead of its waiter.
            if (set == 1 && !wait(L::kFirst, (uint32_t)number & 1u)) return false;
            if (set == 0 && number > 0 && !wait(L::kSecond, (uint32_t)(number - 1) & 1u)) return false;
#pragma unroll
            for (int i = 0; i < kMostTiles; ++i) {
              const int j = (x.t0 + i) * kTile + own;
              if (set == 1) before[i] = slot[i] >= 0 ? a.w.score[slot[i]] : 0.f;
              else before[i] = j < x.pos0 ? before[i] * a.w.decay : 0.f;
            }
#pragma unroll
            for (int i = 0; i < kMostTiles; ++i)
              if (slot[i] >= 0) a.w.score[slot[i]] = before[i] + sum[i];
            arrive(set == 0 ? L::kFirst : L::kSecond);
            ++number;
            return true;
          });
    }
    if (!ok && lane == 0) give_up();
  }
};

template <int D, bool I8, bool SUM>
__global__ void __launch_bounds__(I8 ? kThreadsI8 : kThreads, 1)
weigh_tc_kernel(const __grid_constant__ TcArgs a, const __grid_constant__ CUtensorMap map_hi,
                const __grid_constant__ CUtensorMap map_lo, const __grid_constant__ CUtensorMap map_k) {
  using L = Layout<D, I8>;
  extern __shared__ __align__(1024) uint8_t base[];
  const uint32_t smem = smem_u32(base);
  volatile int* abort = reinterpret_cast<volatile int*>(base + L::MISC);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base + L::MISC + 8);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  if (smem & 1023u) {  // the swizzled tiles need it; never taken where the declared alignment holds
    if (threadIdx.x == 0) atomicOr(a.w.batch.status, kStatusTimeout);
    return;
  }
  if (threadIdx.x == 0) {
    auto init = [&](int i, int count) { mbar_init(smem + L::BARS + 8u * i, count); };
    for (int s = 0; s < L::STAGES; ++s) {
      init(L::kKFull + s, I8 ? 4 : 1);
    }
    for (int s = 0; s < kQStages; ++s) {
      init(L::kQFull + s, 1);
      init(L::kQEmpty + s, 1);
      init(L::kColFull + s, 1);
      init(L::kColEmpty + s, kEpilogue);
    }
    for (int s = 0; s < kS; ++s) {
      init(L::kSFull + s, 2);  // the products, and the issuer for what it has seen of the key tile's notes
      init(L::kSFree + s, SUM ? kEpilogue : kEpilogue / 2 + (I8 ? 0 : 1));
    }
    // issuer, loader, epilogue and, where they work, warp 2 or 3 and the widening warps
    const int readers = 2 + kEpilogue + (SUM || !I8 ? 1 : 0) + (I8 ? 8 : 0);
    for (int s = 0; s < kPieces; ++s) {
      init(L::kPieceFull + s, 1);
      init(L::kPieceFree + s, readers);
    }
    init(L::kFirst, kEpilogue / 2);
    init(L::kSecond, kEpilogue / 2);
    init(L::kDrain, 1);
    *abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async_smem();
  }
  if (warp == 0) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // (the plan is from the launch before the last: the second pass's loader need not wait)
  if (!SUM || warp != 1) pdl_wait();
  pdl_trigger();
  const Kernel<D, I8, SUM> k{a, map_hi, map_lo, map_k, smem, __shfl_sync(0xffffffffu, *tmem_slot, 0), abort,
                             reinterpret_cast<Piece*>(base + L::PIECES)};
  // int8: 96 registers a thread at the start; 64 + 2 x 120 + 2 x 88 <= 5 x 96
  if (warp < 4) {
    if constexpr (I8) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == 0) k.issuer();
    else if (warp == 1) k.loader();
    else if (SUM && warp == 2) k.columns();
    else if (!SUM && !I8 && warp == 3) k.infinities();
  } else if (warp < 4 + kEpilogue) {
    if constexpr (I8) asm volatile("setmaxnreg.inc.sync.aligned.u32 120;");
    k.epilogue();
  } else if constexpr (I8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    k.widen();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(k.tmem, kTmemCols);
  }
}

// Between the passes, a thread a row: its lse, of rows that see nothing one that leaves nothing.
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads) weigh_join_rows_kernel(const __grid_constant__ TcArgs a) {
  pdl_trigger();
  const int64_t row0 = (int64_t)blockIdx.x * kJoinThreads + (threadIdx.x & ~31), row = row0 + (threadIdx.x & 31);
  const int64_t all = a.total * a.w.cache.heads;
  const int group = a.w.group;
  // What the first pass does not write is looked up while it ends: the row's sequence and the keys that it sees.
  int lo = 0, hi = 0;
  const int64_t first = quotient(min(row0, all - 1) % a.total, group);  // the warp's first token
  int b = paged_find(a.w.batch.row_start, a.w.batch.seqs, first);
  if (row < all) {
    const int64_t token = quotient(row % a.total, group);
    if (token < first || (b + 1 < a.w.batch.seqs && __ldg(a.w.batch.row_start + b + 1) <= token)) {  // not the first one's sequence
      int end = a.w.batch.seqs;
      for (b = token < first ? 0 : b; end - b > 1;) {
        const int mid = (b + end) >> 1;
        if (__ldg(a.w.batch.row_start + mid) <= token) b = mid;
        else end = mid;
      }
    }
    const PagedSeq s = paged_seq(a.w.batch, a.w.cache.page_shift, b);
    const int64_t i = token - s.row0;
    if (i >= 0 && i < s.n) row_keys(s, a.w.window, (int)i, lo, hi);
  }
  const int keys = a.plan->range * kTile, end = lo < hi ? (hi - 1) / keys : -1;
  pdl_wait();
  if (row >= all) return;
  float m = -INFINITY, l = a.rows[row].y;
  const float4* parts = reinterpret_cast<const float4*>(a.parts) + row * a.splits;
  for (int split = lo / keys; split <= end; split += 8) {
    float4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = split + i <= end ? parts[split + i] : make_float4(-INFINITY, 0.f, -INFINITY, 0.f);
    float top = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(v[i].x, v[i].z));
    const float base = top == -INFINITY ? 0.f : top;
    l *= exp2_approx(m - base);
#pragma unroll
    for (int i = 0; i < 8; ++i) l += v[i].y * exp2_approx(v[i].x - base) + v[i].w * exp2_approx(v[i].z - base);
    m = top;
  }
  a.rows[row].y = l == 0.f ? INFINITY : m + log2f(l);
}

int splits_of(const PagedCache& c, const PagedBatch& b) {
  const int64_t tiles = ceil_div(b.max_pages << c.page_shift, kTile);
  return (int)std::max<int64_t>(8, ceil_div(tiles, kMostRange));
}
struct Sizes {
  size_t q, rows, parts, plan, sums;
};
Sizes sizes_of(const PagedCache& c, const PagedBatch& b, int64_t q_heads, int head_dim) {
  const int64_t rows = b.rows * q_heads;
  return {(size_t)rows * head_dim * 2, (size_t)round_up(rows * sizeof(float2), 16),
          (size_t)rows * splits_of(c, b) * 2 * sizeof(float2),
          (size_t)round_up(sizeof(WeighPlan) + (int64_t)b.seqs * 2 * sizeof(int64_t), 16),
          (size_t)kSumTiles * (2 * kTile * sizeof(float) + 4 * sizeof(unsigned))};
}

template <int D, bool I8, bool SUM>
spl_status launch_pass(const TcArgs& a, const CUtensorMap (&maps)[3], int blocks, cudaStream_t stream) {
  constexpr uint32_t smem = Layout<D, I8>::SMEM;
  static bool done[kMaxDevices] = {false};
  if (!allow_shared(reinterpret_cast<const void*>(weigh_tc_kernel<D, I8, SUM>), smem, done)) return SPL_ECUDA;
  return launch_pdl(weigh_tc_kernel<D, I8, SUM>, dim3(blocks), dim3(I8 ? kThreadsI8 : kThreads), smem, stream, a, maps[0],
                    maps[1], maps[2]);
}

template <int D, bool I8>
spl_status launch(const TcArgs& a, int blocks, cudaStream_t stream) {
  const WeighCall& w = a.w;
  CUtensorMap maps[3] = {};
  const int64_t rows = a.total * w.cache.heads, slots = (int64_t)w.cache.pages * w.cache.heads << w.cache.page_shift;
  if (!tma_panel_map(&maps[0], a.q_hi, rows, D, kTile) || !tma_panel_map(&maps[1], a.q_lo, rows, D, kTile)) return SPL_ECUDA;
  if (!I8 && !tma_panel_map(&maps[2], w.cache.k, slots, D, std::min(kTile, 1 << w.cache.page_shift))) return SPL_ECUDA;
  const int64_t warps = ceil_div(rows * (D / 4), 32);
  const unsigned prep = 1 + (unsigned)std::min<int64_t>(ceil_div(warps, kPrepThreads / 32), 8 * blocks);
  weigh_prepare_kernel<D><<<prep, kPrepThreads, 0, stream>>>(a, blocks);
  spl_status st = launch_status();
  if (st != SPL_OK) return st;
  if ((st = launch_pass<D, I8, false>(a, maps, blocks, stream)) != SPL_OK) return st;
  st = launch_pdl(weigh_join_rows_kernel, dim3((unsigned)ceil_div(rows, kJoinThreads)), dim3(kJoinThreads), 0, stream, a);
  if (st != SPL_OK) return st;
  return launch_pass<D, I8, true>(a, maps, blocks, stream);
}

}  // namespace

size_t weigh_tc_bytes(const PagedCache& c, const PagedBatch& b, int64_t q_heads, int head_dim) {
  const Sizes s = sizes_of(c, b, q_heads, head_dim);
  return 2 * s.q + s.rows + s.parts + s.plan + s.sums;
}

spl_status run_weigh_tc(const WeighCall& w, int head_dim, bool i8, cudaStream_t stream) {
  const Sizes s = sizes_of(w.cache, w.batch, w.q_heads, head_dim);
  TcArgs a = {};
  a.w = w;
  char* at = static_cast<char*>(w.workspace);
  a.q_hi = reinterpret_cast<uint16_t*>(at);
  a.q_lo = reinterpret_cast<uint16_t*>(at + s.q);
  a.parts = reinterpret_cast<float2*>(at + 2 * s.q);
  a.rows = reinterpret_cast<float2*>(at + 2 * s.q + s.parts);
  a.plan = reinterpret_cast<WeighPlan*>(at + 2 * s.q + s.parts + s.rows);
  a.sums = reinterpret_cast<float*>(at + 2 * s.q + s.parts + s.rows + s.plan);
  a.arrived = reinterpret_cast<unsigned*>(a.sums + (size_t)kSumTiles * 2 * kTile);
  a.first[0] = reinterpret_cast<int64_t*>(a.plan + 1);
  a.first[1] = a.first[0] + w.batch.seqs;
  a.splits = splits_of(w.cache, w.batch);
  a.total = w.batch.rows * w.group;
  const int blocks = device_sm_count();
  if (head_dim == 128) return i8 ? launch<128, true>(a, blocks, stream) : launch<128, false>(a, blocks, stream);
  return i8 ? launch<64, true>(a, blocks, stream) : launch<64, false>(a, blocks, stream);
}

}  // namespace spl
