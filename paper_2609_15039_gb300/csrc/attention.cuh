// Attention over a paged cache: the work and its division among the blocks, shared by both kernels.
//
// The rows of a sequence that read one key head are its n tokens' `group` query heads, r = i group + g.  A tile is RT
// of them; the keys it sees are [key_lo, key_hi), cut into units of U keys.  All units of all tiles, key heads and
// sequences in a row are dealt to the blocks in equal contiguous runs, whatever the lengths (which only the device
// knows), so a block works on pieces of tiles.  A piece that is a whole tile is finished by its block.  The pieces of
// a divided one go to the workspace as (sums, maximum, total) and the last block to arrive joins them in the order of
// the blocks: the result does not depend on timing.  A block leaves at most one piece that begins inside a tile
// (slot 0) and one that only ends inside one (slot 1).  The runs are equal in steps: a tile has a step for each unit and
// `start` before them, in which nothing is done: what a tile's beginning costs a block.  (With equal runs of units the
// blocks of short sequences have most tiles: 64 int8 sequences of one row over 100 to 1360 keys 47 us instead of 37, 2000
// rows over themselves 120 instead of 80.)
// A further piece costs a block as much as several units.  So where there are few tiles, each is cut into pieces of
// `grain` units, the least of kGrains with which every piece has a block of its own, if that is little above the mean
// (512 rows over themselves, 96 tiles of 1 to 4 units: 29 us in equal runs, 23 in pieces of 2, 20.6 as whole tiles; 15
// short int8 sequences of one row 17.8, 16.5, 14.2).
#pragma once

#include "paged.cuh"

namespace spl {

struct AttnArgs {
  float* out;
  const float* q;
  int64_t ldo, ldq;
  PagedCache cache;
  PagedBatch batch;
  int group;         // query heads of a key head
  int window;        // keys a row sees, INT_MAX for all
  float scale_log2;  // scale log2(e): softmax in powers of two
  unsigned int* counters;
  float* slots;      // [blocks][2][slot floats]
  // Units that a piece has at least, that it may have above the mean for being a block's only one, that a join costs, that
  // the start of a tile costs.
  int least, slack, join, start;
};

constexpr int kFewTiles = 4;  // tiles of a sequence that one thread counts
constexpr int kGrains = 8;    // 1 to 8 units

struct AttnTile {
  int b, h, t;           // sequence, key head, tile
  PagedSeq s;
  int r0, rows;          // rows [r0, r0 + rows) of the (sequence, key head)
  int key_lo, key_hi;    // keys that some row sees
  int all_lo, all_hi;    // keys that every row sees
  int unit0, units;      // units [unit0, unit0 + units), at least one
};

// Keys [lo, hi) that token i of sequence s sees.
__device__ __forceinline__ void row_keys(const PagedSeq& s, int window, int i, int& lo, int& hi) {
  const int pos = s.pos0 + i;
  hi = max(0, min(pos + 1, s.len));
  lo = pos >= window ? min(pos - window + 1, hi) : 0;
}

template <int RT, int U>
__device__ __forceinline__ void tile_span(AttnTile& x, int group, int window) {
  x.r0 = x.t * RT;
  x.rows = min(RT, x.s.n * group - x.r0);
  row_keys(x.s, window, x.r0 / group, x.key_lo, x.all_hi);
  row_keys(x.s, window, (x.r0 + x.rows - 1) / group, x.all_lo, x.key_hi);
  x.unit0 = x.key_lo / U;
  x.units = max(1, (x.key_hi + U - 1) / U - x.unit0);
}

// a / b of numbers from 0 on, in 32 bits where they fit: a 64-bit division costs some hundred cycles.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// A block's run of units.  `prefix` (shared, kPrefixBytes a sequence and kGrains numbers for each of as many as there are
// blocks) is filled by the constructor, which every thread of the block calls; afterwards every thread walks the same
// tiles by itself.
constexpr int kPrefixBytes = 8 + sizeof(PagedSeq);
template <int RT, int U, int THREADS>
struct AttnRun {
  AttnTile x;
  int grain, start;        // units of a step; steps before a tile's units
  int64_t total, at, end;  // steps in all; the run [at, end)
  int blocks;              // blocks that have work
  int64_t off;             // step of the current tile at which the run stands
  int first;               // and unit
  const AttnArgs& a;

  // The sequences, behind the prefix sums, and their steps of each grain.
  __device__ PagedSeq& kept(int64_t* prefix, int b) const {
    return reinterpret_cast<PagedSeq*>(prefix + a.batch.seqs)[b];
  }
  __device__ int* steps(int64_t* prefix, int b) const {
    return reinterpret_cast<int*>(&kept(prefix, a.batch.seqs)) + kGrains * b;
  }
  __device__ AttnRun(const AttnArgs& args, int64_t* prefix) : grain(1), start(args.start), a(args) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int seqs = a.batch.seqs, heads = a.cache.heads;
    const bool few = seqs * heads <= (int)gridDim.x;  // a block for each piece is possible
    // A thread a sequence, whose loads then run side by side; the few sequences of many tiles a warp each.
    for (int b = threadIdx.x; b < seqs; b += THREADS) {
      AttnTile y;
      y.s = paged_seq(a.batch, a.cache.page_shift, b);
      kept(prefix, b) = y.s;
      const int tiles = (y.s.n * a.group + RT - 1) / RT;
      int64_t sum = 0;
      int of[kGrains] = {};
      for (y.t = 0; tiles <= kFewTiles && y.t < tiles; ++y.t) {
        tile_span<RT, U>(y, a.group, a.window);
        sum += y.units;
#pragma unroll
        for (int k = 0; k < kGrains; ++k) of[k] += (int)((uint32_t)(y.units + k) / (uint32_t)(k + 1));
      }
      prefix[b] = tiles <= kFewTiles ? (sum + start * tiles) * heads : -1;
      if (few)
#pragma unroll
        for (int k = 0; k < kGrains; ++k) steps(prefix, b)[k] = of[k];
    }
    __syncthreads();
    for (int b = warp; b < seqs; b += THREADS / 32) {
      if (prefix[b] >= 0) continue;
      AttnTile y;
      y.s = kept(prefix, b);
      const int tiles = (y.s.n * a.group + RT - 1) / RT;
      int64_t sum = 0;
      int of[kGrains] = {};
      for (y.t = lane; y.t < tiles; y.t += 32) {
        tile_span<RT, U>(y, a.group, a.window);
        sum += y.units;
        if (!few || tiles > (int)gridDim.x) continue;
#pragma unroll
        for (int k = 0; k < kGrains; ++k) of[k] += (int)((uint32_t)(y.units + k) / (uint32_t)(k + 1));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (few) {
#pragma unroll
        for (int k = 0; k < kGrains; ++k) {
          const int all = __reduce_add_sync(0xffffffffu, of[k]);
          if (lane == k) steps(prefix, b)[k] = tiles > (int)gridDim.x ? (int)gridDim.x + 1 : all;
        }
      }
      __syncwarp();
      if (lane == 0) prefix[b] = (sum + (int64_t)start * tiles) * heads;
    }
    __syncthreads();
    if (warp == 0) {
      const int64_t steps_in_all = scan(prefix, seqs);
      if (few && steps_in_all <= (int64_t)(kGrains + start) * gridDim.x) grain = choose_grain(prefix, (int)steps_in_all);
      else grain = 0;
      if (lane == 0) *steps(prefix, few ? seqs : 0) = grain;
    }
    __syncthreads();
    grain = *steps(prefix, few ? seqs : 0);
    if (grain > 0) start = 0;  // a piece a block
    else grain = 1;
    total = seqs > 0 ? prefix[seqs - 1] : 0;
    blocks = (int)min((int64_t)gridDim.x, max((int64_t)1, total));
    const int c = blockIdx.x;
    at = c < blocks ? quotient(total * c, blocks) : 0;
    end = c < blocks ? quotient(total * (c + 1), blocks) : 0;
    if (at >= end) return;
    int lo = 0, hi = seqs - 1;  // the first sequence whose prefix passes `at`
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (prefix[mid] > at) hi = mid;
      else lo = mid + 1;
    }
    x.b = lo;
    const int64_t before = lo > 0 ? prefix[lo - 1] : 0;
    const int64_t per_head = quotient(prefix[lo] - before, heads);
    x.h = (int)quotient(at - before, per_head);
    int64_t rest = at - before - x.h * per_head;
    x.s = kept(prefix, x.b);
    const int tiles = (x.s.n * a.group + RT - 1) / RT;
    for (int t0 = 0;; t0 += 32) {  // the tile that holds step `rest`, 32 at a time
      AttnTile y;
      y.s = x.s;
      y.t = t0 + lane;
      int64_t v = 0;
      if (y.t < tiles) {
        tile_span<RT, U>(y, a.group, a.window);
        v = start + steps_of(y.units);
      }
      const int64_t own = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t other = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += other;
      }
      const unsigned past = __ballot_sync(0xffffffffu, v > rest);
      if (past || t0 + 32 >= tiles) {
        const int l = past ? __ffs(past) - 1 : 0;
        x.t = t0 + l;
        rest -= __shfl_sync(0xffffffffu, v - own, l);
        break;
      }
      rest -= __shfl_sync(0xffffffffu, v, 31);
    }
    off = rest;
    first = (int)max((int64_t)0, rest - start) * grain;
    tile_span<RT, U>(x, a.group, a.window);
    if (off + (end - at) <= start) at = end;
  }
  // The grain by which all pieces have blocks, and then the prefix sums are of its steps, or 0; by warp 0, of `sum` steps
  // in all.  Whole tiles, which need no join, where they are little longer.
  __device__ int choose_grain(int64_t* prefix, int sum) const {
    const int lane = threadIdx.x & 31, seqs = a.batch.seqs, heads = a.cache.heads, grid = (int)gridDim.x;
    int tiles = 0, split = 0, whole = 0;
    for (int b = lane; b < seqs; b += 32) tiles += (kept(prefix, b).n * a.group + RT - 1) / RT;
    tiles = min(__reduce_add_sync(0xffffffffu, tiles), 1 << 20) * heads;
    const int mean = max(1, (int)((uint32_t)(sum - start * tiles + grid - 1) / (uint32_t)grid));
    for (int k = mean; k <= kGrains && k <= (split ? split : mean + a.slack) + a.join; ++k) {
      int n = 0;
      for (int b = lane; b < seqs; b += 32) n += steps(prefix, b)[k - 1];
      n = __reduce_add_sync(0xffffffffu, n) * heads;
      if (split == 0 && n <= grid && k >= a.least && k <= max(mean + a.slack, a.least)) split = k;
      if (n == tiles) {
        whole = n <= grid ? k : 0;
        break;
      }
    }
    const int g = whole ? whole : split;
    if (g > 0) {
      for (int b = lane; b < seqs; b += 32) prefix[b] = (int64_t)steps(prefix, b)[g - 1] * heads;
      __syncwarp();
      scan(prefix, seqs);
    }
    return g;
  }
  // Sums up to each in place, by a warp; returns the last.
  static __device__ int64_t scan(int64_t* prefix, int seqs) {
    const int lane = threadIdx.x & 31;
    int64_t carry = 0;
    for (int b0 = 0; b0 < seqs; b0 += 32) {
      int64_t v = b0 + lane < seqs ? prefix[b0 + lane] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t other = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += other;
      }
      v += carry;
      if (b0 + lane < seqs) prefix[b0 + lane] = v;
      carry = __shfl_sync(0xffffffffu, v, 31);
    }
    return carry;
  }
  __device__ int steps_of(int units) const { return grain == 1 ? units : (units + grain - 1) / grain; }

  __device__ bool busy() const { return at < end; }
  // Units [first, last()) of the tile are the block's piece.
  __device__ int last() const { return (int)min((int64_t)x.units, (off + (end - at) - start) * grain); }
  __device__ bool whole() const { return first == 0 && last() == x.units; }
  __device__ int block_of(int64_t step) const { return (int)quotient((step + 1) * blocks - 1, total); }
  __device__ int first_block() const { return block_of(at - off + start); }
  __device__ int last_block() const { return block_of(at - off + start + steps_of(x.units) - 1); }

  __device__ void next() {
    at += start + steps_of(x.units) - off;
    off = 0;
    first = 0;
    if (end - at <= start) at = end;
    if (at >= end) return;
    ++x.t;
    if ((int64_t)x.t * RT >= (int64_t)x.s.n * a.group) {
      x.t = 0;
      if (++x.h == a.cache.heads) {
        x.h = 0;
        do x.s = paged_seq(a.batch, a.cache.page_shift, ++x.b);
        while (x.s.n == 0 && x.b + 1 < a.batch.seqs);
      }
    }
    tile_span<RT, U>(x, a.group, a.window);
  }
};

// ---- arithmetic shared by the kernels ----
// 2^x, relative error about 2^-22; 2^-inf = 0.
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two fp32 as binary16 in one register, the first in the low half.
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t h) {
  float2 r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "r"(h));
  return r;
}
// Whether a pair of binary16 holds an infinity or NaN.
__device__ __forceinline__ bool f16_special(uint32_t h) {
  return (h & 0x7c00u) == 0x7c00u || (h & 0x7c000000u) == 0x7c000000u;
}
// (a, b) = hi + lo, each a pair of binary16: 22 significant bits above 2^-14, an absolute 2^-25 below.
__device__ __forceinline__ void split_f16(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack_f16(a, b);
  const float2 h = unpack_f16(hi);
  lo = pack_f16(__fsub_rn(a, h.x), __fsub_rn(b, h.y));
}
__device__ __forceinline__ float exp2_int(int e) { return e < -126 ? 0.0f : __int_as_float((e + 127) << 23); }
// Four int8 (as stored) to two pairs of binary16, exactly: 1024 + 128 + x, less 1152.
__device__ __forceinline__ uint32_t i8_pair(uint32_t bytes, uint32_t select) {
  const uint32_t magic = 0x64646464u, bias = 0x64806480u;
  uint32_t r = __byte_perm(bytes, magic, select), d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(r), "r"(bias));
  return d;
}

constexpr int kSlotStats = 2;  // per row: maximum (in units of log2) and total

// The two kernels' launches and the workspace behind the counters.
spl_status run_attention_tc(const AttnArgs& a, int head_dim, bool i8, int blocks, cudaStream_t stream);
size_t attention_tc_bytes(int head_dim, int blocks);
spl_status run_attention_rows(const AttnArgs& a, int head_dim, bool i8, int blocks, cudaStream_t stream);

}  // namespace spl
