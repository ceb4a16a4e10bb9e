// Attention of few rows over a paged cache (decode), and the entry points.
//
// o = sum_j softmax_j(scale q . k_j) v_j, in one pass over the keys with a running maximum m, total l and sums O.
// For few rows the pass is bound by reading the cache once.  A tile has 8 rows (for one new token, the query heads of
// a key head); its products run on mma.m16n8k16.  q . k: the 8 rows' high and low halves are the 16 rows of A, so that one
// instruction makes both terms of q = (hi + lo) 2^-e.  p . v is made transposed, v^T as A and the low, then the high
// halves of p as B.  The stored binary16 (or int8) values are exact in those products: fp32 accuracy.  The tensor core
// truncates as it accumulates, so the products of 16 keys are added to the sums by themselves, rounding to nearest (131072
// keys in one piece were off by up to 5e-5 in one chain; the additions cost int8 1%, binary16 nothing).
// A block has an SM.  Two or four warps copy units of 128 or 256 keys (some 64 KB of keys and values) into a ring by bulk copies
// of whole runs of a page, so that some 190 KB are on their way on an SM, across the ends of tiles and sequences; 8 warps
// make the sums, each of its 16 or 32 keys of a unit.  The order of the dimensions in a product is free, so a lane reads
// 16 neighbouring bytes for its fragments (dims of a key for q . k, dims of four keys for p . v, whose pairs of keys
// are byte permutes).
// Measured with 64 sequences of 1600 to 15775 keys, one row, 24 query heads on 8, 128 dims: binary16 329 us (the rate of
// a copy), int8 191 us (0.91 of it: bound by widening int8 to binary16); one sequence of 300 keys 10 us, bound by the
// latency of a launch, four dependent loads and three units.  Tiles of 16 to 32 rows, which would share the reads, were not
// faster as they were built: 16 sequences of 8 rows of 4 heads 147 us as one tile of 32 and 137 as four of 8, some 36 us
// an eight of rows, 4.5 times what its products take at the instruction's rate.  That is latency, not a bound.

#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "attention.cuh"
#include "ptx.cuh"

namespace spl {
namespace {

constexpr int kWarps = 8, kThreads = 32 * (kWarps + 4);  // and a warpgroup that copies
constexpr int kRT = 8;  // rows of a tile
// p is held as 2^kShift p, at most 2^13, so that its low half keeps an absolute 2^-38 of the largest.
constexpr float kShift = 13.0f, kUnshift = 0x1p-13f;
constexpr int kMinExp = -100, kMaxExp = 126;  // of the values' scales

__device__ __forceinline__ void mma16816(float (&c)[4], const uint4& a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
template <class T>
__device__ __forceinline__ T lds(const uint8_t* p) {
  return *reinterpret_cast<const T*>(p);
}
// How a lane (g = lane / 4, t = lane % 4) holds 16 keys, and which dimensions those are.
template <int D, bool I8>
struct Frag {
  static constexpr int E = I8 ? 16 : 8;            // elements of 16 bytes
  static constexpr int KB = D / (4 * E);           // keys g and g + 8: 16-byte chunks of each
  static constexpr int STEPS = D / 16;             // k-steps of q . k
  static constexpr int VE = I8 ? D / 8 : 8;        // keys 2t, 2t+1, 2t+8, 2t+9: neighbouring dims of a chunk
  static constexpr int VC = D / (8 * VE);          // and chunks
  static constexpr int VW = VE * (I8 ? 1 : 2) / 4; // words of a chunk
  static constexpr int MB = D / 16;                // m-blocks of v^T . p^T
  // first of the two neighbours (first + {0, 1}, and + {2, 3} for the upper half of a k-step) of step s
  static __device__ __forceinline__ int k_dim(int s, int t) {
    constexpr int per = E / 4;  // steps a chunk
    return (s / per) * 4 * E + t * E + 4 * (s % per);
  }
  // A ring stage, of BLOCKS blocks of 16 keys a warp: keys, values, and the scales of both.
  static constexpr int ESZ = I8 ? 1 : 2, BLOCKS = D * ESZ == 256 ? 1 : 2, UNIT = 16 * kWarps * BLOCKS;
  static constexpr uint32_t K = 0, V = UNIT * D * ESZ, KS = 2 * V, VS = KS + (I8 ? UNIT * 4 : 0);
  static constexpr uint32_t STAGE = VS + (I8 ? UNIT * 4 : 0);
  static constexpr int STAGES = V > 24576 ? 3 : 4;
  static constexpr int COPIERS = I8 ? 4 : 2;  // copying warps
  static constexpr uint32_t RING = STAGES * STAGE;
  // shared memory: the ring (the prefix sums before it), sums of four warps, maxima and totals, barriers (full, empty) and
  // the mask of a stage's blocks that hold keys
  static constexpr int PARTS = 4;
  static constexpr uint32_t SO = RING, SM = SO + PARTS * kRT * D * 4, SL = SM + kWarps * kRT * 4;
  static constexpr uint32_t BARS = SL + kWarps * kRT * 4, MASK = BARS + 16 * STAGES, LAST = MASK + 4 * STAGES;
  static constexpr uint32_t SMEM = LAST + 8;
  static_assert(SMEM <= 232448 && kMaxSeqs * kPrefixBytes + 8192 <= RING, "fits");
  // dim n of the nb-th eight; an m-block is two of them
  static __device__ __forceinline__ int v_dim(int nb, int n) { return (nb / VE) * 8 * VE + n * VE + nb % VE; }
};

// A copying warp: unit after unit of the block's run into the ring's stages in turn.  Each has a part of what a unit
// consists of (keys, values, their scales): with pages of 16 tokens, 64 copies a unit, one warp alone was the
// bound (64 sequences of one row over 1600 to 15775 keys, int8, 352 us instead of 193).  Each arrives at every unit, also
// where it copies nothing: none can fall a turn of the ring behind the others and wait for a phase that has passed.
template <int D, bool I8, bool TREE>
__device__ void copy_units(AttnRun<kRT, Frag<D, I8>::UNIT, kThreads, TREE>& run, uint8_t* smem, int part) {
  using F = Frag<D, I8>;
  constexpr int BLOCKS = F::UNIT / 16;
  const PagedCache& cache = run.a.cache;
  const int lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem), bars = base + F::BARS;
  const uint64_t policy = l2_evict_first();
  const int per_page = min(BLOCKS, 1 << (cache.page_shift - 4));  // blocks of a unit that lie side by side
  volatile int* abort = reinterpret_cast<volatile int*>(smem + F::LAST + 4);
  int it = 0;
  bool ok = true;
  for (; ok && run.busy(); run.next()) {
    const AttnTile& x = run.x;
    const int last = run.last();
    int64_t slot = -1;  // of the first key of the lane's block of 16, -1 where no row sees any
    auto look_up = [&](int u) {
      const int j = (x.unit0 + u) * F::UNIT + 16 * lane;
      slot = -1;
      if (lane < BLOCKS && u < last && j < x.key_hi && j + 16 > x.key_lo) {
        const int page = paged_page(cache, run.a.batch, x.b, j);
        if (page >= 0) slot = paged_slot(cache, page, x.h, j);
      }
    };
    look_up(run.first);
    for (int u = run.first; u < last; ++u, ++it) {
      const int stage = it % F::STAGES;
      const uint32_t at = base + stage * F::STAGE, full = bars + 8u * stage;
      if (it >= F::STAGES) {
        ok = __all_sync(0xffffffffu, mbar_wait_soon(bars + 8u * (F::STAGES + stage), (uint32_t)(it / F::STAGES - 1) & 1u,
                                               kWaitNs, abort));
        if (!ok) break;
      }
      const uint32_t mask = __ballot_sync(0xffffffffu, slot >= 0);
      // The first block of a run of them in a page copies the run.
      const uint32_t page_mask = ((1u << per_page) - 1u) << (lane / per_page * per_page) & mask;
      const bool leads = slot >= 0 && (page_mask & ((1u << lane) - 1u)) == 0;
      const uint32_t keys = 16u * __popc(page_mask);
      if (part == 0 && lane == 0) {
        *reinterpret_cast<volatile uint32_t*>(smem + F::MASK + 4 * stage) = mask;
        mbar_expect_tx(full, 16u * __popc(mask) * (2u * D * F::ESZ + (I8 ? 8u : 0u)));
      } else if (lane == 0) {
        mbar_arrive(full);
      }
      __syncwarp();
      if (leads) {
        const uint32_t key0 = 16u * lane;
        const bool v = part & 1;
        if (part < 2)
          bulk_load(at + (v ? F::V : F::K) + key0 * D * F::ESZ,
                    static_cast<const char*>(v ? cache.v : cache.k) + slot * (D * F::ESZ), keys * D * F::ESZ, full, policy);
        else
          bulk_load(at + (v ? F::VS : F::KS) + key0 * 4u, (v ? cache.v_scale : cache.k_scale) + slot, keys * 4u, full,
                    policy);
      }
      look_up(u + 1);
    }
  }
  if (!ok) {  // given up: what is on its way lands before the block leaves
    *abort = 1;
    if (lane == 0) atomicOr(run.a.batch.status, kStatusTimeout);
    for (int t = max(0, it - F::STAGES); t < it; ++t)
      mbar_wait(bars + 8u * (t % F::STAGES), (uint32_t)(t / F::STAGES) & 1u, kDrainNs, nullptr);
  }
}

template <int D, bool I8, bool TREE>
__global__ void __launch_bounds__(kThreads, 1) attention_rows_kernel(const __grid_constant__ AttnArgs a) {
  using F = Frag<D, I8>;
  constexpr int ESZ = F::ESZ, BLOCKS = F::BLOCKS;
  constexpr int SLOT = kRT * (D + kSlotStats);
  extern __shared__ __align__(128) uint8_t smem[];
  auto s_o = reinterpret_cast<float(*)[kRT][D]>(smem + F::SO);
  auto s_m = reinterpret_cast<float(*)[kRT]>(smem + F::SM);
  auto s_l = reinterpret_cast<float(*)[kRT]>(smem + F::SL);
  volatile int* s_last = reinterpret_cast<volatile int*>(smem + F::LAST);
  volatile int* abort = s_last + 1;
  if (threadIdx.x == 0) *abort = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t bars = smem_u32(smem + F::BARS);
  if (threadIdx.x < 2 * F::STAGES) mbar_init(bars + 8u * threadIdx.x, threadIdx.x < F::STAGES ? F::COPIERS : kWarps);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  AttnRun<kRT, F::UNIT, kThreads, TREE> run(a, reinterpret_cast<int64_t*>(smem));
  fence_proxy_async_smem();
  __syncthreads();  // the prefix sums have been read: their place is the ring's
  // 168 registers a thread at the start; 3 x 168 = 2 x 232 + 40
  if (warp >= kWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp < kWarps + F::COPIERS) copy_units<D, I8, TREE>(run, smem, warp - kWarps);
    return;
  }
  asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
  auto sync = []() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory"); };  // the warps that sum
  int it = 0;
  for (; run.busy(); run.next()) {
    const AttnTile& x = run.x;
    // ---- the tile's rows: q = (hi + lo) 2^-e; the high halves are rows 0-7 of A, the low ones rows 8-15 ----
    const int r = min(x.r0 + g, x.r0 + x.rows - 1);  // rows past the last repeat it
    const int token = r / a.group;
    uint4 qa[F::STEPS];
    float row_scale;
    {
      const float* q = a.q + (x.s.row0 + token) * a.ldq + (int64_t)(x.h * a.group + r % a.group) * D;
      float4 v[F::STEPS];
      float top = 0.f;
#pragma unroll
      for (int s = 0; s < F::STEPS; ++s) {
        v[s] = __ldg(reinterpret_cast<const float4*>(q + F::k_dim(s, t)));
        top = fmaxf(fmaxf(fmaxf(top, fabsf(v[s].x)), fabsf(v[s].y)), fmaxf(fabsf(v[s].z), fabsf(v[s].w)));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = fp16_row_exponent(top);
      const float up = pow2f(e);
      row_scale = a.scale_log2 * pow2f(-e);
#pragma unroll
      for (int s = 0; s < F::STEPS; ++s) {
        split_f16(v[s].x * up, v[s].y * up, qa[s].x, qa[s].y);
        split_f16(v[s].z * up, v[s].w * up, qa[s].z, qa[s].w);
      }
    }
    int row_lo, row_hi;
    const uint32_t* seen = nullptr;  // (of a tree)
    if constexpr (TREE) {
      seen = a.seen + (x.s.row0 + token) * a.words;
      row_lo = tree_lo(seen, a.words, a.window, x.s.pos0, x.s.len);
      row_hi = x.s.len;
    } else {
      row_keys(x.s, a.window, token, row_lo, row_hi);
    }

    // The sums, transposed: dims (16 of an m-block) x rows; a lane has dims g, g + 8 and rows 2t, 2t + 1 of each.  (As rows
    // x dims, with the high and low halves of p as A, they would take twice the registers: 64 sequences, int8, 230 us
    // instead of 216.)
    float o[F::MB][4];
#pragma unroll
    for (int i = 0; i < F::MB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
    float m = -INFINITY, l = 0.f;
    int ev = kMinExp;  // the sums are in units of 2^ev (int8: the exponent of the largest scale met)

    const int u_end = run.last();
    for (int u = run.first; u < u_end; ++u, ++it) {
      const int stage = it % F::STAGES;
      const uint8_t* at = smem + stage * F::STAGE;
      const bool there =
          __all_sync(0xffffffffu, mbar_wait_soon(bars + 8u * stage, (uint32_t)(it / F::STAGES) & 1u, kWaitNs, abort));
      if (!there && lane == 0) {
        *abort = 1;
        atomicOr(a.batch.status, kStatusTimeout);
      }
      const int b0 = warp * BLOCKS;  // the warp's blocks of the unit
      const uint32_t mask = there ? *reinterpret_cast<volatile const uint32_t*>(smem + F::MASK + 4 * stage) >> b0 : 0u;
      const int j0 = (x.unit0 + u) * F::UNIT + 16 * b0;
      if (mask & ((1u << BLOCKS) - 1u)) {
        // ---- scores of keys 2t, 2t + 1, 2t + 8, 2t + 9 of each block and row g ----
        float s[4 * BLOCKS];
        {
          float acc[2][2 * BLOCKS][4] = {};  // two chains of products
#pragma unroll
          for (int i = 0; i < F::KB; ++i) {
            uint4 k16[2 * BLOCKS];
#pragma unroll
            for (int c = 0; c < 2 * BLOCKS; ++c)
              k16[c] = lds<uint4>(at + F::K + (16 * b0 + 8 * c + g) * (D * ESZ) + 64 * i + 16 * t);
#pragma unroll
            for (int c = 0; c < 2 * BLOCKS; ++c) {
              const uint32_t w[4] = {k16[c].x, k16[c].y, k16[c].z, k16[c].w};
              if constexpr (I8) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const uint32_t biased = w[k] ^ 0x80808080u;
                  mma16816(acc[k & 1][c], qa[4 * i + k], i8_pair(biased, 0x4140u), i8_pair(biased, 0x4342u));
                }
              } else {
                mma16816(acc[0][c], qa[2 * i], w[0], w[1]);
                mma16816(acc[1][c], qa[2 * i + 1], w[2], w[3]);
              }
            }
          }
#pragma unroll
          for (int c = 0; c < 2 * BLOCKS; ++c) {
            s[2 * c] = ((acc[0][c][0] + acc[1][c][0]) + (acc[0][c][2] + acc[1][c][2])) * row_scale;
            s[2 * c + 1] = ((acc[0][c][1] + acc[1][c][1]) + (acc[0][c][3] + acc[1][c][3])) * row_scale;
            if constexpr (I8) {
              const float2 sc = lds<float2>(at + F::KS + 4 * (16 * b0 + 8 * c + 2 * t));
              s[2 * c] *= sc.x;
              s[2 * c + 1] *= sc.y;
            }
          }
        }
        float vs[4 * BLOCKS];
        if constexpr (I8) {
#pragma unroll
          for (int c = 0; c < 2 * BLOCKS; ++c) {
            const float2 sc = lds<float2>(at + F::VS + 4 * (16 * b0 + 8 * c + 2 * t));
            vs[2 * c] = sc.x;
            vs[2 * c + 1] = sc.y;
          }
        }
        // A chunk of the values of keys 2t, 2t + 1, 2t + 8, 2t + 9 of a block.
        auto values = [&](int blk, int i, uint32_t (&vr)[4][F::VW]) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint8_t* p = at + F::V + (16 * (b0 + blk) + 8 * (c >> 1) + 2 * t + (c & 1)) * (D * ESZ) +
                               (g + 8 * i) * F::VE * ESZ;
            if constexpr (F::VW == 4) {
              const uint4 w = lds<uint4>(p);
              vr[c][0] = w.x, vr[c][1] = w.y, vr[c][2] = w.z, vr[c][3] = w.w;
            } else {
              const uint2 w = lds<uint2>(p);
              vr[c][0] = w.x, vr[c][1] = w.y;
            }
          }
        };
        // ---- softmax: blocks at an edge of what the rows see, and what no copy brought, mask by row ----
        const bool edge = j0 < x.all_lo || j0 + 16 * BLOCKS > x.all_hi || (~mask & ((1u << BLOCKS) - 1u)) != 0;
        uint32_t hidden = 0, zap = 0;  // bits: scores that the row does not see; keys whose values become zeros
        if (edge) {
          uint32_t bad = 0;  // keys whose values hold an infinity or NaN
          const uint32_t sees = TREE ? tree_keys(seen, a.words, x.s.pos0, row_lo, row_hi, j0) : 0u;
          if constexpr (!I8) {  // a value that only some rows see must not reach the others as 0 times NaN
#pragma unroll
            for (int blk = 0; blk < BLOCKS; ++blk) {
              bool special[4] = {false, false, false, false};
#pragma unroll
              for (int i = 0; i < F::VC; ++i) {
                uint32_t vr[4][F::VW];
                values(blk, i, vr);
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                  for (int w = 0; w < F::VW; ++w) special[c] |= f16_special(vr[c][w]);
              }
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const int j = j0 + 16 * blk + 8 * (c >> 1) + 2 * t + (c & 1);
                const unsigned who = __ballot_sync(0xffffffffu, special[c]);
                if (who & (0x11111111u << t)) bad |= 1u << (4 * blk + c);
                if ((bad >> (4 * blk + c) & 1u) || !(mask >> blk & 1u) || j < x.key_lo || j >= x.key_hi)
                  zap |= 1u << (4 * blk + c);
              }
            }
          }
#pragma unroll
          for (int c = 0; c < 4 * BLOCKS; ++c) {
            const int j = j0 + 16 * (c >> 2) + 8 * (c >> 1 & 1) + 2 * t + (c & 1);
            const bool out_of_sight = TREE ? !(sees >> (j - j0) & 1u) : j < row_lo || j >= row_hi;
            if (!(mask >> (c >> 2) & 1u) || out_of_sight) {
              s[c] = -INFINITY;
              hidden |= 1u << c;
            } else if (bad >> c & 1u) {
              s[c] = __int_as_float(0x7fc00000);
            }
          }
        }
        float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
        if constexpr (BLOCKS == 2) top = fmaxf(top, fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float m_new = fmaxf(m, top);
        int ev_new = ev;
        if constexpr (I8) {
          float big = 0.f;  // of the scales that the row sees
#pragma unroll
          for (int c = 0; c < 4 * BLOCKS; ++c) big = fmaxf(big, (hidden >> c & 1u) ? 0.f : vs[c]);
          big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
          big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
          ev_new = max(ev, min(kMaxExp, ((__float_as_int(big) >> 23) & 255) - 127));
        }
        if (__any_sync(0xffffffffu, m_new > m || ev_new > ev)) {
          const float f = m == -INFINITY ? 0.f : exp2_approx(m - m_new);
          l *= f;
          const float fo = I8 ? f * exp2_int(ev - ev_new) : f;
          const float f0 = __shfl_sync(0xffffffffu, fo, 8 * t), f1 = __shfl_sync(0xffffffffu, fo, 8 * t + 4);
#pragma unroll
          for (int i = 0; i < F::MB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] *= j & 1 ? f1 : f0;
          m = m_new;
          ev = ev_new;
        }
        const float base = kShift - (m == -INFINITY ? 0.f : m);
        const float down = I8 ? exp2_int(-ev) : 1.f;
        float p[4 * BLOCKS];
#pragma unroll
        for (int c = 0; c < 4 * BLOCKS; ++c) {
          p[c] = exp2_approx(s[c] + base);
          l += p[c];
          if constexpr (I8) p[c] = (hidden >> c & 1u) ? 0.f : p[c] * (vs[c] * down);
        }
        // ---- sums ----
#pragma unroll
        for (int blk = 0; blk < BLOCKS; ++blk) {
          uint32_t hi[2], lo[2];
          split_f16(p[4 * blk], p[4 * blk + 1], hi[0], lo[0]);
          split_f16(p[4 * blk + 2], p[4 * blk + 3], hi[1], lo[1]);
          auto add = [&](int i, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
            const uint4 v = make_uint4(a0, a1, a2, a3);
            float c[4] = {0.f, 0.f, 0.f, 0.f};
            mma16816(c, v, lo[0], lo[1]);
            mma16816(c, v, hi[0], hi[1]);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] += c[j];
          };
#pragma unroll
          for (int i = 0; i < F::VC; ++i) {
            uint32_t vr[4][F::VW];
            values(blk, i, vr);
            if (!I8 && edge) {
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if (zap >> (4 * blk + c) & 1u) {
#pragma unroll
                  for (int w = 0; w < F::VW; ++w) vr[c][w] = 0u;
                }
            }
#pragma unroll
            for (int w = 0; w < F::VW; ++w) {
              if constexpr (I8) {
                const uint32_t k0 = vr[0][w] ^ 0x80808080u, k1 = vr[1][w] ^ 0x80808080u;
                const uint32_t k2 = vr[2][w] ^ 0x80808080u, k3 = vr[3][w] ^ 0x80808080u;
                const uint32_t lo0 = __byte_perm(k0, k1, 0x5140u), hi0 = __byte_perm(k0, k1, 0x7362u);
                const uint32_t lo1 = __byte_perm(k2, k3, 0x5140u), hi1 = __byte_perm(k2, k3, 0x7362u);
                const int at = 2 * (i * F::VW + w);
                add(at, i8_pair(lo0, 0x4140u), i8_pair(lo0, 0x4342u), i8_pair(lo1, 0x4140u), i8_pair(lo1, 0x4342u));
                add(at + 1, i8_pair(hi0, 0x4140u), i8_pair(hi0, 0x4342u), i8_pair(hi1, 0x4140u), i8_pair(hi1, 0x4342u));
              } else {
                add(i * F::VW + w, __byte_perm(vr[0][w], vr[1][w], 0x5410u), __byte_perm(vr[0][w], vr[1][w], 0x7632u),
                    __byte_perm(vr[2][w], vr[3][w], 0x5410u), __byte_perm(vr[2][w], vr[3][w], 0x7632u));
              }
            }
          }
        }
      }
      __syncwarp();  // every lane has read the stage
      if (lane == 0) mbar_arrive(bars + 8u * (F::STAGES + stage));
    }

    // ---- the warps' sums together, PARTS warps at a time, always in the same order ----
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    sync();  // the shared arrays' last readers are done
    if (t == 0) {
      s_m[warp][g] = m;
      s_l[warp][g] = l * kUnshift;  // from here on in units of 1: values next to fp32's largest are not multiplied
    }
    sync();
    float m_all = s_m[0][g];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m_all = fmaxf(m_all, s_m[w][g]);
    const float f = (m == -INFINITY ? (l != l ? l : 0.f) : exp2_approx(m - m_all)) * (I8 ? exp2_int(ev) : 1.f) * kUnshift;
    const float f0 = __shfl_sync(0xffffffffu, f, 8 * t), f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
#pragma unroll 1
    for (int turn = kWarps / F::PARTS - 1; turn >= 0; --turn) {
      if (warp / F::PARTS == turn) {
#pragma unroll
        for (int i = 0; i < F::MB; i += 2)  // two m-blocks: four neighbouring dims
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float fj = j ? f1 : f0;
            float4* dst = reinterpret_cast<float4*>(&s_o[warp % F::PARTS][2 * t + j][F::v_dim(2 * i, g)]);
            float4 v = make_float4(o[i][j] * fj, o[i][2 + j] * fj, o[i + 1][j] * fj, o[i + 1][2 + j] * fj);
            if (turn < kWarps / F::PARTS - 1) {
              const float4 w = *dst;
              v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
            }
            *dst = v;
          }
      }
      sync();
    }
    const bool whole = run.whole();
    float* slots = a.slots + (int64_t)blockIdx.x * 2 * SLOT;
    float* mine = slots + (run.first == 0 ? SLOT : 0);
    auto store = [&](int row, int d, float4 v, float total) {
      const int i = (x.r0 + row) / a.group, head = x.h * a.group + (x.r0 + row) % a.group;
      const float inv = total == 0.f ? 0.f : 1.0f / total;
      *reinterpret_cast<float4*>(a.out + (x.s.row0 + i) * a.ldo + (int64_t)head * D + d) =
          make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    };
    constexpr int Q4 = D / 4;
    for (int i = threadIdx.x; i < x.rows * Q4; i += 32 * kWarps) {
      const int row = i / Q4, d = 4 * (i % Q4);
      float top = s_m[0][row];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, s_m[w][row]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float total = 0.f;
#pragma unroll
      for (int w = 0; w < F::PARTS; ++w) {
        const float4 part = *reinterpret_cast<const float4*>(&s_o[w][row][d]);
        v = make_float4(v.x + part.x, v.y + part.y, v.z + part.z, v.w + part.w);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float lw = s_l[w][row];
        total += s_m[w][row] == -INFINITY ? lw : lw * exp2_approx(s_m[w][row] - top);
      }
      if (whole) {
        store(row, d, v, total);
      } else {
        *reinterpret_cast<float4*>(mine + row * D + d) = v;
        if (d == 0) {
          mine[kRT * D + row] = top;
          mine[kRT * D + kRT + row] = total;
        }
      }
    }
    if (whole) continue;
    // ---- a divided tile: the last block joins the pieces ----
    const int c0 = run.first_block(), c1 = run.last_block();
    sync();
    if (threadIdx.x == 0) {
      __threadfence();
      *s_last = atomicAdd(a.counters + c0, 1u) == (unsigned)(c1 - c0);
      __threadfence();
    }
    sync();
    if (!*s_last) continue;
    auto piece = [&](int c) { return a.slots + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * SLOT; };
    // rows' maxima over the pieces
    for (int row = warp; row < x.rows; row += kWarps) {
      float top = -INFINITY;
      for (int c = c0 + lane; c <= c1; c += 32) top = fmaxf(top, __ldcg(piece(c) + kRT * D + row));
#pragma unroll
      for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
      if (lane == 0) s_m[0][row] = top;
    }
    sync();
    // each warp every kWarps-th piece, then the warps together as above
    constexpr int ROWS = 32 / Q4 > 0 ? 32 / Q4 : 1;  // rows a warp covers at once (D = 64: 2)
    float4 acc[kRT / ROWS];
    float tot[kRT / ROWS];
    const int sub = lane / Q4, d4 = 4 * (lane % Q4);
#pragma unroll
    for (int i = 0; i < kRT / ROWS; ++i) {
      acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      tot[i] = 0.f;
    }
#pragma unroll 2
    for (int c = c0 + warp; c <= c1; c += kWarps) {
      const float* p = piece(c);
#pragma unroll
      for (int i = 0; i < kRT / ROWS; ++i) {
        const int row = i * ROWS + sub;
        if (row < x.rows) {
          const float mp = __ldcg(p + kRT * D + row), lp = __ldcg(p + kRT * D + kRT + row);
          const float4 v = __ldcg(reinterpret_cast<const float4*>(p + row * D + d4));
          const float w = mp == -INFINITY ? 1.f : exp2_approx(mp - s_m[0][row]);  // without keys: zeros, or NaN
          acc[i] = make_float4(acc[i].x + v.x * w, acc[i].y + v.y * w, acc[i].z + v.z * w, acc[i].w + v.w * w);
          tot[i] += lp * w;
        }
      }
    }
    sync();
#pragma unroll 1
    for (int turn = kWarps / F::PARTS - 1; turn >= 0; --turn) {
      if (warp / F::PARTS == turn) {
#pragma unroll
        for (int i = 0; i < kRT / ROWS; ++i) {
          float4* dst = reinterpret_cast<float4*>(&s_o[warp % F::PARTS][i * ROWS + sub][d4]);
          const float4 v = turn == kWarps / F::PARTS - 1 ? make_float4(0.f, 0.f, 0.f, 0.f) : *dst;
          *dst = make_float4(acc[i].x + v.x, acc[i].y + v.y, acc[i].z + v.z, acc[i].w + v.w);
          if (d4 == 0) s_l[warp][i * ROWS + sub] = tot[i];
        }
      }
      sync();
    }
    for (int i = threadIdx.x; i < x.rows * Q4; i += 32 * kWarps) {
      const int row = i / Q4, d = 4 * (i % Q4);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float total = 0.f;
#pragma unroll
      for (int w = 0; w < F::PARTS; ++w) {
        const float4 part = *reinterpret_cast<const float4*>(&s_o[w][row][d]);
        v = make_float4(v.x + part.x, v.y + part.y, v.z + part.z, v.w + part.w);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) total += s_l[w][row];
      store(row, d, v, total);
    }
    if (threadIdx.x == 0) a.counters[c0] = 0u;
  }
}

template <int D, bool I8, bool TREE>
spl_status launch_rows(const AttnArgs& a, int blocks, cudaStream_t stream) {
  constexpr uint32_t smem = Frag<D, I8>::SMEM;
  static bool done[kMaxDevices] = {false};
  if (!allow_shared(reinterpret_cast<const void*>(attention_rows_kernel<D, I8, TREE>), smem, done)) return SPL_ECUDA;
  attention_rows_kernel<D, I8, TREE><<<blocks, kThreads, smem, stream>>>(a);
  return launch_status();
}

}  // namespace

template <bool TREE>
spl_status pick_rows(const AttnArgs& a, int head_dim, bool i8, int blocks, cudaStream_t stream) {
  if (head_dim == 128)
    return i8 ? launch_rows<128, true, TREE>(a, blocks, stream) : launch_rows<128, false, TREE>(a, blocks, stream);
  return i8 ? launch_rows<64, true, TREE>(a, blocks, stream) : launch_rows<64, false, TREE>(a, blocks, stream);
}
spl_status run_attention_rows(const AttnArgs& a, int head_dim, bool i8, bool tree, int blocks, cudaStream_t stream) {
  return tree ? pick_rows<true>(a, head_dim, i8, blocks, stream) : pick_rows<false>(a, head_dim, i8, blocks, stream);
}

namespace {

struct Shape {
  bool few;
  int blocks;
  size_t bytes;  // of the workspace
};

spl_status check(const spl_kv_cache* cache, const spl_kv_batch* batch, int64_t rows, int64_t q_heads, PagedCache* c,
                 PagedBatch* b) {
  spl_status st = paged_cache_view(c, cache);
  if (st != SPL_OK) return st;
  if (q_heads < 1 || q_heads % cache->kv_heads != 0 || rows < 0) return SPL_EINVAL;
  if (q_heads / cache->kv_heads > 1024 || rows > INT32_MAX / 2 / (q_heads / cache->kv_heads))
    return SPL_ESHAPE;
  return paged_batch_view(b, *c, batch, rows);
}

// The few-row kernel where every sequence's rows of a key head fit one of its tiles, or a few of them: three over int8,
// which the tensor-core kernel first widens to binary16, two of 64 dims, whose softmax bounds that kernel; or where the
// units (64 keys of a tile) that the batch can have, by its longest chunk and its page table, are few: the tensor-core
// kernel costs some 8 us more at the start and a tenth as much per unit.  Measured, few rows and tensor cores, us, 32 query
// heads on 8, 16 sequences over 800 to 8000 keys: of 4 rows (two tiles) int8 64, 88, binary16 81, 68, 64 dims 45, 55; of
// 5 rows (three) int8 86, 88, binary16 125, 69, 64 dims int8 58, 82, binary16 63, 55; 64 sequences of 5 rows over 1000,
// int8 102, 115.  24 query heads on 8, binary16: 16 rows over 2048 keys 19, 21, over 8192 34, 29; 64 rows over 512 22, 21,
// over 2048 35, 26; 16 sequences of 8 rows over 128 16, 17, over 512 27, 21; 128 rows over 128 16, 17.  The limits go by
// what the host knows, max_rows and the page table's width: one long chunk takes all sequences of its batch along.
constexpr int64_t kFewUnits = 1600;
Shape shape_of(const spl_kv_cache* cache, const spl_kv_batch* batch, int64_t q_heads) {
  const int d = (int)cache->head_dim, sms = device_sm_count();
  Shape s;
  const int64_t rows = std::min<int64_t>(std::max<int64_t>(batch->max_rows, 1), INT32_MAX);  // (it may be any number)
  const int64_t tiles = ceil_div(rows * (q_heads / cache->kv_heads), kRT);
  const int64_t units = cache->pages == 0 ? 0 : ceil_div(batch->max_pages * cache->page_size, 64);
  const int most = cache->format == SPL_KV_I8 ? 3 : d == 64 ? 2 : 1;
  s.few = tiles <= most || (double)tiles * (double)units * (double)(batch->seqs * cache->kv_heads) <= kFewUnits;
  if (s.few) {
    s.blocks = sms;
    s.bytes = kCounterBytes + (size_t)s.blocks * 2 * kRT * (d + kSlotStats) * sizeof(float);
  } else {
    s.blocks = sms;
    s.bytes = kCounterBytes + attention_tc_bytes(d, sms);
  }
  return s;
}

}  // namespace
}  // namespace spl

using namespace spl;

extern "C" size_t spl_paged_attention_workspace_bytes(const spl_kv_cache* cache, const spl_kv_batch* batch,
                                                      int64_t rows, int64_t q_heads) {
  PagedCache c;
  PagedBatch b;
  if (check(cache, batch, rows, q_heads, &c, &b) != SPL_OK || rows == 0 || b.seqs == 0) return 0;
  return shape_of(cache, batch, q_heads).bytes;
}

static spl_status attend(float* out, int64_t ldo, const float* Q, int64_t ldq, const spl_kv_cache* cache,
                         const spl_kv_batch* batch, bool tree, const uint32_t* seen, int64_t words, int64_t rows,
                         int64_t q_heads, float scale, int64_t window, void* workspace, size_t workspace_bytes,
                         cudaStream_t stream) {
  AttnArgs a = {};
  spl_status st = check(cache, batch, rows, q_heads, &a.cache, &a.batch);
  if (st != SPL_OK) return st;
  const int64_t width = q_heads * cache->head_dim;
  if (ldo < 0 || ldq < 0 || window < 0 || words < 0 || !std::isfinite(scale)) return SPL_EINVAL;
  if (rows == 0 || a.batch.seqs == 0) return SPL_OK;
  if (!out || !Q || (words > 0 && !seen)) return SPL_EINVAL;
  if (rows > 1 && (ldo < width || ldq < width)) return SPL_EINVAL;
  if (!aligned16(out) || !aligned16(Q) || !aligned4(seen) || (rows > 1 && (ldo % 4 != 0 || ldq % 4 != 0))) return SPL_EALIGN;
  const Shape s = shape_of(cache, batch, q_heads);
  if (!workspace || workspace_bytes < s.bytes) return SPL_EWORKSPACE;
  if (!aligned16(workspace)) return SPL_EALIGN;
  if (!(a.batch.status = device_status_word())) return SPL_ECUDA;
  a.out = out;
  a.q = Q;
  a.ldo = ldo;
  a.ldq = ldq;
  a.group = (int)(q_heads / cache->kv_heads);
  a.window = window == 0 || window > INT32_MAX ? INT32_MAX : (int)window;
  a.scale_log2 = (float)(scale * 1.4426950408889634);
  a.counters = static_cast<unsigned int*>(workspace);
  a.slots = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
  a.least = s.few ? 1 : 3;
  a.slack = s.few ? 1 : 3;
  a.join = s.few ? 2 : 3;
  a.start = s.few ? 2 : 3;
  a.seen = seen;
  a.words = words;
  const int d = (int)cache->head_dim;
  const bool i8 = cache->format == SPL_KV_I8;
  return s.few ? run_attention_rows(a, d, i8, tree, s.blocks, stream)
               : run_attention_tc(a, d, i8, tree, s.blocks, stream);
}

extern "C" spl_status spl_paged_attention(float* out, int64_t ldo, const float* Q, int64_t ldq,
                                          const spl_kv_cache* cache, const spl_kv_batch* batch, int64_t rows,
                                          int64_t q_heads, float scale, int64_t window, void* workspace,
                                          size_t workspace_bytes, cudaStream_t stream) {
  return attend(out, ldo, Q, ldq, cache, batch, false, nullptr, 0, rows, q_heads, scale, window, workspace,
                workspace_bytes, stream);
}

extern "C" spl_status spl_tree_attention(float* out, int64_t ldo, const float* Q, int64_t ldq, const spl_kv_cache* cache,
                                         const spl_kv_batch* batch, const uint32_t* seen, int64_t words, int64_t rows,
                                         int64_t q_heads, float scale, int64_t window, void* workspace,
                                         size_t workspace_bytes, cudaStream_t stream) {
  return attend(out, ldo, Q, ldq, cache, batch, true, seen, words, rows, q_heads, scale, window, workspace,
                workspace_bytes, stream);
}
