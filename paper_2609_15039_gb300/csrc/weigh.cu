// The attention weight that stored tokens gather: score_j <- decay score_j + sum_i softmax_j(scale q_i . k_j).
//
// Few rows a sequence and key head (decode, drafts), bound by reading the keys once.  One kernel makes the scores
// s = scale log2(e) q . k of tiles of 8 rows on mma.m16n8k16 (the 8 rows' high and low halves are the 16 rows of A; the
// stored values are exact in binary16, so the result has fp32 accuracy) and writes them to the workspace, with the largest
// and the total of 2^(s - largest) of every 32 keys and row.  Another joins those by rows and sums 2^(s - m) / l over the
// rows for each key: a score is 4 bytes beside the 2 D of its key.
// Measured with 24 query heads on 8 of 128 dims: 64 sequences of one row over 1600 to 16000 keys, binary16, 176 us for the scores
// (1.15 GB of keys, 6.6 TB/s) and 31 us for the sums, which read 75 MB of scores and totals from memory under ncu, mostly L2
// otherwise; one sequence of 300 keys 9.4 and 7.6 us, two launches' latency.

#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "ptx.cuh"
#include "weigh.cuh"

namespace spl {
namespace {

constexpr int kWarps = 8, kThreads = 32 * (kWarps + 4);  // and a warpgroup that copies
constexpr int kRT = 8;       // rows of a tile
constexpr int kPart = 32;    // keys that a warp takes at once, for which it leaves a maximum and a total
constexpr int kUnit = kPart * kWarps;

struct WeighArgs {
  AttnArgs attn;
  float* score;        // [pages, heads, page]
  float decay;
  int q_heads;
  int64_t cap;         // keys that a row has places for, a multiple of kUnit
  float* s;            // [rows][q_heads][cap]
  float2* parts;       // [rows][q_heads][cap / kPart]: largest, total
};

__device__ __forceinline__ void mma16816(float (&c)[4], const uint4& a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}

// How a lane (g = lane / 4, t = lane % 4) holds keys and rows: the order of the dimensions in a product is free, so it reads
// 16 neighbouring bytes of a key; and the ring of units in shared memory.
template <int D, bool I8>
struct Keys {
  static constexpr int ESZ = I8 ? 1 : 2, E = 16 / ESZ, KB = D / (4 * E), STEPS = D / 16;
  static __device__ __forceinline__ int dim(int s, int t) {  // first of the two neighbours (and + {2, 3}) of step s
    constexpr int per = E / 4;
    return (s / per) * 4 * E + t * E + 4 * (s % per);
  }
  static constexpr uint32_t SCALE = kUnit * D * ESZ, STAGE = SCALE + (I8 ? kUnit * 4 : 0);
  static constexpr int STAGES = STAGE > 40000 ? 3 : (STAGE > 20000 ? 5 : 8);
  static constexpr int COPIERS = I8 ? 2 : 1;
  static constexpr uint32_t BARS = STAGES * STAGE, MASK = BARS + 16 * STAGES, ABORT = MASK + 4 * STAGES, SMEM = ABORT + 4;
  static_assert(SMEM <= 232448 && kMaxSeqs * kPrefixBytes + 8192 <= BARS, "fits");
};
template <int D, bool I8>
using Run = AttnRun<kRT, kUnit, kThreads>;

// A copying warp: unit after unit of the block's run into the ring's stages in turn, the keys or (int8) their scales.
template <int D, bool I8>
__device__ void copy_keys(Run<D, I8>& run, uint8_t* smem, int part) {
  using F = Keys<D, I8>;
  constexpr int BLOCKS = kUnit / 16;
  const PagedCache& cache = run.a.cache;
  const int lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem), bars = base + F::BARS;
  const uint64_t policy = l2_evict_first();
  const int per_page = min(BLOCKS, 1 << (cache.page_shift - 4));  // blocks of a unit that lie side by side
  volatile int* abort = reinterpret_cast<volatile int*>(smem + F::ABORT);
  int it = 0;
  bool ok = true;
  for (; ok && run.busy(); run.next()) {
    const AttnTile& x = run.x;
    const int last = run.last();
    int64_t slot = -1;  // of the first key of the lane's block of 16, -1 where no row sees any
    auto look_up = [&](int u) {
      const int j = (x.unit0 + u) * kUnit + 16 * lane;
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
      const uint32_t page_mask = (uint32_t)(((1ull << per_page) - 1u) << (lane / per_page * per_page)) & mask;
      const bool leads = slot >= 0 && (page_mask & ((1u << lane) - 1u)) == 0;
      const uint32_t keys = 16u * __popc(page_mask);
      if (part == 0 && lane == 0) {
        *reinterpret_cast<volatile uint32_t*>(smem + F::MASK + 4 * stage) = mask;
        mbar_expect_tx(full, 16u * __popc(mask) * ((uint32_t)D * F::ESZ + (I8 ? 4u : 0u)));
      } else if (lane == 0) {
        mbar_arrive(full);
      }
      __syncwarp();
      if (leads && part == 0)
        bulk_load(at + 16u * lane * D * F::ESZ, static_cast<const char*>(cache.k) + slot * (D * F::ESZ),
                  keys * D * F::ESZ, full, policy);
      else if (leads)
        bulk_load(at + F::SCALE + 64u * lane, cache.k_scale + slot, keys * 4u, full, policy);
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

template <int D, bool I8>
__global__ void __launch_bounds__(kThreads, 1) weigh_scores_kernel(const __grid_constant__ WeighArgs w) {
  using F = Keys<D, I8>;
  const AttnArgs& a = w.attn;
  extern __shared__ __align__(128) uint8_t smem[];
  volatile int* abort = reinterpret_cast<volatile int*>(smem + F::ABORT);
  if (threadIdx.x == 0) *abort = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t bars = smem_u32(smem + F::BARS);
  if (threadIdx.x < 2 * F::STAGES) mbar_init(bars + 8u * threadIdx.x, threadIdx.x < F::STAGES ? F::COPIERS : kWarps);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  Run<D, I8> run(a, reinterpret_cast<int64_t*>(smem));
  fence_proxy_async_smem();
  __syncthreads();  // the prefix sums have been read: their place is the ring's
  pdl_trigger();
  if (warp >= kWarps) {
    if (warp < kWarps + F::COPIERS) copy_keys<D, I8>(run, smem, warp - kWarps);
    return;
  }
  int it = 0;
  for (; run.busy(); run.next()) {
    const AttnTile& x = run.x;
    // ---- the tile's rows: q = (hi + lo) 2^-e; the high halves are rows 0-7 of A, the low ones rows 8-15 ----
    const int r = min(x.r0 + g, x.r0 + x.rows - 1);  // rows past the last repeat it
    const int token = r / a.group, head = x.h * a.group + r % a.group;
    uint4 qa[F::STEPS];
    float row_scale;
    {
      const float* q = a.q + (x.s.row0 + token) * a.ldq + (int64_t)head * D;
      float4 v[F::STEPS];
      float top = 0.f;
#pragma unroll
      for (int s = 0; s < F::STEPS; ++s) {
        v[s] = __ldg(reinterpret_cast<const float4*>(q + F::dim(s, t)));
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
    row_keys(x.s, a.window, token, row_lo, row_hi);
    const int64_t row = (x.s.row0 + token) * (int64_t)w.q_heads + head;
    float* s_row = w.s + row * w.cap;
    float2* part_row = w.parts + row * (w.cap / kPart);
    const bool mine = g < x.rows;

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
      const uint32_t mask = there ? *reinterpret_cast<volatile const uint32_t*>(smem + F::MASK + 4 * stage) >> (2 * warp) : 0u;
      const int k0 = kPart * warp, j0 = (x.unit0 + u) * kUnit + k0;
      // ---- scores of keys 8 c + 2t, + 1 and row g ----
      float s[8];
      float acc[4][4] = {};
#pragma unroll
      for (int i = 0; i < F::KB; ++i) {
        uint4 k16[4];
#pragma unroll
        for (int c = 0; c < 4; ++c)
          k16[c] = *reinterpret_cast<const uint4*>(at + (k0 + 8 * c + g) * (D * F::ESZ) + 64 * i + 16 * t);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t v[4] = {k16[c].x, k16[c].y, k16[c].z, k16[c].w};
          if constexpr (I8) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t biased = v[k] ^ 0x80808080u;
              mma16816(acc[c], qa[4 * i + k], i8_pair(biased, 0x4140u), i8_pair(biased, 0x4342u));
            }
          } else {
            mma16816(acc[c], qa[2 * i], v[0], v[1]);
            mma16816(acc[c], qa[2 * i + 1], v[2], v[3]);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        // An infinity of a key, which both halves of q may make one of the same sign, is a NaN of the score: x - x is NaN there,
        // and 0 else.  (Finite ones are at most 2^39.)
        const float a0 = acc[c][0] + acc[c][2], a1 = acc[c][1] + acc[c][3];
        if constexpr (I8) {
          const float2 sc = *reinterpret_cast<const float2*>(at + F::SCALE + 4 * (k0 + 8 * c + 2 * t));
          s[2 * c] = fmaf(a0 * row_scale, sc.x, sc.x - sc.x);
          s[2 * c + 1] = fmaf(a1 * row_scale, sc.y, sc.y - sc.y);
        } else {
          s[2 * c] = fmaf(a0, row_scale, a0 - a0);
          s[2 * c + 1] = fmaf(a1, row_scale, a1 - a1);
        }
      }
      __syncwarp();  // every lane has read the stage
      if (lane == 0) mbar_arrive(bars + 8u * (F::STAGES + stage));
      if (j0 < x.all_lo || j0 + kPart > x.all_hi || (~mask & 3u) != 0) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const int j = j0 + 8 * (c >> 1) + 2 * t + (c & 1);
          if (!(mask >> (c >> 2) & 1u) || j < row_lo || j >= row_hi) s[c] = -INFINITY;
        }
      }
      // ---- their largest and total, a NaN among them ----
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) top = fmaxf(top, s[c]);
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int c = 0; c < 8; ++c) sum += exp2_approx(s[c] - base);
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      // (A tile whose rows see nothing has a unit all the same, which may lie behind the row's places; nobody reads what no row
      // sees.)
      if (!mine || j0 >= x.key_hi) continue;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float2*>(s_row + j0 + 8 * c + 2 * t) = make_float2(s[2 * c], s[2 * c + 1]);
      if (t == 0) part_row[j0 / kPart] = make_float2(top, sum);
    }
  }
}

// A block has `trips` times 1024 keys of a (sequence, key head): first the rows' maxima and totals, from what the scores'
// kernel left of every 32 keys, then the rows' weights in their order, a thread four neighbouring keys.  blockIdx: keys, key head, sequence.
constexpr int kSumThreads = 256, kTrip = 4 * kSumThreads, kSumRows = 64;
constexpr int kMostTrips = 4;
__global__ void __launch_bounds__(kSumThreads, 6) weigh_sum_kernel(const __grid_constant__ WeighArgs w, int trips) {
  struct Row {
    float m, inverse;  // maximum, 1 / total
    int lo, hi;        // keys that it sees
  };
  __shared__ __align__(16) Row rows_of[kSumRows];
  __shared__ const float* scores_of[kSumRows];
  __shared__ float2 teams[kSumThreads / 32];
  const AttnArgs& a = w.attn;
  const int h = blockIdx.y, b = blockIdx.z, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // (what the scores' kernel does not write may be read before it ends)
  const PagedSeq s = paged_seq(a.batch, a.cache.page_shift, b);
  const int rows = s.n * a.group;
  const bool wide = (reinterpret_cast<uintptr_t>(w.score) & 15u) == 0;
  // row r of the key head: query head r % group of token r / group
  auto row_of = [&](int r) { return (s.row0 + r / a.group) * (int64_t)w.q_heads + h * a.group + r % a.group; };
  for (int64_t from = (int64_t)blockIdx.x * trips * kTrip; from < s.len; from += (int64_t)gridDim.x * trips * kTrip) {
    const int64_t end = min((int64_t)s.len, from + trips * kTrip);
    int pages[kMostTrips];  // (all at once: a trip's would wait for memory before its scores could)
#pragma unroll
    for (int u = 0; u < kMostTrips; ++u) {
      const int64_t j = from + u * kTrip + 4 * threadIdx.x;
      pages[u] = j < end ? __ldg(a.batch.table + b * a.batch.max_pages + (j >> a.cache.page_shift)) : 0;
    }
    // Maxima and totals of up to kSumRows rows from r0 on.
    auto totals = [&](int r0, int some) {
      const int team = some > 4 ? 1 : (some > 2 ? 2 : (some > 1 ? 4 : 8));
      __syncthreads();
      for (int q0 = 0; q0 < some * team; q0 += kSumThreads / 32) {  // `team` warps a row
        const int r = min((q0 + warp) / team, some - 1), mate = warp % team;
        int lo, hi;
        row_keys(s, a.window, (r0 + r) / a.group, lo, hi);
        const float2* parts = w.parts + row_of(r0 + r) * (w.cap / kPart);
        float m = -INFINITY, l = 0.f;
        for (int p0 = lo / kPart + 32 * mate; p0 * kPart < hi; p0 += 4 * 32 * team) {
          float2 v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int p = p0 + 32 * team * k + lane;
            v[k] = p * kPart < hi ? parts[p] : make_float2(-INFINITY, 0.f);
          }
          const float top = fmaxf(fmaxf(fmaxf(v[0].x, v[1].x), fmaxf(v[2].x, v[3].x)), m), base = top == -INFINITY ? 0.f : top;
          l *= exp2_approx(m - base);
#pragma unroll
          for (int k = 0; k < 4; ++k) l += v[k].y * exp2_approx(v[k].x - base);
          m = top;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const float om = __shfl_xor_sync(0xffffffffu, m, o), ol = __shfl_xor_sync(0xffffffffu, l, o);
          const float top = fmaxf(m, om), base = top == -INFINITY ? 0.f : top;
          l = l * exp2_approx(m - base) + ol * exp2_approx(om - base);
          m = top;
        }
        if (lane == 0) teams[warp] = make_float2(m, l);
        __syncthreads();
        if (lane == 0 && mate == 0 && q0 + warp < some * team) {
          for (int k = 1; k < team; ++k) {
            const float2 o = teams[warp + k];
            const float top = fmaxf(m, o.x), base = top == -INFINITY ? 0.f : top;
            l = l * exp2_approx(m - base) + o.y * exp2_approx(o.x - base);
            m = top;
          }
          rows_of[r] = {m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.0f / l, lo, hi};
          scores_of[r] = w.s + row_of(r0 + r) * w.cap;
        }
        __syncthreads();
      }
    };
    pdl_wait();
    if (rows <= kSumRows) totals(0, rows);
#pragma unroll
    for (int u = 0; u < kMostTrips; ++u) {
      if (from + u * kTrip >= end) break;
      const int key = (int)(from + u * kTrip) + 4 * threadIdx.x;
      float* score = nullptr;
      float4 before = make_float4(0.f, 0.f, 0.f, 0.f), sum = before;
      if (key < end) {
        if ((unsigned)pages[u] < (unsigned)a.cache.pages)
          score = w.score + paged_slot(a.cache, pages[u], h, key);  // (four keys lie in one page)
        else
          atomicOr(a.batch.status, kStatusIndex);
      }
      if (score && wide && key + 3 < s.pos0) {
        before = *reinterpret_cast<const float4*>(score);
      } else if (score) {
        if (key < s.pos0) before.x = score[0];
        if (key + 1 < s.pos0) before.y = score[1];
        if (key + 2 < s.pos0) before.z = score[2];
        if (key + 3 < s.pos0) before.w = score[3];
      }
      for (int r0 = 0; r0 < rows; r0 += kSumRows) {
        const int some = min(kSumRows, rows - r0);
        if (rows > kSumRows) totals(r0, some);
        if (!score) continue;
#pragma unroll 4
        for (int r = 0; r < some; ++r) {
          const Row q = rows_of[r];
          if (key + 3 < q.lo || key >= q.hi) continue;
          const float4 v = *reinterpret_cast<const float4*>(scores_of[r] + key);
          const float p[4] = {exp2_approx(v.x - q.m), exp2_approx(v.y - q.m), exp2_approx(v.z - q.m), exp2_approx(v.w - q.m)};
          if (key < q.lo || key + 3 >= q.hi) {
            // Where the row does not see a key anything may be there, and its total may be NaN: what is added is chosen, not p.
            if (key >= q.lo) sum.x = fmaf(p[0], q.inverse, sum.x);
            if (key + 1 >= q.lo && key + 1 < q.hi) sum.y = fmaf(p[1], q.inverse, sum.y);
            if (key + 2 >= q.lo && key + 2 < q.hi) sum.z = fmaf(p[2], q.inverse, sum.z);
            if (key + 3 < q.hi) sum.w = fmaf(p[3], q.inverse, sum.w);
            continue;
          }
          sum.x = fmaf(p[0], q.inverse, sum.x);
          sum.y = fmaf(p[1], q.inverse, sum.y);
          sum.z = fmaf(p[2], q.inverse, sum.z);
          sum.w = fmaf(p[3], q.inverse, sum.w);
        }
      }
      if (!score) continue;
      const float4 after = make_float4(before.x * w.decay + sum.x, before.y * w.decay + sum.y, before.z * w.decay + sum.z,
                                       before.w * w.decay + sum.w);
      if (wide && key + 3 < s.len) {
        *reinterpret_cast<float4*>(score) = after;
      } else {
        score[0] = after.x;
        if (key + 1 < s.len) score[1] = after.y;
        if (key + 2 < s.len) score[2] = after.z;
        if (key + 3 < s.len) score[3] = after.w;
      }
    }
  }
  pdl_wait();  // (of a block without keys: this kernel may not end before the scores' one)
}

template <int D, bool I8>
spl_status launch_scores(const WeighArgs& w, int blocks, cudaStream_t stream) {
  constexpr uint32_t smem = Keys<D, I8>::SMEM;
  static bool done[kMaxDevices] = {false};
  if (!allow_shared(reinterpret_cast<const void*>(weigh_scores_kernel<D, I8>), smem, done)) return SPL_ECUDA;
  weigh_scores_kernel<D, I8><<<blocks, kThreads, smem, stream>>>(w);
  return launch_status();
}

// Few rows: of a key head at most so many, by max_rows, and scores that take no more than kMostScores bytes.  Measured, few and
// many rows, us.  15 sequences over 600 to 6000 keys, 32 query heads on 8: int8, 16 rows of a key head 52, 91, 24 rows 72, 92, 32
// rows 90, 90; binary16, 8 rows 41, 76, 16 rows 62, 76, 24 rows 91, 77.  64 sequences over 1600 to 16000, 24 on 8: int8, 12 rows
// 327, 611, 18 rows 477, 612; binary16, 6 rows 252, 470, 12 rows 486, 471, 18 rows 716, 472.  Two sequences over up to 6000: int8,
// 24 rows 40, 40; binary16, 8 rows 25, 30, 16 rows 32, 31.  One limit a format, by the rows alone: what the keys and the number of
// sequences would ask for differs from it by up to 23% (15 sequences of 16 rows binary16) on one side and 3% (64 of 12) on the other.
// And the scores' places go by the page table's width: many sequences of a row with a wide table leave for the kernels of many.
constexpr int64_t kMostScores = int64_t(1) << 31;
constexpr int64_t few_rows(bool i8) { return i8 ? 24 : 12; }
struct Shape {
  bool few;
  int64_t cap;
  size_t s, parts, bytes;
};
Shape shape_of(const PagedCache& c, const PagedBatch& b, const spl_kv_batch* batch, int64_t q_heads, int head_dim, bool i8) {
  Shape x = {};
  x.few = batch->max_rows <= few_rows(i8) / (q_heads / c.heads) &&  // (max_rows may be any number)
          (double)b.rows * (double)q_heads * (double)(b.max_pages << c.page_shift) * 4 <= (double)kMostScores;
  if (!x.few) {
    x.bytes = b.rows == 0 ? 0 : weigh_tc_bytes(c, b, q_heads, head_dim);
    return x;
  }
  x.cap = round_up(std::max<int64_t>(1, b.max_pages << c.page_shift), kUnit);
  x.s = (size_t)b.rows * q_heads * x.cap * sizeof(float);
  x.parts = x.s / kPart * 2;
  x.bytes = x.s + x.parts;
  return x;
}

spl_status check(const spl_kv_cache* cache, const spl_kv_batch* batch, int64_t rows, int64_t q_heads, PagedCache* c,
                 PagedBatch* b) {
  spl_status st = paged_cache_view(c, cache);
  if (st != SPL_OK) return st;
  if (q_heads < 1 || q_heads % cache->kv_heads != 0 || rows < 0) return SPL_EINVAL;
  if (q_heads / cache->kv_heads > 1024 || rows > INT32_MAX / 2 / (q_heads / cache->kv_heads))
    return SPL_ESHAPE;
  if ((st = paged_batch_view(b, *c, batch, rows)) != SPL_OK) return st;
  if (rows > (INT32_MAX - 1024) / q_heads) return SPL_ESHAPE;  // rows of a copy's coordinates
  return SPL_OK;
}

}  // namespace
}  // namespace spl

using namespace spl;

extern "C" size_t spl_kv_weigh_workspace_bytes(const spl_kv_cache* cache, const spl_kv_batch* batch, int64_t rows,
                                               int64_t q_heads) {
  PagedCache c;
  PagedBatch b;
  if (check(cache, batch, rows, q_heads, &c, &b) != SPL_OK || b.seqs == 0) return 0;
  const size_t bytes = shape_of(c, b, batch, q_heads, (int)cache->head_dim, cache->format == SPL_KV_I8).bytes;
  return bytes ? kCounterBytes + bytes : 0;
}

extern "C" spl_status spl_kv_weigh(float* score, const float* Q, int64_t ldq, const spl_kv_cache* cache,
                                   const spl_kv_batch* batch, int64_t rows, int64_t q_heads, float scale, int64_t window,
                                   float decay, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  WeighArgs w = {};
  AttnArgs& a = w.attn;
  spl_status st = check(cache, batch, rows, q_heads, &a.cache, &a.batch);
  if (st != SPL_OK) return st;
  if (ldq < 0 || window < 0 || !std::isfinite(scale) || !(decay >= 0.f && decay <= 1.f)) return SPL_EINVAL;
  if (a.batch.seqs == 0) return SPL_OK;
  if (rows > 0 && !Q) return SPL_EINVAL;
  if (rows > 1 && ldq < q_heads * cache->head_dim) return SPL_EINVAL;
  if (!aligned16(Q) || !aligned4(score) || (rows > 1 && ldq % 4 != 0)) return SPL_EALIGN;
  const int dim = (int)cache->head_dim;
  const bool i8 = cache->format == SPL_KV_I8;
  const Shape s = shape_of(a.cache, a.batch, batch, q_heads, dim, i8);
  if (s.bytes > 0 && (!workspace || workspace_bytes < kCounterBytes + s.bytes)) return SPL_EWORKSPACE;
  if (!aligned16(workspace)) return SPL_EALIGN;
  if (a.cache.pages == 0 || a.batch.max_pages == 0) return SPL_OK;
  if (!score) return SPL_EINVAL;
  if (!(a.batch.status = device_status_word())) return SPL_ECUDA;
  a.q = Q;
  a.ldq = ldq;
  a.group = (int)(q_heads / cache->kv_heads);
  a.window = window == 0 || window > INT32_MAX ? INT32_MAX : (int)window;
  a.scale_log2 = (float)(scale * 1.4426950408889634);
  a.least = 1;
  a.slack = 1;
  a.join = 0;
  a.start = 1;
  char* at = static_cast<char*>(workspace) + kCounterBytes;  // (the counters are others')
  if (rows > 0 && !s.few)
    return run_weigh_tc({score, Q, ldq, a.cache, a.batch, a.group, (int)q_heads, a.window, a.scale_log2, decay, at}, dim,
                        i8, stream);
  w.score = score;
  w.decay = decay;
  w.q_heads = (int)q_heads;
  w.cap = s.cap;
  w.s = reinterpret_cast<float*>(at);
  w.parts = reinterpret_cast<float2*>(at + s.s);
  const int sms = device_sm_count();
  if (rows > 0) {
    st = cache->head_dim == 128 ? (i8 ? launch_scores<128, true>(w, sms, stream) : launch_scores<128, false>(w, sms, stream))
                                : (i8 ? launch_scores<64, true>(w, sms, stream) : launch_scores<64, false>(w, sms, stream));
    if (st != SPL_OK) return st;
  }
  // Several trips a block where there are blocks enough, which then make the totals once (64 sequences over 1600 to 16000 keys:
  // 30 us instead of 38; one sequence's few blocks are better spread).
  const int64_t room = a.batch.max_pages << a.cache.page_shift;
  const int trips = ceil_div(room, kTrip) * a.cache.heads * a.batch.seqs >= (int64_t)8 * sms ? kMostTrips : 1;
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(room, trips * kTrip), 1 << 16), a.cache.heads, a.batch.seqs);
  if (rows > 0) return launch_pdl(weigh_sum_kernel, grid, dim3(kSumThreads), 0, stream, w, trips);
  weigh_sum_kernel<<<grid, kSumThreads, 0, stream>>>(w, trips);  // (what is before it may have written the scores)
  return launch_status();
}
