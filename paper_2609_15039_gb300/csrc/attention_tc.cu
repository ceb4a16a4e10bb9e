// Attention of many rows over a paged cache on the 5th-generation tensor cores (chunks of new tokens, prefill).
//
// o = sum_j softmax_j(scale q . k_j) v_j over tiles of 256 rows (two halves, A and B, of 128) and 128 keys.  Each half:
//   S = q_hi K^T + q_lo K^T        q = (hi + lo) 2^-e in binary16, a row's largest entry in [2^14, 2^15)
//   p = 2^(scale log2(e) S - m)    m the row's running maximum, l the running total, both fp32
//   O = O 2^(m_old - m) + p_hi V + p_lo V
// The stored keys and values are exact in binary16, so two products instead of one give fp32 accuracy, and the kernel
// is bound by the tensor pipe: 4 products of 128 x 128 x dim a half and tile.  Two halves, so that the products of one
// run while the softmax of the other does; they share the tiles of K and V in shared memory.
//   warps 0-3   producer: K and V tiles from the pages (cp.async; int8: through registers, widened), with zeros for
//               the keys that no row of the tile sees, in the 128-byte-swizzled layout that the MMAs read.
//   warps 4-7   softmax of half A, a thread a row; also q's split, the sums' rescaling and the output.
//   warps 8-11  the same of half B.
//   warp 12     MMA issuer.
// Tensor memory: S of A and of B (128 columns each) and O of A and of B (dim columns each).  p overwrites S in place:
// a chunk of 32 scores becomes 16 columns of p_hi and 16 of p_lo, the A operand of the second product.
// p is held as 2^13 p: the low half keeps an absolute 2^-38 of the row's largest.  The running maximum is raised only
// where it would let p pass 2, so that O is seldom rescaled.  O is folded into an fp32 sum in the workspace with round-to-nearest every kChain tiles, since the
// tensor core truncates as it accumulates (an unbroken chain's bias grows with its length).
// Divided tiles are joined by a second, small launch over all SMs.
// Every wait is bounded; on expiry the status word is raised and the block leaves with its copies and MMAs done.

#include <algorithm>
#include <cmath>

#include <cuda_fp16.h>

#include "attention.cuh"
#include "ptx.cuh"

namespace spl {
namespace {

constexpr int kThreads = 13 * 32;
constexpr int kRows = 256, kKeys = 128, kStages = 3;
constexpr int kChain = 8;        // key tiles of an accumulation chain of O (1024 keys)
constexpr float kShift = 13.0f;  // p is held as 2^kShift p
constexpr float kLazy = 1.0f;    // and may reach 2^(kShift + kLazy), times a scale below 2, before the maximum is raised
constexpr int kMinExp = -100, kMaxExp = 126;
constexpr int kProducerBar = 1;  // named barrier of the producer's warps

// Barriers by index: kFull, kEmpty a stage; kScale the scales of K of two steps; the others a half each, their phases
// counting its own key tiles (kQ: its pieces).
enum { kFull = 0, kEmpty = 3, kScale = 6, kQ = 8, kSFull = 10, kPFull = 12, kPv = 14, kDrain = 16, kBars = 17 };

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
  static constexpr uint32_t BARS = VMAX + 2 * 16, MISC = BARS + 8 * (kBars + 1);
  static constexpr uint32_t BYTES = MISC + 16;
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
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void named_sync(int bar, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(threads) : "memory");
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
  uint32_t smem;   // shared address of the aligned base
  uint32_t tmem;
  volatile int* abort;

  __device__ uint32_t bar(int i) const { return smem + L::BARS + 8u * i; }
  __device__ bool wait(int i, uint32_t parity) const {
    return __all_sync(0xffffffffu, mbar_wait(bar(i), parity, kWaitNs, abort));
  }
  __device__ void give_up() const {
    *abort = 1;
    atomicOr(a.batch.status, kStatusTimeout);
  }
  // Whether some row of the tile sees only a part of the 128 keys from j0 on.
  static __device__ bool edge_of(const AttnTile& x, int j0) { return j0 < x.all_lo || j0 + kKeys > x.all_hi; }

  // ---------------------------------------------------------------- producer
  __device__ void producer(Run& run) const {
    const int i = threadIdx.x, warp = i >> 5, lane = i & 31;
    const int heads = a.cache.heads, shift = a.cache.page_shift, in_page = (1 << shift) - 1;
    int tile = 0, step = 0;  // tiles issued, pairs of them
    bool ok = true;
    // F16: the tile that is issued and not yet handed over
    int open = -1, open_step = 0;
    bool open_scan = false;
    auto hand_over = [&]() {
      if constexpr (!I8) {
        if (open_scan) {  // values that only some rows see: an infinity or NaN becomes 0 and is marked
          const uint32_t marks = smem + L::BAD + 16u * (open_step & 1);
          if (i < 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(marks + 4u * i), "r"(0) : "memory");
          named_sync(kProducerBar, 128);
          const uint32_t base = smem + L::KV + (uint32_t)(open % kStages) * L::TILE;
          constexpr int PARTS = D / 8;
          for (int k = 0; k < kKeys * PARTS / 128; ++k) {
            const int c = i + 128 * k, key = c / PARTS, part = c % PARTS;
            const uint32_t at = base + (part >> 3) * L::PANEL + key * 128 + (((part & 7) ^ (key & 7)) << 4);
            const uint4 v = ld_shared16(at);
            if (f16_special2(v.x) || f16_special2(v.y) || f16_special2(v.z) || f16_special2(v.w)) {
              st_shared16(at, make_uint4(0u, 0u, 0u, 0u));
              asm volatile("red.shared.or.b32 [%0], %1;" ::"r"(marks + 4u * (key >> 5)), "r"(1u << (key & 31)) : "memory");
            }
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(kFull + open % kStages));
      open = -1;
    };
    for (; ok && run.busy(); run.next()) {
      const AttnTile& x = run.x;
      const int last = run.last();
      // page of the keys j0 + 16 lane .. of a tile, -1 where no row sees any of them (lanes 0-7)
      auto pages_of = [&](int u) {
        const int j = (x.unit0 + u) * kKeys + 16 * lane;
        if (lane >= kKeys / 16 || u >= last || j >= x.key_hi || j + 16 <= x.key_lo) return -1;
        return paged_page(a.cache, a.batch, x.b, j);
      };
      int page = pages_of(run.first);
      if constexpr (!I8) {
        for (int u = run.first; ok && u < last; ++u, ++step) {
          const int j0 = (x.unit0 + u) * kKeys;
          constexpr int PARTS = D / 8, PER = kKeys * PARTS / 128;  // 16-byte chunks of a key, of a thread
          constexpr int KEY_STEP = 128 / PARTS;
          for (int which = 0; which < 2; ++which, ++tile) {
            const int stage = tile % kStages;
            if (tile >= kStages) {
              const uint32_t parity = (uint32_t)(tile / kStages - 1) & 1u;
              if (open >= 0 && !__all_sync(0xffffffffu, mbar_try(bar(kEmpty + stage), parity))) {
                cp_async_wait<0>();
                hand_over();
              }
              ok = wait(kEmpty + stage, parity);
              if (!ok) break;
            }
            const char* src = static_cast<const char*>(which ? a.cache.v : a.cache.k);
            const uint32_t base = smem + L::KV + (uint32_t)stage * L::TILE;
            const int part = i % PARTS, key0 = i / PARTS;
            const uint32_t panel = base + (uint32_t)(part >> 3) * L::PANEL;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
              const int key = key0 + KEY_STEP * k, j = j0 + key;
              const int pg = __shfl_sync(0xffffffffu, page, key >> 4);
              const bool there = pg >= 0 && j >= x.key_lo && j < x.key_hi;
              const int64_t slot = there ? ((((int64_t)pg * heads + x.h) << shift) + (j & in_page)) : 0;
              cp_async16(panel + key * 128 + (((part & 7) ^ (key & 7)) << 4), src + slot * (2 * D) + part * 16, there);
            }
            cp_async_commit();
            if (open >= 0) {
              cp_async_wait<1>();
              hand_over();
            }
            open = tile;
            open_step = step;
            open_scan = which && edge_of(x, j0);
          }
          if (!ok) break;
          page = pages_of(u + 1);
        }
      } else {
        constexpr int PARTS = D / 16, PER = kKeys * PARTS / 128, KEY_STEP = 128 / PARTS;
        uint4 regs[2][PER];  // K and V of a step
        float scales[2];
        auto load = [&](int u, int which) {
          const int j0 = (x.unit0 + u) * kKeys;
          const char* src = static_cast<const char*>(which ? a.cache.v : a.cache.k);
          const int part = i % PARTS, key0 = i / PARTS;
#pragma unroll
          for (int k = 0; k < PER; ++k) {
            const int key = key0 + KEY_STEP * k, j = j0 + key;
            const int pg = __shfl_sync(0xffffffffu, page, key >> 4);
            const bool there = pg >= 0 && j >= x.key_lo && j < x.key_hi;
            const int64_t slot = there ? ((((int64_t)pg * heads + x.h) << shift) + (j & in_page)) : 0;
            regs[which][k] = there ? __ldg(reinterpret_cast<const uint4*>(src + slot * D + part * 16))
                                   : make_uint4(0u, 0u, 0u, 0u);
          }
          const int j = j0 + i, pg = __shfl_sync(0xffffffffu, page, (i >> 4) & 7);
          const bool there = pg >= 0 && j >= x.key_lo && j < x.key_hi;
          const int64_t slot = there ? ((((int64_t)pg * heads + x.h) << shift) + (j & in_page)) : 0;
          scales[which] = there ? __ldg((which ? a.cache.v_scale : a.cache.k_scale) + slot) : 0.f;
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
            const uint4 c = regs[which][k];
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
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(sc), "f"(scales[which]) : "memory");
          if (which) {
            float top = scales[1];
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
        load(run.first, 0);
        for (int u = run.first; ok && u < last; ++u, ++step) {
          load(u, 1);
          put(0);
          page = pages_of(u + 1);
          if (u + 1 < last) load(u + 1, 0);
          if (ok) put(1);
        }
      }
    }
    if constexpr (!I8) {
      cp_async_wait<0>();  // nothing in flight when the block leaves
      if (ok && open >= 0) hand_over();
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
  __device__ void issuer(Run& run) const {
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
    for (; ok && run.busy(); run.next()) {
      const int halves = run.x.rows > 128 ? 2 : 1, n = run.last() - run.first;
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
  // q's rows [32 q4, 32 q4 + 32) of the half as hi + lo into shared memory; the lane's own row's scale.
  __device__ float split_q(const AttnTile& x, int half, int q4) const {
    const int lane = threadIdx.x & 31;
    constexpr int LANES = D / 4, PER = 32 / LANES, BATCH = 8;  // lanes of a row, rows at a time
    const int sub = lane / LANES, at = lane % LANES;
    const float sign = a.scale_log2 < 0.f ? -1.f : 1.f;  // the scale's sign goes into q
    float mine = 0.f;
    const uint32_t hi = smem + L::Q + (uint32_t)half * 2 * L::TILE + (uint32_t)(at >> 4) * L::PANEL;
    for (int r0 = 0; r0 < 32; r0 += BATCH * PER) {
      float4 v[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int r = 128 * half + 32 * q4 + r0 + i * PER + sub;  // row of the tile
        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < x.rows) {
          const int fr = x.r0 + r, token = fr / a.group;
          v[i] = __ldg(reinterpret_cast<const float4*>(a.q + (x.s.row0 + token) * a.ldq +
                                                       (int64_t)(x.h * a.group + fr % a.group) * D) + at);
        }
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        float top = fmaxf(fmaxf(fabsf(v[i].x), fabsf(v[i].y)), fmaxf(fabsf(v[i].z), fabsf(v[i].w)));
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int e = fp16_row_exponent(top);
        const float up = sign * pow2f(e);
        const int row = r0 + i * PER + sub;  // of the 32
#pragma unroll
        for (int p = 0; p < PER; ++p) {
          const int ep = __shfl_sync(0xffffffffu, e, p * LANES);
          if (lane == r0 + i * PER + p) mine = fabsf(a.scale_log2) * pow2f(-ep);
        }
        uint32_t h0, l0, h1, l1;
        split_f16(v[i].x * up, v[i].y * up, h0, l0);
        split_f16(v[i].z * up, v[i].w * up, h1, l1);
        const int r = 32 * q4 + row;  // of the half
        const uint32_t addr = hi + (uint32_t)r * 128 + (((uint32_t)(at & 15) / 2 ^ (r & 7)) << 4) + 8u * (at & 1);
        asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(addr), "r"(h0), "r"(h1) : "memory");
        asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(addr + L::TILE), "r"(l0), "r"(l1) : "memory");
      }
    }
    return mine;
  }

  __device__ void softmax(Run& run, int half, Divided* divided) const {
    const int q4 = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
    const uint32_t lanes = (uint32_t)(32 * q4) << 16;
    const uint32_t ts = tmem + lanes + L::S + 128u * half, to = tmem + lanes + L::O + (uint32_t)D * half;
    const int own = 128 * half + 32 * q4 + lane;  // row of the tile
    bool ok = true;
    int step = 0;       // tiles of K so far
    uint32_t phase = 0;  // of this half's barriers: they complete once a key tile of a piece that has the half
    for (; ok && run.busy(); run.next()) {
      const AttnTile& x = run.x;
      const int first = run.first, n = run.last() - first;
      const bool there = x.rows > 128 * half;
      float* slot = a.slots + ((int64_t)blockIdx.x * 2 + (first == 0 ? 1 : 0)) * slot_floats<D>();
      auto slot4 = [&](int d4) { return reinterpret_cast<float4*>(slot) + d4 * kRows + own; };
      const bool whole = run.whole();
      float m = -INFINITY, l = 0.f;
      if (there) {
        const float row_scale = split_q(x, half, q4);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kQ + half));
        int row_lo = 0, row_hi = 0;
        const bool mine = own < x.rows;
        if (mine) row_keys(x.s, a.window, (x.r0 + own) / a.group, row_lo, row_hi);
        int ev = kMinExp, ev_slot = kMinExp;
        float m_slot = -INFINITY;
        bool has_slot = false;
        // The slot's sums (if any) in the units of m, ev, plus O: into the slot, the output or (times `f`) both's place.
        auto fold = [&](bool final) {
          const float keep = !has_slot || m_slot == -INFINITY
                                 ? (has_slot ? 1.f : 0.f)
                                 : exp2_approx(m_slot - m) * (I8 ? exp2_int(ev_slot - ev) : 1.f);
          const bool out = final && whole;
          const float unit = final && I8 ? exp2_int(ev) : 1.f;
          const float f = out ? (l == 0.f ? 0.f : 1.0f / l) * unit : unit;
          float* dst = nullptr;
          if (out && mine) {
            const int fr = x.r0 + own;
            dst = a.out + (x.s.row0 + fr / a.group) * a.ldo + (int64_t)(x.h * a.group + fr % a.group) * D;
          }
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            float v[32];
            tmem_ld_32x32(to + 32u * c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float4 w = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
              if (has_slot) {
                const float4 s = __ldcg(slot4(8 * c + i));
                w = make_float4(fmaf(s.x, keep, w.x), fmaf(s.y, keep, w.y), fmaf(s.z, keep, w.z), fmaf(s.w, keep, w.w));
              }
              w = make_float4(w.x * f, w.y * f, w.z * f, w.w * f);
              if (!out) *slot4(8 * c + i) = w;
              else if (mine) *reinterpret_cast<float4*>(dst + 32 * c + 4 * i) = w;
            }
          }
          has_slot = true;
          m_slot = m;
          ev_slot = ev;
        };
        for (int j = 0; j < n; ++j, ++step, phase ^= 1u) {
          const int j0 = (x.unit0 + first + j) * kKeys;
          const bool edge = edge_of(x, j0);
          ok = wait(kSFull + half, phase);
          if (!ok) break;
          tc_fence_after();
          const uint32_t ks = smem + L::KS + (uint32_t)(step & 1) * (kKeys * 4);
          const uint32_t vs = smem + L::VS + (uint32_t)(step & 1) * (kKeys * 4);
          // The scales, or the marks, of this step's tiles.  A stage of V is not filled again before this half's p is
          // there; one of K may be, so its scales have barriers of their own.
          if (I8) ok = wait(kScale + (step & 1), (uint32_t)(step >> 1) & 1u);
          if (ok && (I8 || edge)) {
            const int tv = 2 * step + 1;
            ok = wait(kFull + tv % kStages, (uint32_t)(tv / kStages) & 1u);
          }
          if (!ok) break;
          const int rel_lo = mine ? row_lo - j0 : 0, rel_hi = mine ? row_hi - j0 : kKeys;
          // 32 scores from column 32 c on, scaled and masked
          auto scores = [&](int c, float (&s)[32]) {
            tmem_ld_32x32(ts + 32u * c, s);
            if constexpr (I8) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const uint4 w = ld_shared16(ks + 128u * c + 16u * i);
                s[4 * i] *= __uint_as_float(w.x) * row_scale;
                s[4 * i + 1] *= __uint_as_float(w.y) * row_scale;
                s[4 * i + 2] *= __uint_as_float(w.z) * row_scale;
                s[4 * i + 3] *= __uint_as_float(w.w) * row_scale;
              }
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) s[i] *= row_scale;
            }
            if (edge) {
              uint32_t bad = 0u;
              if constexpr (!I8)
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(bad) : "r"(smem + L::BAD + 16u * (step & 1) + 4u * c));
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                if (!I8 && (bad >> i & 1u)) s[i] = __int_as_float(0x7fc00000);
                if (32 * c + i < rel_lo || 32 * c + i >= rel_hi) s[i] = -INFINITY;
              }
            }
          };
          float top = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            float s[32];
            scores(c, s);
#pragma unroll
            for (int i = 0; i < 32; ++i) top = fmaxf(top, s[i]);
          }
          int ev_new = ev;
          if constexpr (I8) {
            float big = 0.f;
            if (edge) {
              for (int i = 0; i < kKeys; ++i) {
                float v;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(vs + 4u * i));
                if (i >= rel_lo && i < rel_hi) big = fmaxf(big, v);
              }
            } else {
              const uint4 w = ld_shared16(smem + L::VMAX + 16u * (step & 1));
              big = fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)),
                          fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
            }
            ev_new = max(ev, min(kMaxExp, ((__float_as_int(big) >> 23) & 255) - 127));
          }
          const bool raise = m == -INFINITY ? top > -INFINITY : top > m + kLazy;
          const bool fresh = j % kChain == 0;
          if (fresh && j > 0) {  // a chain is complete: O into the slot, before m or ev change
            ok = wait(kPv + half, phase ^ 1u);
            if (!ok) break;
            tc_fence_after();
            fold(false);
          }
          if (__any_sync(0xffffffffu, raise || ev_new > ev)) {
            const float f = !raise ? 1.f : (m == -INFINITY ? 0.f : exp2_approx(m - top));
            if (!fresh) {
              ok = wait(kPv + half, phase ^ 1u);
              if (!ok) break;
              tc_fence_after();
              const float fo = I8 ? f * exp2_int(ev - ev_new) : f;
#pragma unroll 1
              for (int c = 0; c < D / 32; ++c) {
                float v[32];
                tmem_ld_32x32(to + 32u * c, v);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] *= fo;
                tmem_st_32x32(to + 32u * c, v);
              }
            }
            l *= f;
            if (raise) m = top;
            ev = ev_new;
          }
          const float base = kShift - (m == -INFINITY ? 0.f : m);
          const float down = I8 ? exp2_int(-ev) : 1.f;
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            float s[32];
            scores(c, s);
            float out[32];
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              float p[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                p[k] = exp2_approx(s[i + k] + base);
                l += p[k];
              }
              if constexpr (I8) {
                const uint4 w = ld_shared16(vs + 128u * c + 4u * i);
                const float sc[4] = {__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z),
                                     __uint_as_float(w.w)};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const bool hidden = edge && (32 * c + i + k < rel_lo || 32 * c + i + k >= rel_hi);
                  p[k] = hidden ? 0.f : p[k] * (sc[k] * down);
                }
              }
#pragma unroll
              for (int k = 0; k < 4; k += 2) {
                uint32_t hi, lo;
                split_f16(p[k], p[k + 1], hi, lo);
                out[(i + k) / 2] = __uint_as_float(hi);
                out[16 + (i + k) / 2] = __uint_as_float(lo);
              }
            }
            tmem_st_32x32(ts + 32u * c, out);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(kPFull + half));
        }
        if (ok) {
          ok = wait(kPv + half, phase ^ 1u);
          if (ok) {
            tc_fence_after();
            fold(true);
            tc_fence_before();
          }
        }
      } else {
        step += n;
      }
      if (!ok) break;
      if (!whole) {
        if (own < x.rows) {
          slot[(int64_t)kRows * D + own] = m;
          slot[(int64_t)kRows * D + kRows + own] = l;
        }
        if (first == 0 && half == 0 && q4 == 0 && lane == 0)
          *divided = {run.last_block(), x.h, (int)x.s.row0, x.s.n, x.r0, x.rows};
      }
    }
    if (!ok && lane == 0) give_up();
  }
};

template <int D, bool I8>
__global__ void __launch_bounds__(kThreads, 1) attention_tc_kernel(const AttnArgs a, Divided* divided) {
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
      mbar_init(smem + L::BARS + 8u * (kFull + s), 4);   // a producer warp each
      mbar_init(smem + L::BARS + 8u * (kEmpty + s), 1);  // the MMAs
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(smem + L::BARS + 8u * (kScale + h), 4);
      mbar_init(smem + L::BARS + 8u * (kQ + h), 4);      // a softmax warp each
      mbar_init(smem + L::BARS + 8u * (kSFull + h), 1);
      mbar_init(smem + L::BARS + 8u * (kPFull + h), 4);
      mbar_init(smem + L::BARS + 8u * (kPv + h), 1);
    }
    mbar_init(smem + L::BARS + 8u * kDrain, 1);
    *abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async_smem();
  }
  if (warp == 12) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
  Run run(a, reinterpret_cast<int64_t*>(base));  // the prefix sums lie where the tiles will
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const Kernel<D, I8> k{a, smem, __shfl_sync(0xffffffffu, *tmem_slot, 0), abort};
  if (warp < 4) k.producer(run);
  else if (warp < 12) k.softmax(run, (warp - 4) >> 2, divided + blockIdx.x);
  else k.issuer(run);
  tc_fence_before();
  __syncthreads();
  if (warp == 12) {
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
  attention_tc_kernel<D, I8><<<blocks, kThreads, smem, stream>>>(a, divided);
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
