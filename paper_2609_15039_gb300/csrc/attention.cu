// Attention of few rows over a paged cache (decode), and the entry points.
//
// o = sum_j softmax_j(scale q . k_j) v_j, in one pass over the keys with a running maximum m, total l and sums O.
// For few rows the pass is bound by reading the cache once.  A tile has 8 rows (for one new token, the query heads of
// a key head); its products run on mma.m16n8k16 with the 8 rows' high and low halves as the 16 rows of A, so that one
// instruction makes both terms of q = hi + lo, or of p = hi + lo, for which the stored binary16 (or int8) values are
// exact: fp32 accuracy at no further cost.  Keys and values go from global memory to the B fragments' registers
// directly, 16 bytes a lane, without shared memory: the order of the dimensions in a product is free, so a lane takes
// neighbouring ones (dims of a key for q . k, dims of four keys for p . v, whose pairs of keys are byte permutes).
// A warp takes 16 keys at a time, of one page, and holds the values' loads in flight while it makes the scores, the
// next keys' while it makes the sums.

#include <algorithm>
#include <atomic>
#include <cmath>

#include <cuda_fp16.h>

#include "attention.cuh"

namespace spl {
namespace {

constexpr int kThreads = 128, kWarps = 4;
constexpr int kRT = kRowsTile, kUnit = 64;
// p is held as 2^kShift p, at most 2^13, so that its low half keeps an absolute 2^-38 of the largest.
constexpr float kShift = 13.0f;
constexpr int kMinExp = -100, kMaxExp = 126;  // of the values' scales

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 ldg_stream(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}
__device__ __forceinline__ uint2 ldg_stream8(const void* p) {
  uint2 r;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}
// Whether a pair of binary16 holds an infinity or NaN.
__device__ __forceinline__ bool f16_special(uint32_t h) {
  return (h & 0x7c00u) == 0x7c00u || (h & 0x7c000000u) == 0x7c000000u;
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
  static constexpr int NB = D / 8;                 // n-blocks of p . v
  // first of the two neighbours (first + {0, 1}, and + {2, 3} for the upper half of a k-step) of step s
  static __device__ __forceinline__ int k_dim(int s, int t) {
    constexpr int per = E / 4;  // steps a chunk
    return (s / per) * 4 * E + t * E + 4 * (s % per);
  }
  // dim of column n of n-block nb
  static __device__ __forceinline__ int v_dim(int nb, int n) { return (nb / VE) * 8 * VE + n * VE + nb % VE; }
};

template <int D, bool I8>
__global__ void __launch_bounds__(kThreads, D == 128 ? 2 : 3) attention_rows_kernel(const AttnArgs a) {
  using F = Frag<D, I8>;
  constexpr int ESZ = I8 ? 1 : 2;
  constexpr int SLOT = kRT * (D + kSlotStats);
  extern __shared__ int64_t prefix[];
  __shared__ float s_o[kWarps][kRT][D];
  __shared__ float s_m[kWarps][kRT], s_l[kWarps][kRT];
  __shared__ int s_last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  AttnRun<kRT, kUnit, kThreads> run(a, prefix);
  for (; run.busy(); run.next()) {
    const AttnTile& x = run.x;
    // ---- the tile's rows: q = (hi + lo) 2^-e ----
    const int r = min(x.r0 + g, x.r0 + x.rows - 1);  // rows past the last repeat it
    const int token = r / a.group;
    uint32_t qa[F::STEPS][4];
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
      const float up = __int_as_float((e + 127) << 23);
      row_scale = a.scale_log2 * __int_as_float((127 - e) << 23);
#pragma unroll
      for (int s = 0; s < F::STEPS; ++s) {
        split_f16(v[s].x * up, v[s].y * up, qa[s][0], qa[s][1]);
        split_f16(v[s].z * up, v[s].w * up, qa[s][2], qa[s][3]);
      }
    }
    int row_lo, row_hi;
    row_keys(x.s, a.window, token, row_lo, row_hi);

    float o[F::NB][4];
#pragma unroll
    for (int i = 0; i < F::NB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
    float m = -INFINITY, l = 0.f;
    int ev = kMinExp;  // the sums are in units of 2^ev (int8: the exponent of the largest scale met)

    const int u_end = run.last();
    const int64_t head_slot = (int64_t)x.h << a.cache.page_shift;
    const int64_t page_slots = (int64_t)a.cache.heads << a.cache.page_shift;
    const int in_page = (1 << a.cache.page_shift) - 1;
    // the first slot of the 16 keys from j0 on, -1 if none of them is there
    auto slot_of = [&](int u) -> int64_t {
      const int j0 = (x.unit0 + u) * kUnit + warp * 16;
      if (u >= u_end || j0 >= x.key_hi || j0 + 16 <= x.key_lo) return -1;
      const int page = paged_page(a.cache, a.batch, x.b, j0);
      return page < 0 ? -1 : page * page_slots + head_slot + (j0 & in_page);
    };
    uint4 kr[2][F::KB];
    float ks[4];
    auto load_k = [&](int64_t slot, int j0) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int j = j0 + 8 * c + g;
        const bool there = slot >= 0 && j >= x.key_lo && j < x.key_hi;
        const char* p = static_cast<const char*>(a.cache.k) + ((slot + 8 * c + g) * D + t * F::E) * ESZ;
#pragma unroll
        for (int i = 0; i < F::KB; ++i) kr[c][i] = there ? ldg_stream(p + i * 64) : make_uint4(0u, 0u, 0u, 0u);
        if constexpr (I8) {
          const float2 sc = slot >= 0 ? __ldg(reinterpret_cast<const float2*>(a.cache.k_scale + slot + 8 * c + 2 * t))
                                      : make_float2(0.f, 0.f);
          ks[2 * c] = sc.x;
          ks[2 * c + 1] = sc.y;
        }
      }
    };
    int64_t slot = slot_of(run.first);
    load_k(slot, (x.unit0 + run.first) * kUnit + warp * 16);
    for (int u = run.first; u < u_end; ++u) {
      const int j0 = (x.unit0 + u) * kUnit + warp * 16;
      const int64_t next_slot = slot_of(u + 1);
      if (slot >= 0) {
        // ---- values in flight, scores meanwhile ----
        uint32_t vr[4][F::VC * F::VW];
        float vs[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int dj = 8 * (c >> 1) + 2 * t + (c & 1), j = j0 + dj;
          const bool there = j >= x.key_lo && j < x.key_hi;
          const char* p = static_cast<const char*>(a.cache.v) + ((slot + dj) * D + g * F::VE) * ESZ;
#pragma unroll
          for (int i = 0; i < F::VC; ++i) {
            if constexpr (F::VW == 4) {
              const uint4 w = there ? ldg_stream(p + i * 8 * F::VE * ESZ) : make_uint4(0u, 0u, 0u, 0u);
              vr[c][4 * i] = w.x, vr[c][4 * i + 1] = w.y, vr[c][4 * i + 2] = w.z, vr[c][4 * i + 3] = w.w;
            } else {
              const uint2 w = there ? ldg_stream8(p) : make_uint2(0u, 0u);
              vr[c][0] = w.x, vr[c][1] = w.y;
            }
          }
        }
        if constexpr (I8) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float2 sc = __ldg(reinterpret_cast<const float2*>(a.cache.v_scale + slot + 8 * c + 2 * t));
            vs[2 * c] = sc.x;
            vs[2 * c + 1] = sc.y;
          }
        }
        float s[4];  // keys 2t, 2t + 1, 2t + 8, 2t + 9 of row g
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < F::KB; ++i) {
            const uint32_t w[4] = {kr[c][i].x, kr[c][i].y, kr[c][i].z, kr[c][i].w};
            if constexpr (I8) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t biased = w[k] ^ 0x80808080u;
                mma16816(acc, qa[4 * i + k], i8_pair(biased, 0x4140u), i8_pair(biased, 0x4342u));
              }
            } else {
              mma16816(acc, qa[2 * i], w[0], w[1]);
              mma16816(acc, qa[2 * i + 1], w[2], w[3]);
            }
          }
          s[2 * c] = (acc[0] + acc[2]) * row_scale;
          s[2 * c + 1] = (acc[1] + acc[3]) * row_scale;
          if constexpr (I8) {
            s[2 * c] *= ks[2 * c];
            s[2 * c + 1] *= ks[2 * c + 1];
          }
        }
        load_k(next_slot, j0 + kUnit);
        // ---- softmax: a warp's edge blocks mask by row ----
        const bool edge = j0 < x.all_lo || j0 + 16 > x.all_hi;
        unsigned hidden = 0;
        if (edge) {
          bool bad[4] = {false, false, false, false};
          if constexpr (!I8) {  // a value that only some rows see must not reach the others as 0 times NaN
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
              for (int i = 0; i < F::VC * F::VW; ++i) bad[c] |= f16_special(vr[c][i]);
              const unsigned who = __ballot_sync(0xffffffffu, bad[c]);
              bad[c] = (who & (0x11111111u << t)) != 0;
              if (bad[c]) {
#pragma unroll
                for (int i = 0; i < F::VC * F::VW; ++i) vr[c][i] = 0u;
              }
            }
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int j = j0 + 8 * (c >> 1) + 2 * t + (c & 1);
            if (j < row_lo || j >= row_hi) {
              s[c] = -INFINITY;
              hidden |= 1u << c;
            } else if (bad[c]) {
              s[c] = __int_as_float(0x7fc00000);
            }
          }
        }
        float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float m_new = fmaxf(m, top);
        int ev_new = ev;
        if constexpr (I8) {
          float big = 0.f;  // of the scales that the row sees
#pragma unroll
          for (int c = 0; c < 4; ++c) big = fmaxf(big, (hidden >> c & 1u) ? 0.f : vs[c]);
          big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
          big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
          ev_new = max(ev, min(kMaxExp, ((__float_as_int(big) >> 23) & 255) - 127));
        }
        if (__any_sync(0xffffffffu, m_new > m || ev_new > ev)) {
          const float f = m == -INFINITY ? 0.f : exp2_approx(m - m_new);
          l *= f;
          const float fo = I8 ? f * exp2_int(ev - ev_new) : f;
#pragma unroll
          for (int i = 0; i < F::NB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] *= fo;
          m = m_new;
          ev = ev_new;
        }
        const float base = kShift - (m == -INFINITY ? 0.f : m);
        float p[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          p[c] = exp2_approx(s[c] + base);
          l += p[c];
          if constexpr (I8) p[c] = (hidden >> c & 1u) ? 0.f : p[c] * (vs[c] * exp2_int(-ev));
        }
        // ---- sums ----
        uint32_t pa[4];
        split_f16(p[0], p[1], pa[0], pa[1]);
        split_f16(p[2], p[3], pa[2], pa[3]);
#pragma unroll
        for (int w = 0; w < F::VC * F::VW; ++w) {
          if constexpr (I8) {
            const uint32_t k0 = vr[0][w] ^ 0x80808080u, k1 = vr[1][w] ^ 0x80808080u;
            const uint32_t k2 = vr[2][w] ^ 0x80808080u, k3 = vr[3][w] ^ 0x80808080u;
            const uint32_t lo0 = __byte_perm(k0, k1, 0x5140u), hi0 = __byte_perm(k0, k1, 0x7362u);
            const uint32_t lo1 = __byte_perm(k2, k3, 0x5140u), hi1 = __byte_perm(k2, k3, 0x7362u);
            mma16816(o[4 * w], pa, i8_pair(lo0, 0x4140u), i8_pair(lo1, 0x4140u));
            mma16816(o[4 * w + 1], pa, i8_pair(lo0, 0x4342u), i8_pair(lo1, 0x4342u));
            mma16816(o[4 * w + 2], pa, i8_pair(hi0, 0x4140u), i8_pair(hi1, 0x4140u));
            mma16816(o[4 * w + 3], pa, i8_pair(hi0, 0x4342u), i8_pair(hi1, 0x4342u));
          } else {
            mma16816(o[2 * w], pa, __byte_perm(vr[0][w], vr[1][w], 0x5410u), __byte_perm(vr[2][w], vr[3][w], 0x5410u));
            mma16816(o[2 * w + 1], pa, __byte_perm(vr[0][w], vr[1][w], 0x7632u),
                     __byte_perm(vr[2][w], vr[3][w], 0x7632u));
          }
        }
      } else {
        load_k(next_slot, j0 + kUnit);
      }
      slot = next_slot;
    }

    // ---- the warps' sums together, in their order ----
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    __syncthreads();  // the shared arrays' last readers are done
    if (t == 0) {
      s_m[warp][g] = m;
      s_l[warp][g] = l;
    }
    __syncthreads();
    float m_all = s_m[0][g];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m_all = fmaxf(m_all, s_m[w][g]);
    const float f = (m == -INFINITY ? (l != l ? l : 0.f) : exp2_approx(m - m_all)) * (I8 ? exp2_int(ev) : 1.f);
#pragma unroll
    for (int nb = 0; nb < F::NB; ++nb) {
      s_o[warp][g][F::v_dim(nb, 2 * t)] = (o[nb][0] + o[nb][2]) * f;
      s_o[warp][g][F::v_dim(nb, 2 * t + 1)] = (o[nb][1] + o[nb][3]) * f;
    }
    __syncthreads();
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
    for (int i = threadIdx.x; i < x.rows * Q4; i += kThreads) {
      const int row = i / Q4, d = 4 * (i % Q4);
      float top = s_m[0][row];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, s_m[w][row]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float total = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 part = *reinterpret_cast<const float4*>(&s_o[w][row][d]);
        v = make_float4(v.x + part.x, v.y + part.y, v.z + part.z, v.w + part.w);
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
    __syncthreads();
    if (threadIdx.x == 0) {
      __threadfence();
      s_last = atomicAdd(a.counters + c0, 1u) == (unsigned)(c1 - c0);
      __threadfence();
    }
    __syncthreads();
    if (!s_last) continue;
    auto piece = [&](int c) { return a.slots + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * SLOT; };
    // rows' maxima over the pieces
    for (int row = warp; row < x.rows; row += kWarps) {
      float top = -INFINITY;
      for (int c = c0 + lane; c <= c1; c += 32) top = fmaxf(top, __ldcg(piece(c) + kRT * D + row));
#pragma unroll
      for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
      if (lane == 0) s_m[0][row] = top;
    }
    __syncthreads();
    // each warp every kWarps-th piece, then the warps in order
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
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRT / ROWS; ++i) {
      const int row = i * ROWS + sub;
      *reinterpret_cast<float4*>(&s_o[warp][row][d4]) = acc[i];
      if (d4 == 0) s_l[warp][row] = tot[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < x.rows * Q4; i += kThreads) {
      const int row = i / Q4, d = 4 * (i % Q4);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float total = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 part = *reinterpret_cast<const float4*>(&s_o[w][row][d]);
        v = make_float4(v.x + part.x, v.y + part.y, v.z + part.z, v.w + part.w);
        total += s_l[w][row];
      }
      store(row, d, v, total);
    }
    if (threadIdx.x == 0) a.counters[c0] = 0u;
  }
}

template <int D, bool I8>
int rows_blocks(int sms) {
  static std::atomic<int> known{0};
  int per_sm = known.load(std::memory_order_relaxed);
  if (per_sm == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, attention_rows_kernel<D, I8>, kThreads,
                                                      kMaxSeqs * sizeof(int64_t)) != cudaSuccess ||
        per_sm < 1)
      return sms;
    known.store(per_sm, std::memory_order_relaxed);
  }
  return per_sm * sms;
}

}  // namespace

int attention_rows_blocks(int head_dim, bool i8, int sms) {
  if (head_dim == 128) return i8 ? rows_blocks<128, true>(sms) : rows_blocks<128, false>(sms);
  return i8 ? rows_blocks<64, true>(sms) : rows_blocks<64, false>(sms);
}

spl_status run_attention_rows(const AttnArgs& a, int head_dim, bool i8, int blocks, cudaStream_t stream) {
  auto launch = [&](auto kernel) {
    kernel<<<blocks, kThreads, a.batch.seqs * sizeof(int64_t), stream>>>(a);
    return launch_status();
  };
  if (head_dim == 128) return i8 ? launch(attention_rows_kernel<128, true>) : launch(attention_rows_kernel<128, false>);
  return i8 ? launch(attention_rows_kernel<64, true>) : launch(attention_rows_kernel<64, false>);
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
  if (q_heads / cache->kv_heads > 1024 || rows * (q_heads / cache->kv_heads) > INT32_MAX / 2) return SPL_ESHAPE;
  return paged_batch_view(b, batch, rows);
}

// The few-row kernel where every sequence's rows of a key head fit its tile, or where the units (64 keys of a tile) that
// the batch can have, by its longest chunk and its page table, are few: the tensor-core kernel costs 15 us more at the
// start and a tenth as much per unit.  Measured with 24 query heads on 8 (few rows, tensor cores): 16 rows over 2048 keys
// 24, 27 us, over 8192 50, 39; 64 rows over 512 25, 35, over 2048 47, 42; 16 sequences of 8 rows over 128 22, 32, over
// 512 41, 40.
constexpr int64_t kFewUnits = 3000;
Shape shape_of(const spl_kv_cache* cache, const spl_kv_batch* batch, int64_t q_heads) {
  const int d = (int)cache->head_dim, sms = device_sm_count();
  Shape s;
  const int64_t tiles = ceil_div(std::max<int64_t>(batch->max_rows, 1) * (q_heads / cache->kv_heads), kRowsTile);
  const int64_t units = ceil_div(batch->max_pages * cache->page_size, kUnit);
  s.few = tiles == 1 || (double)tiles * (double)units * (double)(batch->seqs * cache->kv_heads) <= kFewUnits;
  if (s.few) {
    s.blocks = attention_rows_blocks(d, cache->format == SPL_KV_I8, sms);
    s.bytes = kCounterBytes + (size_t)s.blocks * 2 * kRowsTile * (d + kSlotStats) * sizeof(float);
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

extern "C" spl_status spl_paged_attention(float* out, int64_t ldo, const float* Q, int64_t ldq,
                                          const spl_kv_cache* cache, const spl_kv_batch* batch, int64_t rows,
                                          int64_t q_heads, float scale, int64_t window, void* workspace,
                                          size_t workspace_bytes, cudaStream_t stream) {
  AttnArgs a = {};
  spl_status st = check(cache, batch, rows, q_heads, &a.cache, &a.batch);
  if (st != SPL_OK) return st;
  const int64_t width = q_heads * cache->head_dim;
  if (ldo < 0 || ldq < 0 || window < 0 || !std::isfinite(scale)) return SPL_EINVAL;
  if (rows == 0 || a.batch.seqs == 0) return SPL_OK;
  if (!out || !Q) return SPL_EINVAL;
  if (rows > 1 && (ldo < width || ldq < width)) return SPL_EINVAL;
  if (!aligned16(out) || !aligned16(Q) || (rows > 1 && (ldo % 4 != 0 || ldq % 4 != 0))) return SPL_EALIGN;
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
  a.min_units = 2;
  const int d = (int)cache->head_dim;
  const bool i8 = cache->format == SPL_KV_I8;
  return s.few ? run_attention_rows(a, d, i8, s.blocks, stream) : run_attention_tc(a, d, i8, s.blocks, stream);
}
