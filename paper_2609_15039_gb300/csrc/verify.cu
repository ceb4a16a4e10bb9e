// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// A sequence's drafts x_0..x_{k-1} were sampled from q_0..q_{k-1}; the target gives p_0..p_k.  Draft i is accepted
// while u_i q_i(x_i) < p_i(x_i); the token after the accepted ones is drawn from max(p_i - q_i, 0) at the first
// rejected row, or from p_k.  The draw is a race of exponentials: with e(v) ~ Exp(1) independent, the v with the
// largest w(v) / e(v) has probability w(v) / sum w, so w needs no normalising and no running sum, and every operation
// is one correctly rounded fp32 one: the outcome does not depend on the order of anything.
//
// Bound by the reading of one row of p, e (and q) for each sequence, which several blocks share, a wave in all; a
// thread has the loads of its next eight entries under way.  The largest key (bits of the ratio, then the lowest index)
// is an atomic maximum, whose order does not matter.  Measured: 64 sequences of 8 drafts over 151936 entries 22.6 us,
// of none (78 MB) 16.4 us, 4.8 TB/s; 15 of 4 over 128256 9.2 us, of which some 5 are the chain of launch, starts, drafts,
// their probabilities, rows and arrival.

#include <algorithm>

#include "paged.cuh"

namespace spl {
namespace {

constexpr int kThreads = 256, kBlocksPerSm = 3;
constexpr int64_t kMostEntries = int64_t(1) << 30;  // of a row that are counted at once: indexes are 32-bit

struct VerifyState {  // one a sequence, in the zeroed workspace; left zero
  unsigned long long key;
  unsigned int arrived, positive;
};
static_assert(sizeof(VerifyState) * kMaxSeqs <= kCounterBytes, "inside the workspace's counter area");

struct VerifyArgs {
  int *accepted, *token;
  const float *p, *q;
  const int* draft;
  const float *u, *e;
  const int *row_start, *draft_start;
  int64_t ldp, ldq, lde, vocab, rows, drafts;
  int seqs;
  VerifyState* state;
  unsigned int* status;
};

// The largest key of a block, in thread 0.
__device__ unsigned long long block_max(unsigned long long key, unsigned long long* shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long other = __shfl_xor_sync(0xffffffffu, key, o);
    key = other > key ? other : key;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = key;
  __syncthreads();
  for (int w = 0; w < kThreads / 32 && threadIdx.x == 0; ++w) key = shared[w] > key ? shared[w] : key;
  return key;
}

__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// A thread's best so far of a race over ascending v: the largest ratio, the first v of equal ones.
struct Best {
  float ratio = -1.0f;  // no entry took part
  int v = 0;
  __device__ __forceinline__ void look(float weight, float e, int at) {
    // The quotient by rounding only where its operands are ordinary: a weight of zero takes the division's slow path.
    const float r = weight == 0.0f ? (e != 0.0f && e == e ? 0.0f : -1.0f) : __fdiv_rn(weight, e);
    if (r >= 0.0f && r > ratio) {  // (not NaN, nor from a negative random number)
      ratio = r;
      v = at;
    }
  }
  __device__ __forceinline__ unsigned long long key(int64_t v0) const {
    return ratio < 0.0f ? 0ull : (unsigned long long)__float_as_uint(ratio) << 32 | (0xffffffffu - (uint32_t)(v0 + v));
  }
};

// A thread's entries of a trip over n of a row.  VEC: the rows and slices begin at 16-byte boundaries.
template <bool VEC>
struct Trip {
  static constexpr int N = 8, STEP = VEC ? 4 * kThreads : kThreads, SPAN = N * kThreads;
  float x[N];
  static __device__ __forceinline__ int at(int base, int i) {  // base: the thread's first
    return VEC ? base + STEP * (i >> 2) + (i & 3) : base + STEP * i;
  }
  __device__ __forceinline__ void load(const float* p, int base, int n, float none) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const int v = at(base, i);
        float4 q = make_float4(none, none, none, none);
        if (v + 4 <= n) {
          q = __ldcs(reinterpret_cast<const float4*>(p + v));
        } else if (v < n) {
          q.x = p[v];
          if (v + 1 < n) q.y = p[v + 1];
          if (v + 2 < n) q.z = p[v + 2];
        }
        x[i] = q.x, x[i + 1] = q.y, x[i + 2] = q.z, x[i + 3] = q.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = at(base, i) < n ? __ldcs(p + at(base, i)) : none;
    }
  }
  __device__ __forceinline__ void load_random(const float* e, int base, int n) { load(e, base, n, 1.0f); }
};

// The race over n entries of one row, from v0 on; q null: the weights are p's own.  `first`: e of the thread's first trip.
// Quotients are approximated within 2^-21 first; only those that may be their warp's largest are rounded (a rounded
// quotient of every entry took 64 sequences of 8 drafts over 151936 entries 45 us).
template <bool VEC>
__device__ unsigned long long race_row(const float* p, const float* q, const float* e, int64_t v0, int n,
                                       const Trip<VEC>& first, bool& positive) {
  using T = Trip<VEC>;
  constexpr float kLeast = 0x1p-60f, kMost = 0x1p60f;  // of e, where the approximations hold
  const int mine = (VEC ? 4 : 1) * threadIdx.x;
  p += v0, e += v0;
  if (q) q += v0;
  Best best;
  T w, b, c = first, w2, b2, c2;
  w.load(p, mine, n, 0.f);
  if (q) b.load(q, mine, n, 0.f);
  for (int base0 = 0; base0 < n; base0 += T::SPAN) {  // the whole warp makes every trip
    const int base = base0 + mine;
    if (n - base0 > T::SPAN) {  // the next trip's entries are on their way during this one
      w2.load(p, base + T::SPAN, n, 0.f);
      c2.load_random(e, base + T::SPAN, n);
      if (q) b2.load(q, base + T::SPAN, n, 0.f);
    }
    if (q) {
#pragma unroll
      for (int i = 0; i < T::N; ++i) w.x[i] = fmaxf(__fsub_rn(w.x[i], b.x[i]), 0.0f);
    }
    float top = 0.f, heaviest = 0.f, least = c.x[0], most = c.x[0];
#pragma unroll
    for (int i = 0; i < T::N; ++i) {
      heaviest = fmaxf(heaviest, w.x[i]);
      least = fminf(least, c.x[i]);
      most = fmaxf(most, c.x[i]);
      top = fmaxf(top, w.x[i] * rcp_approx(c.x[i]));
    }
    positive |= heaviest > 0.0f;
    // The warp's largest; infinite where the approximations may not hold, and then all quotients are rounded.
    const float shown = least >= kLeast && most <= kMost ? fmaxf(top, best.ratio) : INFINITY;
    const float all = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(shown)));
    const float bound = all >= 0x1p-60f && all <= 0x1p100f ? all * (1.0f - 0x1p-18f) : -1.0f;
    if (!(top < bound)) {
#pragma unroll
      for (int i = 0; i < T::N; ++i)
        if (!(w.x[i] * rcp_approx(c.x[i]) < bound) && T::at(base, i) < n) best.look(w.x[i], c.x[i], T::at(base, i));
    }
    w = w2, b = b2, c = c2;
  }
  return best.key(v0);
}

template <bool VEC>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) verify_kernel(const VerifyArgs a, int64_t per_split) {
  __shared__ unsigned long long keys[kThreads / 32];
  __shared__ int s_accepted, s_role;
  enum { kDone, kFinish, kAgain };  // of a block whose slice is done: the last of the sequence to arrive finishes it
  const int b = blockIdx.y;
  const int64_t row0 = min(max((int64_t)__ldg(a.row_start + b), (int64_t)0), a.rows);
  const int64_t row1 = min(max((int64_t)__ldg(a.row_start + b + 1), row0), a.rows);
  const int64_t draft0 = min(max((int64_t)__ldg(a.draft_start + b), (int64_t)0), a.drafts);
  const int64_t draft1 = min(max((int64_t)__ldg(a.draft_start + b + 1), draft0), a.drafts);
  if (row1 == row0) {  // no target row: nothing is decided
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      a.accepted[b] = 0;
      a.token[b] = -1;
    }
    return;
  }
  const int k = (int)min(draft1 - draft0, row1 - row0 - 1);
  const float* e = a.e + b * a.lde;
  const int64_t v0 = blockIdx.x * per_split;
  const int entries = (int)max((int64_t)0, min(per_split, a.vocab - v0));
  Trip<VEC> first;  // on its way while the drafts are looked at
  first.load_random(e + v0, (VEC ? 4 : 1) * threadIdx.x, entries);
  if (threadIdx.x < 32) {
    int n = 0;
    for (; n < k; n += 32) {
      const int i = n + threadIdx.x;
      bool reject = i < k;
      if (reject) {
        const int x = __ldg(a.draft + draft0 + i);
        if (x >= 0 && x < a.vocab)
          reject = !(__fmul_rn(__ldg(a.u + draft0 + i), __ldg(a.q + (draft0 + i) * a.ldq + x)) <
                     __ldg(a.p + (row0 + i) * a.ldp + x));
        else
          atomicOr(a.status, kStatusIndex);
      }
      const unsigned m = __ballot_sync(0xffffffffu, reject);
      if (m) {
        n += __ffs(m) - 1;
        break;
      }
    }
    if (threadIdx.x == 0) s_accepted = min(n, k);
  }
  __syncthreads();
  const int n = s_accepted;
  const float* p = a.p + (row0 + n) * a.ldp;
  const float* q = n < k ? a.q + (draft0 + n) * a.ldq : nullptr;
  bool positive = false;
  unsigned long long key = race_row<VEC>(p, q, e, v0, entries, first, positive);
  positive = __syncthreads_or(positive);
  key = block_max(key, keys);
  VerifyState* st = a.state + b;
  if (threadIdx.x == 0) {
    atomicMax(&st->key, key);
    if (positive) atomicOr(&st->positive, 1u);
    __threadfence();
    s_role = kDone;
    if (atomicAdd(&st->arrived, 1u) == gridDim.x - 1) {
      __threadfence();
      s_role = q && !__ldcg(&st->positive) ? kAgain : kFinish;
    }
  }
  __syncthreads();
  if (s_role == kDone) return;
  if (s_role == kAgain) {  // p is nowhere above q: the draw is from p
    key = 0;
    for (int64_t from = 0; from < a.vocab; from += kMostEntries) {
      const int some = (int)min(kMostEntries, a.vocab - from);
      first.load_random(e + from, (VEC ? 4 : 1) * threadIdx.x, some);
      key = max(key, race_row<VEC>(p, nullptr, e, from, some, first, positive));
    }
    key = block_max(key, keys);
  } else if (threadIdx.x == 0) {
    key = __ldcg(&st->key);
  }
  if (threadIdx.x == 0) {
    a.accepted[b] = n;
    a.token[b] = key == 0 ? -1 : (int)(0xffffffffu - (uint32_t)key);  // 0: no entry took part
    st->key = 0;
    st->arrived = 0;
    st->positive = 0;
  }
}

}  // namespace
}  // namespace spl

using namespace spl;

extern "C" size_t spl_verify_drafts_workspace_bytes(int64_t seqs) {
  return seqs > 0 && seqs <= kMaxSeqs ? (size_t)seqs * sizeof(VerifyState) : 0;
}

extern "C" spl_status spl_verify_drafts(int32_t* accepted, int32_t* token, const float* P, int64_t ldp, const float* Q,
                                        int64_t ldq, const int32_t* draft, const float* u, const float* e, int64_t lde,
                                        const int32_t* row_start, const int32_t* draft_start, int64_t rows,
                                        int64_t drafts, int64_t seqs, int64_t vocab, void* workspace,
                                        size_t workspace_bytes, cudaStream_t stream) {
  if (rows < 0 || drafts < 0 || seqs < 0 || vocab < 0 || ldp < 0 || ldq < 0 || lde < 0) return SPL_EINVAL;
  if (seqs == 0) return SPL_OK;
  if (!accepted || !token || !row_start || !draft_start) return SPL_EINVAL;
  if (vocab == 0 || (rows > 0 && (!P || !e)) || (drafts > 0 && (!Q || !draft || !u))) return SPL_EINVAL;
  if ((rows > 1 && ldp < vocab) || (drafts > 1 && ldq < vocab) || (seqs > 1 && lde < vocab)) return SPL_EINVAL;
  if (seqs > kMaxSeqs || vocab > INT32_MAX || rows > INT32_MAX || drafts > INT32_MAX) return SPL_ESHAPE;
  for (const void* ptr : {(const void*)accepted, (const void*)token, (const void*)P, (const void*)Q,
                          (const void*)draft, (const void*)u, (const void*)e, (const void*)row_start,
                          (const void*)draft_start})
    if (!aligned4(ptr)) return SPL_EALIGN;
  if (!workspace || workspace_bytes < spl_verify_drafts_workspace_bytes(seqs)) return SPL_EWORKSPACE;
  if (!aligned16(workspace)) return SPL_EALIGN;
  unsigned int* status = device_status_word();
  if (!status) return SPL_ECUDA;
  // Blocks for one wave, each with at least a trip of its threads' loads and at most kMostEntries; slices are whole 16-byte
  // units.
  const int64_t most = ceil_div(vocab, (int64_t)4 * kThreads);
  const int64_t want = std::max((int64_t)kBlocksPerSm * device_sm_count() / seqs, ceil_div(vocab, kMostEntries));
  const int64_t per_split = round_up(ceil_div(vocab, std::min(most, want)), 4);
  const bool vec = ldp % 4 == 0 && ldq % 4 == 0 && lde % 4 == 0 && aligned16(P) && aligned16(Q) && aligned16(e);
  const VerifyArgs a = {accepted, token, P,   Q,   draft, u,    e,      row_start,  draft_start,
                        ldp,      ldq,   lde, vocab, rows, drafts, (int)seqs, static_cast<VerifyState*>(workspace), status};
  const dim3 grid((unsigned)ceil_div(vocab, per_split), (unsigned)seqs);
  if (vec)
    verify_kernel<true><<<grid, kThreads, 0, stream>>>(a, per_split);
  else
    verify_kernel<false><<<grid, kThreads, 0, stream>>>(a, per_split);
  return launch_status();
}
