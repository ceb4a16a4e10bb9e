// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// A sequence's drafts x_0..x_{k-1} were sampled from q_0..q_{k-1}; the target gives p_0..p_k.  Draft i is accepted
// while u_i q_i(x_i) < p_i(x_i); the token after the accepted ones is drawn from max(p_i - q_i, 0) at the first
// rejected row, or from p_k.  The draw is a race of exponentials: with e(v) ~ Exp(1) independent, the v with the
// largest w(v) / e(v) has probability w(v) / sum w, so w needs no normalising and no running sum, and every operation
// is one correctly rounded fp32 one: the outcome does not depend on the order of anything.
//
// Bound by the reading of one row of p, e (and q) for each sequence, which several blocks share; the largest key
// (bits of the ratio, then the lowest index) is an atomic maximum, whose order does not matter.

#include <algorithm>

#include "paged.cuh"

namespace spl {
namespace {

constexpr int kThreads = 256;

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

__device__ __forceinline__ void race(unsigned long long& key, float weight, float e, int64_t v) {
  const float r = __fdiv_rn(weight, e) + 0.0f;  // -0 counts as 0
  if (!(r >= 0.0f)) return;                     // NaN, or a negative random number: never chosen
  const unsigned long long k = (unsigned long long)__float_as_uint(r) << 32 | (0xffffffffu - (uint32_t)v);
  key = k > key ? k : key;
}

// The race over [v0, v1) of one row; q null: the weights are p's own.  VEC: rows and v0 are 16-byte aligned.
template <bool VEC>
__device__ unsigned long long race_row(const float* p, const float* q, const float* e, int64_t v0, int64_t v1,
                                       bool& positive) {
  unsigned long long key = 0;
  auto one = [&](float pv, float qv, float ev, int64_t v) {
    const float w = q ? fmaxf(__fsub_rn(pv, qv), 0.0f) : pv;
    positive |= w > 0.0f;
    race(key, w, ev, v);
  };
  if constexpr (VEC) {
    constexpr int UNROLL = 4;
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int64_t base = v0 + 4 * threadIdx.x; base < v1; base += 4 * kThreads * UNROLL) {
      float4 a[UNROLL], b[UNROLL], c[UNROLL];
#pragma unroll
      for (int i = 0; i < UNROLL; ++i) {
        const int64_t v = base + 4 * kThreads * i;
        const bool in = v + 4 <= v1;
        a[i] = in ? __ldcs(reinterpret_cast<const float4*>(p + v)) : zero;
        b[i] = in && q ? __ldcs(reinterpret_cast<const float4*>(q + v)) : zero;
        c[i] = in ? __ldcs(reinterpret_cast<const float4*>(e + v)) : zero;
      }
#pragma unroll
      for (int i = 0; i < UNROLL; ++i) {
        const int64_t v = base + 4 * kThreads * i;
        if (v + 4 <= v1) {
          one(a[i].x, b[i].x, c[i].x, v);
          one(a[i].y, b[i].y, c[i].y, v + 1);
          one(a[i].z, b[i].z, c[i].z, v + 2);
          one(a[i].w, b[i].w, c[i].w, v + 3);
        } else {
          for (int64_t t = v; t < v1; ++t) one(p[t], q ? q[t] : 0.f, e[t], t);
        }
      }
    }
  } else {
    constexpr int UNROLL = 8;
    for (int64_t base = v0 + threadIdx.x; base < v1; base += kThreads * UNROLL) {
      float a[UNROLL], b[UNROLL], c[UNROLL];
#pragma unroll
      for (int i = 0; i < UNROLL; ++i) {
        const int64_t v = base + kThreads * i;
        a[i] = v < v1 ? __ldcs(p + v) : 0.f;
        b[i] = v < v1 && q ? __ldcs(q + v) : 0.f;
        c[i] = v < v1 ? __ldcs(e + v) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < UNROLL; ++i)
        if (base + kThreads * i < v1) one(a[i], b[i], c[i], base + kThreads * i);
    }
  }
  return key;
}

template <bool VEC>
__global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyArgs a, int64_t per_split) {
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
  const float* e = a.e + b * a.lde;
  const int64_t v0 = blockIdx.x * per_split, v1 = min(v0 + per_split, a.vocab);
  bool positive = false;
  unsigned long long key = race_row<VEC>(p, q, e, v0, v1, positive);
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
    key = block_max(race_row<VEC>(p, nullptr, e, 0, a.vocab, positive), keys);
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
  // About four blocks an SM in all, each with at least one trip of its threads; slices are whole 16-byte units.
  const int64_t most = ceil_div(vocab, (int64_t)4 * kThreads);
  const int64_t want = ceil_div((int64_t)4 * device_sm_count(), seqs);
  const int64_t per_split = round_up(ceil_div(vocab, std::max<int64_t>(1, std::min(most, want))), 4);
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
