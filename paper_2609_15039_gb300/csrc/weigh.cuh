// Attention weights of stored tokens: what the kernels for few and for many rows share.
#pragma once

#include "attention.cuh"

namespace spl {

struct WeighCall {
  float* score;  // [pages, heads, page]
  const float* q;
  int64_t ldq;
  PagedCache cache;
  PagedBatch batch;
  int group, q_heads;
  int window;        // INT_MAX for all
  float scale_log2;  // scale log2(e)
  float decay;
  void* workspace;
};

// Many rows, on the 5th-generation tensor cores (weigh_tc.cu).
size_t weigh_tc_bytes(const PagedCache& cache, const PagedBatch& batch, int64_t q_heads, int head_dim);
spl_status run_weigh_tc(const WeighCall& w, int head_dim, bool i8, cudaStream_t stream);

}  // namespace spl
