// What the kernels over a paged KV cache share: the cache and the ragged batch as the device sees them.
#pragma once

#include "common.cuh"

namespace spl {

// Device status bit of a page id, length or token id outside its range (spl_get_device_status).
constexpr unsigned int kStatusIndex = 2u;
// Address of the device status word on the current device (gemm_tc.cu).
unsigned int* device_status_word();

struct PagedCache {
  void* k;         // [pages, heads, page, dim] binary16 or int8
  void* v;
  float* k_scale;  // [pages, heads, page], int8 only
  float* v_scale;
  int pages, heads, page_shift;  // page = 1 << page_shift tokens
};

struct PagedBatch {
  const int* row_start;  // [seqs + 1]
  const int* kv_len;     // [seqs]
  const int* table;      // [seqs, max_pages]
  int seqs;
  int64_t max_pages;
  int64_t rows;
  unsigned int* status;
};

// Sequence b's first row, rows, stored tokens and first row's position, brought inside the arrays whatever the device
// arrays hold.  A length past the table ends there, but its rows stand where it says: those past the end have no place.
struct PagedSeq {
  int row0, n, len, pos0;
};
// LATE: by plain loads, for a kernel that may begin before the one ahead of it has written the batch's arrays: __ldg is for
// what nobody writes while the kernel lives, and may be moved above the wait for that one.
template <bool LATE>
__device__ __forceinline__ int paged_load(const int* p) {
  if constexpr (LATE) return *p;
  else return __ldg(p);
}
template <bool LATE = false>
__device__ __forceinline__ PagedSeq paged_seq(const PagedBatch& batch, int page_shift, int b) {
  PagedSeq s;
  const int64_t a = paged_load<LATE>(batch.row_start + b), e = paged_load<LATE>(batch.row_start + b + 1);
  const int64_t row0 = a < 0 ? 0 : (a > batch.rows ? batch.rows : a);
  const int64_t end = e < row0 ? row0 : (e > batch.rows ? batch.rows : e);
  s.row0 = (int)row0;
  s.n = (int)(end - row0);
  const int64_t room = batch.max_pages << page_shift;
  const int said = paged_load<LATE>(batch.kv_len + b), len = said < 0 ? 0 : said;
  s.len = len > room ? (int)room : len;
  s.pos0 = len - s.n;
  if (s.len != said) atomicOr(batch.status, kStatusIndex);
  return s;
}

// The page of position pos (inside the table) of sequence b, or -1 (and the status bit) for an id outside the pool.
__device__ __forceinline__ int paged_page(const PagedCache& cache, const PagedBatch& batch, int b, int pos) {
  const int page = __ldg(batch.table + b * batch.max_pages + (pos >> cache.page_shift));
  if ((unsigned)page < (unsigned)cache.pages) return page;
  atomicOr(batch.status, kStatusIndex);
  return -1;
}

// Index of (page, head, slot of position pos) among the stored vectors.
__device__ __forceinline__ int64_t paged_slot(const PagedCache& cache, int page, int head, int pos) {
  return ((((int64_t)page * cache.heads + head) << cache.page_shift) + (pos & ((1 << cache.page_shift) - 1)));
}

// The last b of [0, seqs) with start[b] <= row (0 if there is none), found by a whole warp 32 ways at a time.
__device__ __forceinline__ int paged_find(const int* start, int seqs, int64_t row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = seqs;
  while (n > 1) {
    const int step = (n + 31) >> 5, i = lane * step;
    const unsigned below = __ballot_sync(0xffffffffu, i < n && __ldg(start + lo + (i < n ? i : 0)) <= row);
    const int pick = below ? 31 - __clz(below) : 0;
    lo += pick * step;
    n = n - pick * step < step ? n - pick * step : step;
  }
  return lo;
}

// Checks shared by the entries; fill the device's view of the cache and of the batch (but for its status word, which
// an entry sets before it launches).
spl_status paged_cache_view(PagedCache* out, const spl_kv_cache* cache);
spl_status paged_batch_view(PagedBatch* out, const PagedCache& cache, const spl_kv_batch* batch, int64_t rows);
constexpr int kMaxSeqs = 4096;
constexpr int64_t kMaxLength = int64_t(1) << 30;  // tokens of a sequence: positions and ends of tiles are 32-bit
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace spl
