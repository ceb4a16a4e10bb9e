// Moves within a paged cache: the eviction of all but the heaviest and the latest tokens, and an accepted path's rows.
//
// Eviction, for each sequence and key head by itself: of `len` tokens the last `recent` stay and of the others the
// keep - recent with the largest scores, the earliest of equal ones; they keep their order and go to the positions 0 ..
// keep - 1.  Two launches.  The first chooses: the scores become whole numbers that order as they do, the smallest that
// stays is found digit by digit (8 bits a round, a histogram in shared memory), and the positions that stay are written
// down in order, strip after strip, by a prefix sum.  The second moves, bound by HBM: a block has K's or V's vectors of one
// head, or 32 bytes of each.  In place a target lies at or before its source, and a block's trips are
// in the targets' order, so that it suffices that a trip's loads are done before its stores: what a trip overwrites are
// sources of itself or of trips before it.  Into other pages there is no such order, and a head's tokens are shared out.
//
// Measured with 8 heads of 128 dims, binary16: 32 sequences of 1600 to 16000 tokens cut to 6000, into other pages, 21 and 231 us
// (5.8 TB/s); one cut from 1250 to 1000 8.9 and 7.6 us (launches and three dependent loads each).  15 of 500 to 5000, int8, cut
// to 800: 12.4 and 17 us, in columns of 32 bytes (whole vectors: 20).
//
// An accepted path (a handful of tokens): a thread has 16 bytes of a vector, or a scale, and moves them one after another.

#include <algorithm>

#include "paged.cuh"

namespace spl {
namespace {

constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32;
constexpr int kHeld = 24576;  // scores held in shared memory (96 KB: two blocks an SM); past them they are read again
constexpr int kPer = 4, kStrip = kPer * kSelectThreads;

constexpr int kPlan = 3;
struct EvictArgs {
  PagedCache cache;
  PagedBatch batch;
  float* score;          // [pages, heads, page]
  const int* out_table;  // where the tokens go: [seqs, max_pages], or null for where they are
  int* out_len;
  int keep, recent;
  int64_t chosen;  // places of a (sequence, head) in `list`
  int* list;       // the positions that stay of those before the last `recent`, in order
  int* plan;       // [seqs][kPlan]: tokens that move, length after and before
};

// A whole number that orders like the score: -inf .. +inf from 1 on (both zeros are one), NaN below them as 0.
__device__ __forceinline__ uint32_t score_order(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// One block a (key head, sequence).
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const EvictArgs a) {
  extern __shared__ __align__(16) uint32_t held[];
  __shared__ int histogram[256], warp_sums[kSelectWarps], s_digit, s_left;
  __shared__ uint32_t s_low, s_high;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_trigger();
  const PagedSeq s = paged_seq(a.batch, a.cache.page_shift, b);
  const bool over = s.len > a.keep;
  if (h == 0 && tid == 0) {
    a.plan[kPlan * b] = over ? a.keep : (a.out_table ? s.len : 0);
    a.plan[kPlan * b + 1] = over ? a.keep : s.len;
    a.plan[kPlan * b + 2] = s.len;
  }
  const int early = s.len - a.recent, want = a.keep - a.recent;
  if (!over || want == 0) return;
  int* list = a.list + ((int64_t)b * a.cache.heads + h) * a.chosen;
  const bool wide = (reinterpret_cast<uintptr_t>(a.score) & 15u) == 0;
  // Four scores at a time: they lie in one page.
  auto read = [&](int pos) {
    const int page = paged_page(a.cache, a.batch, b, pos);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (page >= 0) {
      const float* at = a.score + paged_slot(a.cache, page, h, pos);
      if (wide) {
        const float4 x = __ldg(reinterpret_cast<const float4*>(at));
        v = make_uint4(score_order(x.x), score_order(x.y), score_order(x.z), score_order(x.w));
      } else {
        v = make_uint4(score_order(__ldg(at)), score_order(__ldg(at + 1)), score_order(__ldg(at + 2)), score_order(__ldg(at + 3)));
      }
    }
    return v;
  };
  const int kept = min(early, kHeld);
  uint32_t low = ~0u, high = 0u;
  auto look = [&](const uint4& v, int pos) {
    const uint32_t x[kPer] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (pos + i < early) {
        low = min(low, x[i]);
        high = max(high, x[i]);
      }
  };
  uint4* held4 = reinterpret_cast<uint4*>(held);
  for (int p0 = kPer * tid; p0 < kept; p0 += 4 * kStrip) {
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = p0 + i * kStrip < kept ? read(p0 + i * kStrip) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p0 + i * kStrip < kept) {
        held4[(p0 + i * kStrip) / kPer] = v[i];
        look(v[i], p0 + i * kStrip);
      }
  }
  for (int p = kHeld + kPer * tid; p < early; p += kStrip) look(read(p), p);
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  if (tid == 0) s_low = ~0u, s_high = 0u;
  __syncthreads();
  if (lane == 0) {
    atomicMin(&s_low, low);
    atomicMax(&s_high, high);
  }
  __syncthreads();
  low = s_low;
  // The smallest that stays, less the smallest of all, and how many equal to it do.  Digits of the difference: those of the
  // numbers themselves would be few in the first round (the exponents' upper bits), and the counts would wait for one another.
  const int width = s_high > low ? 32 - __clz(s_high - low) : 0;
  uint32_t least = 0;
  int left = want;
  for (int above = width; above > 0;) {
    const int shift = max(0, above - 8);
    const uint32_t digits = (1u << (above - shift)) - 1u, prefix = above < 32 ? least >> above : 0u;
    if (tid < 256) histogram[tid] = 0;
    __syncthreads();
    auto count = [&](const uint4& v, int pos) {
      const uint32_t x[kPer] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const uint32_t d = x[i] - low;
        if (pos + i < early && (above < 32 ? d >> above : 0u) == prefix) atomicAdd(histogram + (d >> shift & digits), 1);
      }
    };
    for (int p = kPer * tid; p < kept; p += kStrip) count(held4[p / kPer], p);
    for (int p = kHeld + kPer * tid; p < early; p += kStrip) count(read(p), p);
    __syncthreads();
    if (warp == 0) {  // lane i: the digits from 255 - 8 i down
      int own = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) own += histogram[255 - 8 * lane - i];
      int sum = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int other = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += other;
      }
      // the lane in whose digits the count reaches `left` (there are more than `left` in all)
      const unsigned reach = __ballot_sync(0xffffffffu, sum >= left);
      if (reach && lane == __ffs(reach) - 1) {
        int above = sum - own, i = 0;
        while (i < 7 && above + histogram[255 - 8 * lane - i] < left) above += histogram[255 - 8 * lane - i++];
        s_digit = 255 - 8 * lane - i;
        s_left = left - above;
      }
    }
    __syncthreads();
    least |= (uint32_t)s_digit << shift;
    left = s_left;
    above = shift;
  }
  least += low;
  // Those above `least`, and the first `left` equal to it, in order of their positions.
  int above0 = 0, equal0 = 0;  // in the strips before
  for (int p0 = 0; p0 < early; p0 += kStrip) {
    const int p = p0 + kPer * tid;
    const uint4 v4 = p < kept ? held4[p / kPer] : (p < early ? read(p) : make_uint4(0u, 0u, 0u, 0u));
    const uint32_t v[kPer] = {v4.x, v4.y, v4.z, v4.w};
    int packed = 0;  // those above in the low half, those equal in the high one (a strip has 4096)
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (p + i < early) packed += v[i] > least ? 1 : (v[i] == least ? 1 << 16 : 0);
    int sum = packed;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int other = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += other;
    }
    if (lane == 31) warp_sums[warp] = sum;
    __syncthreads();
    const int other = warp_sums[lane];
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? other : 0) + sum - packed;
    const int total = __reduce_add_sync(0xffffffffu, other);
    __syncthreads();
    int above = above0 + (before & 0xffff), equal = equal0 + (before >> 16);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (p + i >= early) break;
      if (v[i] > least) {
        list[above + min(equal, left)] = p + i;
        ++above;
      } else if (v[i] == least) {
        if (equal < left) list[above + equal] = p + i;
        ++equal;
      }
    }
    above0 += total & 0xffff;
    equal0 += total >> 16;
  }
}

// W bytes of each vector a block, 16 a thread.  blockIdx.x: the part of the vector (K's, then V's, then the scores and scales),
// and of the tokens (into other pages only); blockIdx.y: key head; blockIdx.z: sequence.
template <int ROW, int W, int THREADS>  // bytes of a vector
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : 5) evict_move_kernel(const EvictArgs a, int shares) {
  constexpr int SLICES = ROW / W;
  const int part = blockIdx.x / shares, share = blockIdx.x % shares, h = blockIdx.y, b = blockIdx.z;
  pdl_wait();
  const int moves = a.plan[kPlan * b], len = a.plan[kPlan * b + 1], before = a.plan[kPlan * b + 2];
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) a.out_len[b] = len;
  const int want = a.keep - a.recent;
  const bool over = before > a.keep;  // (else all of them move, to the same positions elsewhere)
  const int* list = a.list + ((int64_t)b * a.cache.heads + h) * a.chosen;
  // (a plain load: the kernel before, beside which this one began, wrote it, and __ldg is for what nobody writes meanwhile)
  auto source = [&](int i) { return !over ? i : (i < want ? list[i] : before - a.keep + i); };
  auto slot_of = [&](const int* table, int pos) -> int {  // (a pool has fewer than 2^31)
    const int page = __ldg(table + b * a.batch.max_pages + (pos >> a.cache.page_shift));
    if ((unsigned)page >= (unsigned)a.cache.pages) {
      atomicOr(a.batch.status, kStatusIndex);
      return -1;
    }
    return (int)paged_slot(a.cache, page, h, pos);
  };
  const int* to_table = a.out_table ? a.out_table : a.batch.table;
  const int first = (int)((int64_t)moves * share / shares), last = (int)((int64_t)moves * (share + 1) / shares);
  if (part < 2 * SLICES) {
    constexpr int LANES = W / 16, ROWS = THREADS / LANES, U = 4;
    char* base = static_cast<char*>(part < SLICES ? a.cache.k : a.cache.v) + part % SLICES * W + threadIdx.x % LANES * 16;
    const int row = threadIdx.x / LANES;
    int from[U], to[U], next_from[U], next_to[U];
    auto places = [&](int i0, int (&f)[U], int (&g)[U]) {  // of a trip's tokens
      int pos[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * ROWS + row;
        f[u] = g[u] = -1;
        pos[u] = i < last ? source(i) : i;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * ROWS + row;
        if (i >= last || (pos[u] == i && !a.out_table)) continue;
        f[u] = slot_of(a.batch.table, pos[u]);
        g[u] = slot_of(to_table, i);
      }
    };
    places(first, from, to);
    for (int i0 = first; i0 < last; i0 += ROWS * U) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (from[u] >= 0 && to[u] >= 0) v[u] = *reinterpret_cast<const uint4*>(base + (int64_t)from[u] * ROW);
      places(i0 + ROWS * U, next_from, next_to);  // while the vectors are on their way
      if (!a.out_table) __syncthreads();
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (from[u] >= 0 && to[u] >= 0) *reinterpret_cast<uint4*>(base + (int64_t)to[u] * ROW) = v[u];
        from[u] = next_from[u];
        to[u] = next_to[u];
      }
    }
  } else {
    constexpr int U = 4;
    for (int i0 = first; i0 < last; i0 += THREADS * U) {
      int from[U], to[U];
      float v[U], k[U], w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * THREADS + threadIdx.x;
        from[u] = to[u] = -1;
        if (i >= last) continue;
        const int pos = source(i);
        if (pos == i && !a.out_table) continue;
        from[u] = slot_of(a.batch.table, pos);
        to[u] = slot_of(to_table, i);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (from[u] < 0 || to[u] < 0) continue;
        v[u] = a.score[from[u]];
        if (a.cache.k_scale) {
          k[u] = a.cache.k_scale[from[u]];
          w[u] = a.cache.v_scale[from[u]];
        }
      }
      if (!a.out_table) __syncthreads();
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (from[u] < 0 || to[u] < 0) continue;
        a.score[to[u]] = v[u];
        if (a.cache.k_scale) {
          a.cache.k_scale[to[u]] = k[u];
          a.cache.v_scale[to[u]] = w[u];
        }
      }
    }
  }
}

template <int ROW>
spl_status launch_move(const EvictArgs& a, int blocks, cudaStream_t stream) {
  // Whole vectors where there are blocks enough, else 32 bytes of each; blocks of 1024 threads, of fewer and longer trips, where
  // there are few even then and they go through their tokens one trip after another (one sequence cut in place from 16000
  // tokens to 12000: 77 us with blocks of 256, 50 so; 32 sequences into other pages: 273 us in columns of 128 bytes, 229 whole).
  const int64_t heads = a.cache.heads, seqs = a.batch.seqs;
  const bool wide = heads * seqs * 2 >= 2 * blocks;
  const int parts = wide ? 3 : 2 * ROW / 32 + 1;
  const bool large = !wide && !a.out_table && parts * heads * seqs <= 2 * blocks;
  int shares = 1;  // of a head's tokens, where their order does not matter
  if (a.out_table) shares = (int)std::max<int64_t>(1, std::min<int64_t>(4 * blocks / (parts * heads * seqs), 64));
  const dim3 grid(parts * shares, (unsigned)heads, (unsigned)seqs);
  if (large) return launch_pdl(evict_move_kernel<ROW, 32, 1024>, grid, dim3(1024), 0, stream, a, shares);
  return launch_pdl(wide ? evict_move_kernel<ROW, ROW, 256> : evict_move_kernel<ROW, 32, 256>, grid, dim3(256), 0, stream, a,
                    shares);
}

// ---- an accepted path ----
struct PathArgs {
  PagedCache cache;
  PagedBatch batch;
  float* score;  // or null
  const int *path, *accepted;
  int64_t ldpath;
  int levels;
};
constexpr int kPathThreads = 256, kPathBatch = 4;

// A sequence's places, T a thread's part of each: the nodes path[0] < path[1] < ... of its rows to those from 1 on.  A node
// lies at or behind its place, so moving them in order overwrites no later one's source.
template <class T, class At>
__device__ void move_path(const PathArgs& a, const PagedSeq& s, int b, int count, At at) {
  // Plain loads, of what kernels before may have written beside this one's start; a batch's side by side.
  const int *path = a.path + b * a.ldpath, *table = a.batch.table + b * a.batch.max_pages;
  const int shift = a.cache.page_shift, pages = a.cache.pages;
  int last = 0;  // the node before
  bool bad = false;
  for (int i0 = 0; i0 < count; i0 += kPathBatch) {
    int node[kPathBatch], place[kPathBatch], from_page[kPathBatch], to_page[kPathBatch];
#pragma unroll
    for (int i = 0; i < kPathBatch; ++i) node[i] = i0 + i < count ? path[i0 + i] : 0;
#pragma unroll
    for (int i = 0; i < kPathBatch; ++i) {
      place[i] = -1;
      if (i0 + i >= count) continue;
      if (node[i] <= last || node[i] >= s.n) {  // not a path: what follows stays where it is
        bad = true;
        count = i0 + i;
        continue;
      }
      last = node[i];
      if (node[i] != 1 + i0 + i && s.pos0 + node[i] < s.len) place[i] = s.pos0 + 1 + i0 + i;  // (or no place in the table, or -1)
    }
#pragma unroll
    for (int i = 0; i < kPathBatch; ++i) {
      from_page[i] = place[i] >= 0 ? table[(s.pos0 + node[i]) >> shift] : 0;
      to_page[i] = place[i] >= 0 ? table[place[i] >> shift] : 0;
    }
    T v[kPathBatch] = {};
    T* to[kPathBatch];
#pragma unroll
    for (int i = 0; i < kPathBatch; ++i) {
      to[i] = nullptr;
      if (place[i] < 0) continue;
      if ((unsigned)from_page[i] >= (unsigned)pages || (unsigned)to_page[i] >= (unsigned)pages) {
        bad = true;
        continue;
      }
      v[i] = *at(from_page[i], s.pos0 + node[i]);
      to[i] = at(to_page[i], place[i]);
    }
#pragma unroll
    for (int i = 0; i < kPathBatch; ++i)
      if (to[i]) *to[i] = v[i];
  }
  if (bad) atomicOr(a.batch.status, kStatusIndex);
}

template <int ROW>
__global__ void __launch_bounds__(kPathThreads) keep_path_kernel(const PathArgs a) {
  constexpr int LANES = ROW / 16;
  pdl_wait();
  const int b = blockIdx.y, heads = a.cache.heads;
  int count = a.accepted[b];
  const PagedSeq s = paged_seq<true>(a.batch, a.cache.page_shift, b);
  if (count < 0 || count > a.levels) {
    atomicOr(a.batch.status, kStatusIndex);
    count = 0;
  }
  const int64_t vectors = (int64_t)2 * heads * LANES;
  int64_t task = (int64_t)blockIdx.x * kPathThreads + threadIdx.x;
  if (task < vectors) {
    const int part = (int)(task % LANES), h = (int)(task / LANES % heads);
    char* base = static_cast<char*>(task < vectors / 2 ? a.cache.k : a.cache.v) + 16 * part;
    move_path<uint4>(a, s, b, count, [&](int page, int pos) {
      return reinterpret_cast<uint4*>(base + paged_slot(a.cache, page, h, pos) * ROW);
    });
    return;
  }
  task -= vectors;
  float* of[3] = {a.score, a.cache.k_scale, a.cache.v_scale};
  if (task >= 3 * heads || !of[task / heads]) return;
  move_path<float>(a, s, b, count, [&](int page, int pos) {
    return of[task / heads] + paged_slot(a.cache, page, (int)(task % heads), pos);
  });
}

// The tokens that a page table has room for.
int64_t room_of(const PagedCache& c, const PagedBatch& b) { return b.max_pages << c.page_shift; }
size_t chosen_of(const PagedCache& c, const PagedBatch& b, int64_t keep) {
  return (size_t)std::min(keep, room_of(c, b)) * c.heads * b.seqs;
}
size_t evict_bytes(const PagedCache& c, const PagedBatch& b, int64_t keep) {
  return kCounterBytes + round_up((int64_t)b.seqs * kPlan * sizeof(int), 16) + chosen_of(c, b, keep) * sizeof(int);
}

}  // namespace
}  // namespace spl

using namespace spl;

extern "C" size_t spl_kv_evict_workspace_bytes(const spl_kv_cache* cache, const spl_kv_batch* batch, int64_t keep) {
  PagedCache c;
  PagedBatch b;
  if (paged_cache_view(&c, cache) != SPL_OK || paged_batch_view(&b, c, batch, 0) != SPL_OK || keep < 0 || b.seqs == 0)
    return 0;
  return evict_bytes(c, b, keep);
}

extern "C" spl_status spl_kv_evict(const spl_kv_cache* cache, float* score, const spl_kv_batch* batch, int64_t keep,
                                   int64_t recent, const int32_t* out_table, int32_t* out_len, void* workspace,
                                   size_t workspace_bytes, cudaStream_t stream) {
  EvictArgs a = {};
  spl_status st = paged_cache_view(&a.cache, cache);
  if (st != SPL_OK) return st;
  if ((st = paged_batch_view(&a.batch, a.cache, batch, 0)) != SPL_OK) return st;
  if (keep < 0 || recent < 0 || recent > keep) return SPL_EINVAL;
  if (a.batch.seqs == 0) return SPL_OK;
  if (!out_len || (a.cache.pages > 0 && !score)) return SPL_EINVAL;
  if (!aligned4(score) || !aligned4(out_table) || !aligned4(out_len)) return SPL_EALIGN;
  if (!workspace || workspace_bytes < evict_bytes(a.cache, a.batch, keep)) return SPL_EWORKSPACE;
  if (!aligned16(workspace)) return SPL_EALIGN;
  if (!(a.batch.status = device_status_word())) return SPL_ECUDA;
  const bool i8 = cache->format == SPL_KV_I8;
  if (!i8) a.cache.k_scale = a.cache.v_scale = nullptr;
  a.score = score;
  a.out_table = out_table == batch->page_table ? nullptr : out_table;
  a.out_len = out_len;
  a.keep = (int)std::min(keep, kMaxLength);
  a.recent = (int)std::min(recent, kMaxLength);
  a.chosen = std::min(keep, room_of(a.cache, a.batch));
  a.plan = reinterpret_cast<int*>(static_cast<char*>(workspace) + kCounterBytes);  // (the counters are others')
  a.list = a.plan + round_up((int64_t)a.batch.seqs * kPlan, 4);
  const size_t held = (size_t)std::min<int64_t>(kHeld, room_of(a.cache, a.batch)) * sizeof(uint32_t);  // (room: whole pages)
  static bool done[kMaxDevices] = {false};
  if (!allow_shared(reinterpret_cast<const void*>(evict_select_kernel), kHeld * sizeof(uint32_t), done)) return SPL_ECUDA;
  evict_select_kernel<<<dim3(a.cache.heads, a.batch.seqs), kSelectThreads, held, stream>>>(a);
  if ((st = launch_status()) != SPL_OK) return st;
  const int sms = device_sm_count(), row = (int)cache->head_dim * (i8 ? 1 : 2);
  return row == 256 ? launch_move<256>(a, sms, stream)
                    : (row == 128 ? launch_move<128>(a, sms, stream) : launch_move<64>(a, sms, stream));
}

extern "C" spl_status spl_kv_keep_path(const spl_kv_cache* cache, float* score, const spl_kv_batch* batch, int64_t rows,
                                       const int32_t* path, int64_t ldpath, const int32_t* accepted, int64_t levels,
                                       cudaStream_t stream) {
  PathArgs a = {};
  spl_status st = paged_cache_view(&a.cache, cache);
  if (st != SPL_OK) return st;
  if (levels < 0 || ldpath < 0) return SPL_EINVAL;
  if ((st = paged_batch_view(&a.batch, a.cache, batch, rows)) != SPL_OK) return st;
  if (a.batch.seqs == 0 || levels == 0 || rows == 0) return SPL_OK;
  if (!path || !accepted || (a.batch.seqs > 1 && ldpath < levels)) return SPL_EINVAL;
  if (levels > INT32_MAX) return SPL_ESHAPE;
  if (!aligned4(score) || !aligned4(path) || !aligned4(accepted)) return SPL_EALIGN;
  if (a.batch.max_pages == 0 || a.cache.pages == 0) return SPL_OK;
  if (!(a.batch.status = device_status_word())) return SPL_ECUDA;
  const bool i8 = cache->format == SPL_KV_I8;
  if (!i8) a.cache.k_scale = a.cache.v_scale = nullptr;
  a.score = score;
  a.path = path;
  a.accepted = accepted;
  a.ldpath = ldpath;
  a.levels = (int)levels;
  const int row = (int)cache->head_dim * (i8 ? 1 : 2);
  const int64_t tasks = (int64_t)a.cache.heads * (2 * row / 16 + 3);
  const dim3 grid((unsigned)ceil_div(tasks, kPathThreads), a.batch.seqs);
  return launch_pdl(row == 256 ? keep_path_kernel<256> : (row == 128 ? keep_path_kernel<128> : keep_path_kernel<64>), grid,
                    dim3(kPathThreads), 0, stream, a);
}
