// The paged KV cache: keys and values written as they are made, in 16 bits or quantised to 8, and read back.
//
// Stored vectors are [pages, heads, page, dim]: the tokens of one head in one page are contiguous, so attention of
// one head streams whole blocks.  Formats:
//   F16  fp16(x), rounded to nearest, finite and infinite values beyond +-65504 saturated
//   I8   per token and head s = fl(max|x| / 127), code = rint(fl(x / s)) in [-127, 127], read back as fl(code s);
//        a vector of zeros has s = 0 and codes 0; one with an infinity or NaN has s = NaN and codes 0 (it reads back
//        as NaN, and the codes stay finite)
// Both kernels move each byte once and are bound by HBM, or by their latency for few rows.  One warp takes the heads
// of one row of K or of V, kHeadsInFlight at a time, a lane four neighbours of the vector: the loads of a row are
// whole 512-byte vectors and those of several heads are in flight together.  Measured with 8 heads of 128 dims: 64000
// tokens written and read 116, 117 us as binary16 (6.8 TB/s, the rate of a copy), 103, 100 us as int8 (6.4, 6.6 TB/s);
// one token 2.0 us and 2.7 us (int8), a launch and three dependent loads.

#include <algorithm>

#include <cuda_fp16.h>

#include "paged.cuh"

namespace spl {
namespace {

constexpr int kThreads = 256;
constexpr int kHeadsInFlight = 8;

__device__ __forceinline__ uint32_t f16x2_sat(float a, float b) {
  uint32_t r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

template <int D, bool I8>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const PagedCache cache, const PagedBatch batch, const float* __restrict__ K,
                 const float* __restrict__ V, int64_t ldk, int64_t ldv) {
  constexpr int LANES = D / 4, PER_WARP = 32 / LANES;  // lanes of a vector, vectors of a warp
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31, part = lane / LANES, at = lane % LANES;
  const int64_t row = w >> 1;
  if (row >= batch.rows) return;
  const bool is_v = w & 1;
  const float* src = is_v ? V + row * ldv : K + row * ldk;
  float4 x[kHeadsInFlight];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < kHeadsInFlight; ++u) {
      const int h = h0 + u * PER_WARP + part;
      x[u] = h < cache.heads ? __ldcs(reinterpret_cast<const float4*>(src + (int64_t)h * D) + at)
                             : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  load(0);  // on its way while the row's place is looked up
  const int b = paged_find(batch.row_start, batch.seqs, row);
  const PagedSeq s = paged_seq(batch, cache.page_shift, b);
  const int64_t i = row - s.row0;
  const int64_t pos = s.pos0 + i;
  if (i < 0 || i >= s.n || pos < 0 || pos >= s.len) return;  // no sequence's row, or without a place in its table
  const int page = paged_page(cache, batch, b, (int)pos);
  if (page < 0) return;
  void* dst = is_v ? cache.v : cache.k;
  float* scales = is_v ? cache.v_scale : cache.k_scale;
  for (int h0 = 0; h0 < cache.heads; h0 += kHeadsInFlight * PER_WARP) {
    if (h0 > 0) load(h0);
#pragma unroll
    for (int u = 0; u < kHeadsInFlight; ++u) {
      const int h = h0 + u * PER_WARP + part;
      if (h0 + u * PER_WARP >= cache.heads) break;
      const int64_t slot = paged_slot(cache, page, h < cache.heads ? h : 0, (int)pos);
      if constexpr (I8) {
        // |x| as bits orders like |x|, with infinities and NaN on top
        uint32_t top = max(max(__float_as_uint(x[u].x) & 0x7fffffffu, __float_as_uint(x[u].y) & 0x7fffffffu),
                           max(__float_as_uint(x[u].z) & 0x7fffffffu, __float_as_uint(x[u].w) & 0x7fffffffu));
        if constexpr (LANES == 32) {
          top = __reduce_max_sync(0xffffffffu, top);
        } else {
#pragma unroll
          for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        }
        const bool finite = top < 0x7f800000u;
        const float scale = finite ? __fdiv_rn(__uint_as_float(top), 127.0f) : __uint_as_float(0x7fc00000u);
        // rint(x / s) by a product with 1 / s, within 2^-14 of the quotient; where that is closer than 2^-13 to the middle
        // of two codes, or 1 / s is out of range, by the division itself (some 3% of the warps; dividing always was bound
        // by arithmetic, 149 us for 64000 tokens of 8 heads of 128 instead of 103).
        const float magic = 12582912.0f;  // 1.5 2^23: x + magic holds rint(x) in its low bits
        float inverse;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(scale));
        const float q[4] = {x[u].x * inverse, x[u].y * inverse, x[u].z * inverse, x[u].w * inverse};
        float t[4], off = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          t[k] = __fadd_rn(q[k], magic);
          off = fmaxf(off, fabsf(__fsub_rn(q[k], __fsub_rn(t[k], magic))));
        }
        uint32_t c = __byte_perm(__byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040u),
                                 __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040u), 0x5410u);
        if (!(off < 0.5f - 0x1p-13f) || !(scale > 0x1p-100f && scale < 0x1p100f)) {
          auto code = [&](float v) {
            if (!(scale > 0.0f)) return 0;
            return max(-127, min(127, __float2int_rn(__fdiv_rn(v, scale))));
          };
          c = (uint32_t)(code(x[u].x) & 255) | (uint32_t)(code(x[u].y) & 255) << 8 |
              (uint32_t)(code(x[u].z) & 255) << 16 | (uint32_t)(code(x[u].w) & 255) << 24;
        }
        if (h < cache.heads) {
          *reinterpret_cast<uint32_t*>(static_cast<int8_t*>(dst) + slot * D + 4 * at) = c;
          if (at == 0) scales[slot] = scale;
        }
      } else if (h < cache.heads) {
        const uint2 c = make_uint2(f16x2_sat(x[u].x, x[u].y), f16x2_sat(x[u].z, x[u].w));
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(dst) + slot * D + 4 * at) = c;
      }
    }
  }
}

template <int D, bool I8>
__global__ void __launch_bounds__(kThreads)
kv_read_kernel(float* __restrict__ K, float* __restrict__ V, const PagedCache cache, const PagedBatch batch,
               const int* __restrict__ out_start, int64_t out_rows) {
  constexpr int LANES = D / 4, PER_WARP = 32 / LANES;
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31, part = lane / LANES, at = lane % LANES;
  const int64_t row = w >> 1;
  if (row >= out_rows) return;
  const int b = paged_find(out_start, batch.seqs, row);
  const int64_t pos = row - __ldg(out_start + b);
  const PagedSeq s = paged_seq(batch, cache.page_shift, b);
  if (pos < 0 || pos >= s.len || row >= __ldg(out_start + b + 1)) return;  // no stored token's row
  const int page = paged_page(cache, batch, b, (int)pos);
  if (page < 0) return;
  const bool is_v = w & 1;
  float* dst = (is_v ? V : K) + row * (int64_t)cache.heads * D;
  const void* src = is_v ? cache.v : cache.k;
  const float* scales = is_v ? cache.v_scale : cache.k_scale;
  for (int h0 = 0; h0 < cache.heads; h0 += kHeadsInFlight * PER_WARP) {
    uint2 c[kHeadsInFlight];
    float scale[kHeadsInFlight];
#pragma unroll
    for (int u = 0; u < kHeadsInFlight; ++u) {
      const int h = h0 + u * PER_WARP + part;
      c[u] = make_uint2(0u, 0u);
      scale[u] = 0.f;
      if (h >= cache.heads) continue;
      const int64_t slot = paged_slot(cache, page, h, (int)pos);
      if constexpr (I8) {
        c[u].x = __ldcs(reinterpret_cast<const uint32_t*>(static_cast<const int8_t*>(src) + slot * D) + at);
        scale[u] = __ldg(scales + slot);
      } else {
        c[u] = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(src) + slot * D) + at);
      }
    }
#pragma unroll
    for (int u = 0; u < kHeadsInFlight; ++u) {
      const int h = h0 + u * PER_WARP + part;
      if (h >= cache.heads) continue;
      float4 x;
      if constexpr (I8) {
        x = make_float4(__fmul_rn((float)(int8_t)(c[u].x), scale[u]), __fmul_rn((float)(int8_t)(c[u].x >> 8), scale[u]),
                        __fmul_rn((float)(int8_t)(c[u].x >> 16), scale[u]),
                        __fmul_rn((float)(int8_t)(c[u].x >> 24), scale[u]));
      } else {
        const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&c[u].x));
        const float2 hi = __half22float2(*reinterpret_cast<const __half2*>(&c[u].y));
        x = make_float4(lo.x, lo.y, hi.x, hi.y);
      }
      __stcs(reinterpret_cast<float4*>(dst + (int64_t)h * D) + at, x);
    }
  }
}

unsigned blocks_of(int64_t rows) { return (unsigned)ceil_div(2 * rows * 32, kThreads); }

}  // namespace

spl_status paged_cache_view(PagedCache* out, const spl_kv_cache* c) {
  if (!c) return SPL_EINVAL;
  if (c->format != SPL_KV_F16 && c->format != SPL_KV_I8) return SPL_EINVAL;
  if (c->pages < 0 || c->kv_heads < 1 || c->page_size < 1 || c->head_dim < 1) return SPL_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return SPL_ESHAPE;
  int shift = 4;
  while (shift < 8 && (int64_t(1) << shift) != c->page_size) ++shift;
  if ((int64_t(1) << shift) != c->page_size) return SPL_ESHAPE;
  if (c->pages > INT32_MAX || c->kv_heads > 1024) return SPL_ESHAPE;
  if (c->pages * c->kv_heads * c->page_size > INT32_MAX - 1024) return SPL_ESHAPE;  // rows of a copy's coordinates
  const bool i8 = c->format == SPL_KV_I8;
  if (c->pages > 0 && (!c->k || !c->v || (i8 && (!c->k_scale || !c->v_scale)))) return SPL_EINVAL;
  if (!aligned16(c->k) || !aligned16(c->v) || (i8 && (!aligned16(c->k_scale) || !aligned16(c->v_scale))))
    return SPL_EALIGN;
  *out = {c->k, c->v, c->k_scale, c->v_scale, (int)c->pages, (int)c->kv_heads, shift};
  return SPL_OK;
}

spl_status paged_batch_view(PagedBatch* out, const PagedCache& cache, const spl_kv_batch* b, int64_t rows) {
  if (!b || b->seqs < 0 || b->max_pages < 0 || b->max_rows < 0 || rows < 0) return SPL_EINVAL;
  if (b->seqs > kMaxSeqs || rows > INT32_MAX || b->max_pages > INT32_MAX) return SPL_ESHAPE;
  if (b->max_pages << cache.page_shift > kMaxLength) return SPL_ESHAPE;
  if (b->seqs > 0 && (!b->row_start || !b->kv_len || (b->max_pages > 0 && !b->page_table))) return SPL_EINVAL;
  if (!aligned4(b->row_start) || !aligned4(b->kv_len) || !aligned4(b->page_table)) return SPL_EALIGN;
  *out = {b->row_start, b->kv_len, b->page_table, (int)b->seqs, b->max_pages, rows, nullptr};
  return SPL_OK;
}

}  // namespace spl

using namespace spl;

extern "C" spl_status spl_kv_append(const spl_kv_cache* cache, const spl_kv_batch* batch, const float* K, int64_t ldk,
                                    const float* V, int64_t ldv, int64_t rows, cudaStream_t stream) {
  PagedCache c;
  PagedBatch b;
  spl_status st = paged_cache_view(&c, cache);
  if (st != SPL_OK) return st;
  const int64_t width = cache->kv_heads * cache->head_dim;
  if (!batch || rows < 0 || ldk < 0 || ldv < 0) return SPL_EINVAL;
  if (rows > 0 && batch->seqs > 0 && (!K || !V)) return SPL_EINVAL;
  if (rows > 1 && (ldk < width || ldv < width)) return SPL_EINVAL;
  if (!aligned16(K) || !aligned16(V) || (rows > 1 && (ldk % 4 != 0 || ldv % 4 != 0))) return SPL_EALIGN;
  if ((st = paged_batch_view(&b, c, batch, rows)) != SPL_OK) return st;
  if (rows == 0 || b.seqs == 0 || b.max_pages == 0 || c.pages == 0) return SPL_OK;
  if (!(b.status = device_status_word())) return SPL_ECUDA;
  auto launch = [&](auto kernel) {
    kernel<<<blocks_of(rows), kThreads, 0, stream>>>(c, b, K, V, ldk, ldv);
    return launch_status();
  };
  const bool i8 = cache->format == SPL_KV_I8;
  if (cache->head_dim == 128) return i8 ? launch(kv_append_kernel<128, true>) : launch(kv_append_kernel<128, false>);
  return i8 ? launch(kv_append_kernel<64, true>) : launch(kv_append_kernel<64, false>);
}

extern "C" spl_status spl_kv_read(float* K, float* V, const spl_kv_cache* cache, const spl_kv_batch* batch,
                                  const int32_t* out_start, int64_t out_rows, cudaStream_t stream) {
  PagedCache c;
  PagedBatch b;
  spl_status st = paged_cache_view(&c, cache);
  if (st != SPL_OK) return st;
  if (!batch || out_rows < 0) return SPL_EINVAL;
  if (out_rows > 0 && batch->seqs > 0 && (!K || !V || !out_start)) return SPL_EINVAL;
  if (out_rows > INT32_MAX) return SPL_ESHAPE;
  if (!aligned16(K) || !aligned16(V) || !aligned4(out_start)) return SPL_EALIGN;
  if ((st = paged_batch_view(&b, c, batch, INT32_MAX)) != SPL_OK) return st;
  if (out_rows == 0 || b.seqs == 0 || b.max_pages == 0 || c.pages == 0) return SPL_OK;
  if (!(b.status = device_status_word())) return SPL_ECUDA;
  auto launch = [&](auto kernel) {
    kernel<<<blocks_of(out_rows), kThreads, 0, stream>>>(K, V, c, b, out_start, out_rows);
    return launch_status();
  };
  const bool i8 = cache->format == SPL_KV_I8;
  if (cache->head_dim == 128) return i8 ? launch(kv_read_kernel<128, true>) : launch(kv_read_kernel<128, false>);
  return i8 ? launch(kv_read_kernel<64, true>) : launch(kv_read_kernel<64, false>);
}
