// The paged KV cache as the kernels see it, and the launchers of its operators.
#pragma once

#include "sl_common.h"

namespace sl {

// n / d for 0 <= n < 2^31 without a division: with s = ceil(log2 d) and m = ceil(2^(31+s) / d),
// m * d - 2^(31+s) < 2^s, so that n * m / 2^(31+s) has the quotient as its whole part.
struct FastDiv {
  uint32_t d, m, s;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while (((uint64_t)1 << s) < d) ++s;
  return {d, (uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d), s};
}

// Host-side, validated view of sl_page_cache with defaults resolved.
struct PageCache {
  void *K, *V;
  int32_t *tables, *lens, *refs;
  int64_t layer, page, head, tok;  // strides in elements; of a cache in 4 bits in bytes, tok of its codes
  int layers, n_pages, n_seqs, max_pages, ps, Hkv, D, dtype;  // dtype: of the rows
  FastDiv by_ps;
  bool fp4;  // a head's part of a page: ps rows of D / 2 bytes of codes, then ps of D / 32 scales (fp4.h)
};

struct PagedBatch {
  const int32_t *seqs, *cu;
  int B, rows, layer;
  int L;  // positions lie below
};

struct PagedAttention {
  int Hq, G, S, topk;
  float scale;
  int64_t qsh, qst, ish, ist;
  bool combined;
};

sl_status pages_extend(const PageCache& c, const PagedBatch& b, int32_t* ok, hipStream_t st);
sl_status pages_served(const int32_t* seqs, const int32_t* ok, int n, int32_t* served, hipStream_t st);
sl_status pages_fork(const PageCache& c, const int32_t* src, const int32_t* dst, int n, int32_t* ok, hipStream_t st);
sl_status pages_free(const PageCache& c, const int32_t* seqs, int n, hipStream_t st);
size_t pages_compact_ws_bytes(const PageCache& c);
sl_status pages_compact(const PageCache& c, int32_t* map, void* ws, hipStream_t st);
sl_status paged_append(const PageCache& c, const PagedBatch& b, const void* K, const void* V, int64_t sh, int64_t st_, hipStream_t st);
sl_status paged_append_fp4(const PageCache& c, const PagedBatch& b, const void* K, const void* V, int64_t sh, int64_t st_, hipStream_t st);
sl_status paged_read(const PageCache& c, const PagedBatch& b, void* K, void* V, int64_t sh, int64_t st_, hipStream_t st);
sl_status paged_span_keys(const PageCache& c, const PagedBatch& b, int S, int n_spans, void* Ks, hipStream_t st);
sl_status paged_span_keys_fp4(const PageCache& c, const PagedBatch& b, int S, int n_spans, void* Ks, hipStream_t st);
size_t paged_attention_ws_bytes(const PageCache& c, const PagedBatch& b, const PagedAttention& a);
sl_status paged_attention(const PageCache& c, const PagedBatch& b, const PagedAttention& a, const void* Q, const int32_t* idx,
                          const float* scores, void* O, float* LSE, void* ws, hipStream_t st);
sl_status paged_attention_fp4(const PageCache& c, const PagedBatch& b, const PagedAttention& a, const void* Q, const int32_t* idx,
                              const float* scores, void* O, float* LSE, void* ws, hipStream_t st);

#if defined(__HIPCC__)

__host__ __device__ __forceinline__ uint32_t operator/(uint32_t n, const FastDiv& f) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __umulhi(2 * n, f.m) >> f.s;
#else
  return (uint32_t)(((uint64_t)n * f.m) >> (31 + f.s));
#endif
}

// The entry whose rows hold row r, cu[0] <= r < cu[B]: the last b with cu[b] <= r.
__device__ __forceinline__ int entry_of_row(const int32_t* __restrict__ cu, int B, int r) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A sequence's length as its table can hold it; -1 for a sequence number out of range.
__device__ __forceinline__ int length_of(const PageCache& c, int s) {
  if ((uint32_t)s >= (uint32_t)c.n_seqs) return -1;
  const int most = c.max_pages * c.ps, len = c.lens[s];
  return len < 0 ? 0 : len < most ? len : most;
}

// Where a batch's row lies: its page and its place there; page < 0: the row is no entry's, holds no token, or its token has no page.
struct RowPlace {
  int page, at;
  bool listed;  // a row of some entry
};
__device__ __forceinline__ RowPlace place_of_row(const PageCache& c, const PagedBatch& b, int row) {
  if (row >= b.rows || row < b.cu[0] || row >= b.cu[b.B]) return {-1, 0, false};
  const int e = entry_of_row(b.cu, b.B, row), s = b.seqs[e], len = length_of(c, s), t = len - (b.cu[e + 1] - row);
  if (t < 0 || t >= b.L || t >= len) return {-1, 0, true};
  const int k = (uint32_t)t / c.by_ps, page = c.tables[(int64_t)s * c.max_pages + k];
  return {(uint32_t)page < (uint32_t)c.n_pages ? page : -1, t - k * c.ps, true};
}

#endif

}  // namespace sl
