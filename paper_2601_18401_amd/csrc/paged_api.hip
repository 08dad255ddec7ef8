// C-ABI layer of the paged cache: argument validation on the host, then dispatch to the launchers.
#include <algorithm>
#include <cmath>

#include "paged.h"

namespace sl {

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

constexpr int64_t kMaxStride = (int64_t)1 << 40;     // elements
constexpr int64_t kMaxExtent = (int64_t)1 << 56;     // ... of the cache: byte offsets stay inside 64 bits
constexpr int32_t kMaxPages = 1 << 30;               // a page's number and a pass of a thousand threads count in 32 bits
constexpr int64_t kMaxTokenStride = (int64_t)1 << 20;
constexpr int64_t kMaxRows = (int64_t)1 << 25;       // 16-byte pieces of a row tensor's head count in 32 bits
constexpr int64_t kMaxRowHeads = (int64_t)1 << 26;   // a row, its head and a slot of 32 count in 31 bits

sl_status make_cache(const sl_page_cache* p, PageCache* c) {
  if (!p || !p->K || !p->V || !p->tables || !p->lens || !p->refs) return SL_ERR_INVALID_ARG;
  if (!aligned16(p->K) || !aligned16(p->V) || !aligned16(p->refs) || !aligned4(p->tables) || !aligned4(p->lens))
    return SL_ERR_INVALID_ARG;
  if (p->layers < 1 || p->n_pages < 1 || p->n_seqs < 1 || p->max_pages < 1 || p->page_size < 1 || p->Hkv < 1) return SL_ERR_INVALID_ARG;
  if (p->dtype != SL_F32 && p->dtype != SL_BF16) return SL_ERR_INVALID_ARG;
  if (p->D != 64 && p->D != 128) return SL_ERR_UNSUPPORTED;
  if ((int64_t)p->max_pages * p->page_size > (int64_t)1 << 30 || p->n_pages > kMaxPages) return SL_ERR_UNSUPPORTED;
  // (grid dimensions are 16 bits wide in y)
  if (p->Hkv > 1024 || p->layers > 4096 || (int64_t)p->layers * 2 * p->Hkv + p->max_pages / 1024 > 65000 || p->max_pages > (1 << 25))
    return SL_ERR_UNSUPPORTED;
  if (p->kv_stride_t < 0 || p->kv_stride_h < 0 || p->page_stride < 0 || p->layer_stride < 0) return SL_ERR_INVALID_ARG;
  if (p->kv_stride_t > kMaxTokenStride || p->kv_stride_h > kMaxStride || p->page_stride > kMaxStride || p->layer_stride > kMaxStride << 8)
    return SL_ERR_UNSUPPORTED;
  c->tok = p->kv_stride_t ? p->kv_stride_t : p->D;
  c->head = p->kv_stride_h ? p->kv_stride_h : p->page_size * c->tok;
  // (heads first or tokens first: whichever is the outer one of the two has the larger extent)
  c->page = p->page_stride ? p->page_stride : std::max(p->Hkv * c->head, p->page_size * c->tok);
  if (c->head > kMaxExtent / p->Hkv || c->page > kMaxExtent / p->n_pages) return SL_ERR_UNSUPPORTED;
  c->layer = p->layer_stride ? p->layer_stride : p->n_pages * c->page;
  if (c->layer > kMaxExtent / p->layers) return SL_ERR_UNSUPPORTED;
  const int64_t epl = p->dtype == SL_BF16 ? 8 : 4;
  if (c->tok % epl || c->head % epl || c->page % epl || c->layer % epl) return SL_ERR_INVALID_ARG;
  if (c->tok < p->D || (p->Hkv > 1 && c->head < p->D) || (p->n_pages > 1 && c->page < p->D) || (p->layers > 1 && c->layer < p->D))
    return SL_ERR_INVALID_ARG;
  c->K = p->K;
  c->V = p->V;
  c->tables = p->tables;
  c->lens = p->lens;
  c->refs = p->refs;
  c->layers = p->layers;
  c->n_pages = p->n_pages;
  c->n_seqs = p->n_seqs;
  c->max_pages = p->max_pages;
  c->ps = p->page_size;
  c->Hkv = p->Hkv;
  c->D = p->D;
  c->dtype = p->dtype;
  c->by_ps = fast_div((uint32_t)p->page_size);
  return SL_OK;
}

sl_status make_batch(const sl_paged_batch* p, const PageCache& c, PagedBatch* b) {
  if (!p || p->B < 0 || p->rows < 0 || p->L < 0) return SL_ERR_INVALID_ARG;
  if (p->B > 65535 || p->rows > kMaxRows) return SL_ERR_UNSUPPORTED;
  if (p->layer < 0 || p->layer >= c.layers) return SL_ERR_INVALID_ARG;
  if (p->B > 0 && (!p->seqs || !p->cu_rows || !aligned4(p->seqs) || !aligned4(p->cu_rows))) return SL_ERR_INVALID_ARG;
  const int64_t most = (int64_t)c.max_pages * c.ps;
  b->seqs = p->seqs;
  b->cu = p->cu_rows;
  b->B = p->B;
  b->rows = (int)p->rows;
  b->layer = p->layer;
  b->L = (int)(p->L == 0 || p->L > most ? most : p->L);
  return SL_OK;
}

sl_status make_attention(const sl_paged_attention* p, const PageCache& c, const PagedBatch& b, PagedAttention* a) {
  if (!p || p->Hq < 1 || p->Hq % c.Hkv != 0 || p->S < 1 || p->topk < 0) return SL_ERR_INVALID_ARG;
  if (!(p->scale >= 0.f) || std::isinf(p->scale)) return SL_ERR_INVALID_ARG;
  if (p->topk > SL_MAX_TOPK || p->Hq / c.Hkv > 64 || p->Hq > 65535) return SL_ERR_UNSUPPORTED;
  if ((int64_t)b.rows * p->Hq >= kMaxRowHeads) return SL_ERR_UNSUPPORTED;
  if (p->q_stride_h < 0 || p->q_stride_t < 0 || p->idx_stride_h < 0 || p->idx_stride_t < 0) return SL_ERR_INVALID_ARG;
  if (p->q_stride_h > kMaxStride || p->q_stride_t > kMaxStride >> 8 || p->idx_stride_h > kMaxStride || p->idx_stride_t > kMaxStride >> 8)
    return SL_ERR_UNSUPPORTED;
  const int64_t epl = c.dtype == SL_BF16 ? 8 : 4;
  a->qst = p->q_stride_t ? p->q_stride_t : c.D;
  a->qsh = p->q_stride_h ? p->q_stride_h : b.rows * a->qst;
  a->ist = p->idx_stride_t ? p->idx_stride_t : p->topk;
  a->ish = p->idx_stride_h ? p->idx_stride_h : b.rows * a->ist;
  if (a->qst < c.D || a->qst % epl || a->qsh % epl) return SL_ERR_INVALID_ARG;
  a->Hq = p->Hq;
  a->G = p->Hq / c.Hkv;
  a->S = p->S;
  a->topk = p->topk;
  a->scale = p->scale > 0.f ? p->scale : 1.0f / std::sqrt((float)c.D);
  a->combined = false;
  return SL_OK;
}

sl_status attention_entry(const sl_page_cache* pc, const sl_paged_batch* pb, const sl_paged_attention* pa, const void* Q,
                          const int32_t* idx, const float* scores, bool combined, void* O, float* LSE, void* ws, size_t ws_bytes,
                          void* stream) {
  PageCache c;
  PagedBatch b;
  PagedAttention a;
  sl_status s = make_cache(pc, &c);
  if (s == SL_OK) s = make_batch(pb, c, &b);
  if (s == SL_OK) s = make_attention(pa, c, b, &a);
  if (s != SL_OK) return s;
  if (b.B == 0 || b.rows == 0) return SL_OK;
  if (!Q || !O || (!combined && !LSE) || (a.topk > 0 && (!idx || (combined && !scores)))) return SL_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(O) || !aligned4(LSE) || !aligned4(idx) || !aligned4(scores)) return SL_ERR_INVALID_ARG;
  a.combined = combined && a.topk > 0;  // (without slots: attention over the window)
  const size_t need = paged_attention_ws_bytes(c, b, a);
  if (need && (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u))) return SL_ERR_WORKSPACE;
  return paged_attention(c, b, a, Q, idx, scores, O, LSE, ws, static_cast<hipStream_t>(stream));
}

}  // namespace

}  // namespace sl

extern "C" {

sl_status sl_pages_extend(const sl_page_cache* pc, const sl_paged_batch* pb, int32_t* ok, void* hip_stream) {
  sl::PageCache c;
  sl::PagedBatch b;
  sl_status s = sl::make_cache(pc, &c);
  if (s == SL_OK) s = sl::make_batch(pb, c, &b);
  if (s != SL_OK) return s;
  if (b.B > SL_MAX_PAGE_OPS) return SL_ERR_UNSUPPORTED;
  if (b.B > 0 && (!ok || !sl::aligned4(ok))) return SL_ERR_INVALID_ARG;
  return sl::pages_extend(c, b, ok, static_cast<hipStream_t>(hip_stream));
}

sl_status sl_pages_served(const int32_t* seqs, const int32_t* ok, int32_t n, int32_t* served, void* hip_stream) {
  if (n < 0 || (n > 0 && (!seqs || !ok || !served || !sl::aligned4(seqs) || !sl::aligned4(ok) || !sl::aligned4(served))))
    return SL_ERR_INVALID_ARG;
  if (n > 65535) return SL_ERR_UNSUPPORTED;
  return sl::pages_served(seqs, ok, n, served, static_cast<hipStream_t>(hip_stream));
}

sl_status sl_pages_fork(const sl_page_cache* pc, const int32_t* src, const int32_t* dst, int32_t n, int32_t* ok, void* hip_stream) {
  sl::PageCache c;
  sl_status s = sl::make_cache(pc, &c);
  if (s != SL_OK) return s;
  if (n < 0 || (n > 0 && (!src || !dst || !ok || !sl::aligned4(src) || !sl::aligned4(dst) || !sl::aligned4(ok)))) return SL_ERR_INVALID_ARG;
  if (n > SL_MAX_PAGE_OPS) return SL_ERR_UNSUPPORTED;
  return sl::pages_fork(c, src, dst, n, ok, static_cast<hipStream_t>(hip_stream));
}

sl_status sl_pages_free(const sl_page_cache* pc, const int32_t* seqs, int32_t n, void* hip_stream) {
  sl::PageCache c;
  sl_status s = sl::make_cache(pc, &c);
  if (s != SL_OK) return s;
  if (n < 0 || (n > 0 && (!seqs || !sl::aligned4(seqs)))) return SL_ERR_INVALID_ARG;
  if (n > 65535) return SL_ERR_UNSUPPORTED;
  return sl::pages_free(c, seqs, n, static_cast<hipStream_t>(hip_stream));
}

size_t sl_pages_compact_workspace_bytes(const sl_page_cache* pc) {
  sl::PageCache c;
  return sl::make_cache(pc, &c) == SL_OK ? sl::pages_compact_ws_bytes(c) : SL_WORKSPACE_INVALID;
}

sl_status sl_pages_compact(const sl_page_cache* pc, int32_t* map, void* ws, size_t ws_bytes, void* hip_stream) {
  sl::PageCache c;
  sl_status s = sl::make_cache(pc, &c);
  if (s != SL_OK) return s;
  if (!map || !sl::aligned4(map)) return SL_ERR_INVALID_ARG;
  if (!ws || ws_bytes < sl::pages_compact_ws_bytes(c) || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SL_ERR_WORKSPACE;
  return sl::pages_compact(c, map, ws, static_cast<hipStream_t>(hip_stream));
}

sl_status sl_paged_append(const sl_page_cache* pc, const sl_paged_batch* pb, const void* K, const void* V, int64_t stride_h,
                          int64_t stride_t, void* hip_stream) {
  sl::PageCache c;
  sl::PagedBatch b;
  sl_status s = sl::make_cache(pc, &c);
  if (s == SL_OK) s = sl::make_batch(pb, c, &b);
  if (s != SL_OK) return s;
  if (stride_h < 0 || stride_t < 0) return SL_ERR_INVALID_ARG;
  if (stride_h > sl::kMaxStride || stride_t > sl::kMaxStride >> 8) return SL_ERR_UNSUPPORTED;
  if (b.B == 0 || b.rows == 0) return SL_OK;
  if (!K || !V || !sl::aligned16(K) || !sl::aligned16(V)) return SL_ERR_INVALID_ARG;
  const int64_t epl = c.dtype == SL_BF16 ? 8 : 4, st = stride_t ? stride_t : c.D, sh = stride_h ? stride_h : b.rows * st;
  if (st < c.D || st % epl || sh % epl) return SL_ERR_INVALID_ARG;
  return sl::paged_append(c, b, K, V, sh, st, static_cast<hipStream_t>(hip_stream));
}

sl_status sl_paged_span_keys(const sl_page_cache* pc, const sl_paged_batch* pb, int32_t S, int32_t n_spans, void* Ks, void* hip_stream) {
  sl::PageCache c;
  sl::PagedBatch b;
  sl_status s = sl::make_cache(pc, &c);
  if (s == SL_OK) s = sl::make_batch(pb, c, &b);
  if (s != SL_OK) return s;
  if (S < 1 || n_spans < 1 || !Ks || !sl::aligned16(Ks)) return SL_ERR_INVALID_ARG;
  if (n_spans > 65535 * 64) return SL_ERR_UNSUPPORTED;
  return sl::paged_span_keys(c, b, S, n_spans, Ks, static_cast<hipStream_t>(hip_stream));
}

size_t sl_paged_attention_workspace_bytes(const sl_page_cache* pc, const sl_paged_batch* pb, const sl_paged_attention* pa) {
  sl::PageCache c;
  sl::PagedBatch b;
  sl::PagedAttention a;
  if (sl::make_cache(pc, &c) != SL_OK || sl::make_batch(pb, c, &b) != SL_OK || sl::make_attention(pa, c, b, &a) != SL_OK)
    return SL_WORKSPACE_INVALID;
  if (b.B == 0 || b.rows == 0) return 0;
  return sl::paged_attention_ws_bytes(c, b, a);
}

sl_status sl_paged_span_attention(const sl_page_cache* c, const sl_paged_batch* b, const sl_paged_attention* a, const void* Q,
                                  const int32_t* idx, void* O, float* LSE, void* ws, size_t ws_bytes, void* hip_stream) {
  return sl::attention_entry(c, b, a, Q, idx, nullptr, false, O, LSE, ws, ws_bytes, hip_stream);
}

sl_status sl_paged_span_attention_combined(const sl_page_cache* c, const sl_paged_batch* b, const sl_paged_attention* a, const void* Q,
                                           const int32_t* idx, const float* scores, void* O, void* ws, size_t ws_bytes,
                                           void* hip_stream) {
  return sl::attention_entry(c, b, a, Q, idx, scores, true, O, nullptr, ws, ws_bytes, hip_stream);
}

}  // extern "C"
