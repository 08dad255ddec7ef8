// Span-attention over a paged cache of bf16 or fp32 rows; which form a cache takes.
#include "paged_attention.h"

namespace sl {

size_t paged_attention_ws_bytes(const PageCache& c, const PagedBatch& b, const PagedAttention& a) {
  const Form f = form_of(c, b, a);
  return f.o_bytes + 2 * f.lse_bytes + f.plan_bytes;
}

sl_status paged_attention(const PageCache& c, const PagedBatch& b, const PagedAttention& a, const void* Q, const int32_t* idx,
                          const float* scores, void* O, float* LSE, void* ws, hipStream_t st) {
  return c.fp4 ? paged_attention_fp4(c, b, a, Q, idx, scores, O, LSE, ws, st) : attend_pages<false>(c, b, a, Q, idx, scores, O, LSE, ws, st);
}

}  // namespace sl
