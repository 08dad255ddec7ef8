// Span-attention over a paged cache held in 4 bits.
#include "paged_attention.h"

namespace sl {

sl_status paged_attention_fp4(const PageCache& c, const PagedBatch& b, const PagedAttention& a, const void* Q, const int32_t* idx,
                              const float* scores, void* O, float* LSE, void* ws, hipStream_t st) {
  return attend_pages<true>(c, b, a, Q, idx, scores, O, LSE, ws, st);
}

}  // namespace sl
