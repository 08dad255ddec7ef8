/* The paged cache's size functions (host only, nothing is enqueued) over records whose fields stand at their limits, beyond them and at
 * small values.  Built with AddressSanitizer + UBSan against the sanitizer build of the library: an overflow in the validation or
 * in the size arithmetic is reported.  Prints how many records were accepted; exit code 0 = every size was one that can be. */
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>

#include "sl.h"

typedef size_t (*size_fn)(const sl_page_cache*, const sl_paged_batch*, const sl_paged_attention*);
typedef size_t (*compact_fn)(const sl_page_cache*);

static uint64_t state = 1;
static int64_t pick(const int64_t* from, int n) {
  state = state * 6364136223846793005u + 1442695040888963407u;
  return from[(state >> 33) % (uint64_t)n];
}
#define PICK(...) pick((const int64_t[]){__VA_ARGS__}, (int)(sizeof((int64_t[]){__VA_ARGS__}) / sizeof(int64_t)))

int main(int argc, char** argv) {
  if (argc < 2) return 2;
  void* lib = dlopen(argv[1], RTLD_NOW | RTLD_LOCAL);
  if (!lib) {
    fprintf(stderr, "dlopen: %s\n", dlerror());
    return 3;
  }
  size_fn size = (size_fn)dlsym(lib, "sl_paged_attention_workspace_bytes");
  compact_fn compact = (compact_fn)dlsym(lib, "sl_pages_compact_workspace_bytes");
  if (!size || !compact) return 4;
  void* const p = (void*)(uintptr_t)(1 << 20);
  int accepted = 0, wrong = 0;
  for (int i = 0; i < 400000; ++i) {
    sl_page_cache c = {p, p, (int32_t*)p, (int32_t*)p, (int32_t*)p, 0, 0, 0, 0, 1, 100, 8, 50, 64, 4, 128, SL_BF16};
    sl_paged_batch b = {(int32_t*)p, (int32_t*)p, 40, 0, 3, 0};
    sl_paged_attention a = {32, 256, 8, 0.f, 0, 0, 0, 0};
    c.layer_stride = PICK(0, 0, 0, 1 << 20, (int64_t)1 << 48, INT64_MAX);
    c.page_stride = PICK(0, 0, 0, 1 << 20, (int64_t)1 << 40, INT64_MAX);
    c.kv_stride_h = PICK(0, 0, 0, 128, 1 << 20, (int64_t)1 << 40, INT64_MAX);
    c.kv_stride_t = PICK(0, 0, 0, 128, 1 << 20, INT64_MAX);
    c.layers = (int32_t)PICK(1, 1, 2, 4096, INT32_MAX);
    c.n_pages = (int32_t)PICK(1, 100, 1 << 20, 1 << 30, INT32_MAX);
    c.max_pages = (int32_t)PICK(1, 50, 1 << 14, 1 << 25, INT32_MAX);
    c.page_size = (int32_t)PICK(1, 32, 64, 1 << 16, 1 << 30, INT32_MAX);
    c.Hkv = (int32_t)PICK(1, 4, 4, 1024);
    c.D = (int32_t)PICK(64, 128);
    c.dtype = (int32_t)PICK(SL_F32, SL_BF16);
    b.rows = PICK(1, 40, 4096, (1 << 20) - 1, (1 << 25) - 1, 1 << 25, INT64_MAX);
    b.L = PICK(0, 0, 1, 1 << 16, 1 << 30, INT64_MAX);
    b.B = (int32_t)PICK(1, 3, 4096, 65535);
    a.Hq = c.Hkv * (int32_t)PICK(1, 2, 8, 64);
    a.S = (int32_t)PICK(1, 4, 256, 1 << 24, INT32_MAX);
    a.topk = (int32_t)PICK(0, 1, 8, 32);
    a.q_stride_h = PICK(0, 0, 128, (int64_t)1 << 40, INT64_MAX);
    a.q_stride_t = PICK(0, 0, 128, (int64_t)1 << 32, INT64_MAX);
    a.idx_stride_h = PICK(0, 0, 8, (int64_t)1 << 40, INT64_MAX);
    a.idx_stride_t = PICK(0, 0, 8, (int64_t)1 << 32, INT64_MAX);
    const size_t n = size(&c, &b, &a), m = compact(&c);
    if (n != SL_WORKSPACE_INVALID) {
      ++accepted;
      /* 2^26 rows and heads, 32 * 64 + 256 pieces, 512 + 8 bytes each, is below 2^47 */
      if (n > (size_t)1 << 47 || m == SL_WORKSPACE_INVALID) ++wrong;
    }
    if (m != SL_WORKSPACE_INVALID && (m < 4 * (size_t)c.n_pages || m > 4 * (size_t)c.n_pages + 1024)) ++wrong;
  }
  printf("accepted=%d wrong=%d\n", accepted, wrong);
  return wrong != 0 || accepted < 1000;
}
