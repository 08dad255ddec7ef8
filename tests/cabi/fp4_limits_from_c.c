/* Caches in 4 bits at the limits of their records' fields, beyond them and at small values, on the host alone: sizes of scratch memory, and
 * reads of rows, all of which are refused, K and V being one tensor.  Built with AddressSanitizer + UBSan against the sanitizer build of
 * the library.  Prints how many records were accepted; exit code 0 = every answer was one that can be. */
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>

#include "sl.h"

typedef size_t (*size_fn)(const sl_page_cache*, const sl_paged_batch*, const sl_paged_attention*);
typedef size_t (*compact_fn)(const sl_page_cache*);
typedef sl_status (*read_fn)(const sl_page_cache*, const sl_paged_batch*, void*, void*, int64_t, int64_t, void*);

static uint64_t state = 7;
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
  read_fn read = (read_fn)dlsym(lib, "sl_paged_read");
  if (!size || !compact || !read) return 4;
  void* const p = (void*)(uintptr_t)(1 << 20);
  int accepted = 0, met = 0, wrong = 0;
  for (int i = 0; i < 200000; ++i) {
    sl_page_cache c = {p, p, (int32_t*)p, (int32_t*)p, (int32_t*)p, 0, 0, 0, 0, 1, 100, 8, 50, 64, 4, 128, SL_MXFP4_BF16};
    sl_paged_batch b = {(int32_t*)p, (int32_t*)p, 40, 0, 3, 0};
    sl_paged_attention a = {32, 256, 8, 0.f, 0, 0, 0, 0};
    c.layer_stride = PICK(0, 0, 0, 1 << 20, (int64_t)1 << 48, INT64_MAX);
    c.page_stride = PICK(0, 0, 0, 1 << 20, (int64_t)1 << 40, INT64_MAX);
    c.kv_stride_h = PICK(0, 0, 0, 4352, 1 << 20, (int64_t)1 << 40, INT64_MAX);
    c.kv_stride_t = PICK(0, 0, 0, 32, 64, INT64_MAX);
    c.layers = (int32_t)PICK(1, 1, 2, 4096, INT32_MAX);
    c.n_pages = (int32_t)PICK(1, 100, 1 << 20, 1 << 30, INT32_MAX);
    c.max_pages = (int32_t)PICK(1, 50, 1 << 14, 1 << 25, INT32_MAX);
    c.page_size = (int32_t)PICK(1, 32, 64, 1 << 16, 1 << 30, INT32_MAX);
    c.Hkv = (int32_t)PICK(1, 4, 4, 1024);
    c.D = (int32_t)PICK(64, 128);
    c.dtype = (int32_t)PICK(SL_MXFP4_F32, SL_MXFP4_BF16, SL_MXFP4_BF16);
    b.rows = PICK(1, 40, 4096, (1 << 20) - 1, (1 << 25) - 1, 1 << 25, INT64_MAX);
    b.L = PICK(0, 0, 1, 1 << 16, 1 << 30, INT64_MAX);
    b.B = (int32_t)PICK(1, 3, 4096, 65535);
    a.Hq = c.Hkv * (int32_t)PICK(1, 2, 8, 64);
    a.S = (int32_t)PICK(1, 4, 256, 1 << 24, INT32_MAX);
    a.topk = (int32_t)PICK(0, 1, 8, 32);
    const size_t n = size(&c, &b, &a), m = compact(&c);
    if (n != SL_WORKSPACE_INVALID) {
      ++accepted;
      /* 2^26 rows and heads, 32 * 64 + 256 pieces, 512 + 8 bytes each, is below 2^47 */
      if (n > (size_t)1 << 47 || m == SL_WORKSPACE_INVALID) ++wrong;
    }
    if (m != SL_WORKSPACE_INVALID && (m < 4 * (size_t)c.n_pages || m > 4 * (size_t)c.n_pages + 1024)) ++wrong;
    const int64_t sh = PICK(0, 0, 64, 128, 1 << 20, (int64_t)1 << 40, INT64_MAX);
    const int64_t st = PICK(0, 0, 64, 128, 1 << 20, (int64_t)1 << 32, INT64_MAX);
    const sl_status s = read(&c, &b, p, (char*)p + 16 * PICK(0, 1, 7, -3), sh, st, NULL);
    if (s != SL_ERR_INVALID_ARG && s != SL_ERR_UNSUPPORTED) ++wrong;
    met += s == SL_ERR_INVALID_ARG;
  }
  printf("accepted=%d met=%d wrong=%d\n", accepted, met, wrong);
  return wrong != 0 || accepted < 1000 || met < 1000;
}
