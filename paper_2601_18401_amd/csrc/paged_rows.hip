// Rows of a paged cache: written in 4 bits, read back, span keys of a cache in 4 bits.  (fp4.h has the format.)
//
// A lane takes eight channels of a row: 16 or 32 bytes of it, four of codes; four lanes a block of 32, whose largest value they find
// together.
#include "fp4.h"
#include "paged.h"

namespace sl {

namespace {

// Rows of a workgroup: 64 hold 2 or 4 loads of a lane in flight.  Both kernels are bound by memory, at 4.9 (rounded, 99000 rows of 8 heads,
// 128 channels, and read back: 920 MB in 187 us; with 32 rows 194, 256 216) and 4.2 TB/s (162000 rows of 8 heads read, 835 MB in 200 us; 32 rows
// 218; with plain stores 240), where a large copy reaches 5.0.
constexpr int kRows = 64;

template <typename T>
__device__ __forceinline__ void load_row8(const T* from, uint4* to) {
  to[0] = load16_stream(from);
  if constexpr (sizeof(T) == 4) to[1] = load16_stream(from + 4);
}
template <typename T>
__device__ __forceinline__ void store_row8(T* to, const uint4* from) {
  store16_stream(to, from[0]);
  if constexpr (sizeof(T) == 4) store16_stream(to + 4, from[1]);
}

// Largest of the four lanes of a block.
__device__ __forceinline__ uint32_t max_of_block(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));  // lane ^ 1
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));  // lane ^ 2
}

// Workgroup (x, y): kRows rows of head y.  A lane for each row finds its place, then all lanes work.
template <typename T, int D>
__global__ __launch_bounds__(256) void append_fp4_kernel(const PageCache c, const PagedBatch b, const T* __restrict__ K,
                                                         const T* __restrict__ V, int64_t sh, int64_t st) {
  __shared__ int64_t s_block[kRows];  // the head's part of the row's page; < 0: nowhere
  __shared__ int s_at[kRows];
  constexpr int LANES = D / 8, N = kRows * LANES / 256;
  static_assert(N >= 1 && kRows <= 256, "every thread has rows, and every row a thread");
  const int first = blockIdx.x * kRows, head = blockIdx.y;
  if (threadIdx.x < kRows) {
    const RowPlace p = place_of_row(c, b, first + threadIdx.x);
    // (a page of several sequences holds tokens of each, whatever the batch says of this one)
    const bool on = p.page >= 0 && c.refs[p.page] <= 1;
    s_block[threadIdx.x] = on ? b.layer * c.layer + p.page * c.page + head * c.head : -1;
    s_at[threadIdx.x] = p.at;
  }
  __syncthreads();
  const int lr = threadIdx.x % LANES;
  constexpr int W = sizeof(T) == 2 ? 1 : 2;
  uint4 x[2][N][W];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int row = threadIdx.x / LANES + i * (256 / LANES);
    if (s_block[row] < 0) continue;
    const int64_t from = head * sh + (int64_t)(first + row) * st + lr * 8;
    load_row8(K + from, x[0][i]);
    load_row8(V + from, x[1][i]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int row = threadIdx.x / LANES + i * (256 / LANES);
    const int64_t block = s_block[row];
    if (block < 0) continue;
    const int64_t at = s_at[row];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const uint32_t scale = fp4_scale(max_of_block(largest_bits<T>(x[v][i])));
      uint8_t* const to = static_cast<uint8_t*>(v ? c.V : c.K) + block;
      *reinterpret_cast<uint32_t*>(to + at * (D / 2) + lr * 4) = row8_to_fp4<T>(x[v][i], scale);
      if (lr % 4 == 0) to[(int64_t)c.ps * (D / 2) + at * (D / 32) + lr / 4] = (uint8_t)scale;
    }
  }
}

// The batch's tokens as rows: what the pages hold, zeros where there is no token or no page for it.
template <typename T, int D, bool FP4>
__global__ __launch_bounds__(256) void read_kernel(const PageCache c, const PagedBatch b, T* __restrict__ K, T* __restrict__ V, int64_t sh,
                                                   int64_t st) {
  __shared__ int64_t s_block[kRows];  // the head's part of the row's page; -1: zeros, -2: a row of nobody
  __shared__ int s_at[kRows];
  constexpr int LANES = D / 8, N = kRows * LANES / 256;
  static_assert(N >= 1 && kRows <= 256, "every thread has rows, and every row a thread");
  const int first = blockIdx.x * kRows, head = blockIdx.y;
  if (threadIdx.x < kRows) {
    const RowPlace p = place_of_row(c, b, first + threadIdx.x);
    s_block[threadIdx.x] = p.page >= 0 ? b.layer * c.layer + p.page * c.page + head * c.head : p.listed ? -1 : -2;
    s_at[threadIdx.x] = p.at;
  }
  __syncthreads();
  const int lr = threadIdx.x % LANES;
  constexpr int W = sizeof(T) == 2 ? 1 : 2;
  uint4 x[2][N][W];
  uint32_t code[2][N], scale[2][N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int row = threadIdx.x / LANES + i * (256 / LANES);
    const int64_t block = s_block[row], at = s_at[row];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      code[v][i] = scale[v][i] = 0;
      for (uint4& w : x[v][i]) w = make_uint4(0, 0, 0, 0);
      if (block < 0) continue;
      if constexpr (FP4) {
        const uint8_t* const from = static_cast<const uint8_t*>(v ? c.V : c.K) + block;
        code[v][i] = *reinterpret_cast<const uint32_t*>(from + at * (D / 2) + lr * 4);
        scale[v][i] = from[(int64_t)c.ps * (D / 2) + at * (D / 32) + lr / 4];
      } else {
        load_row8(static_cast<const T*>(v ? c.V : c.K) + block + at * c.tok + lr * 8, x[v][i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int row = threadIdx.x / LANES + i * (256 / LANES);
    if (s_block[row] == -2) continue;
    const int64_t to = head * sh + (int64_t)(first + row) * st + lr * 8;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      if constexpr (FP4) fp4_to_row8<T>(code[v][i], scale[v][i], x[v][i]);
      store_row8((v ? V : K) + to, x[v][i]);
    }
  }
}

constexpr int kKeySpans = 64;  // spans of a workgroup

// Workgroup (e, y, head): those of entry e's completed spans that lie in [64 y, 64 y + 64).
template <typename T, int D>
__global__ __launch_bounds__(256) void span_keys_fp4_kernel(const PageCache c, const PagedBatch b, int S, int n_spans, T* __restrict__ Ks) {
  constexpr int LANES = D / 8;
  const int e = blockIdx.x, head = blockIdx.z;
  const int s = b.seqs[e], len = length_of(c, s), n = b.cu[e + 1] - b.cu[e];
  if (n <= 0 || len <= 0) return;
  const int first = max(max(len - n, 0) / S, (int)blockIdx.y * kKeySpans);
  const int end = min(min(min(len, b.L) / S, n_spans), ((int)blockIdx.y + 1) * kKeySpans);
  const int lr = threadIdx.x % LANES;
  for (int j = first + threadIdx.x / LANES; j < end; j += 256 / LANES) {
    const int t = j * S + (S - 1), k = (uint32_t)t / c.by_ps, page = c.tables[(int64_t)s * c.max_pages + k];
    if ((uint32_t)page >= (uint32_t)c.n_pages) continue;
    const uint8_t* const from = static_cast<const uint8_t*>(c.K) + b.layer * c.layer + page * c.page + head * c.head;
    const int64_t at = t - k * c.ps;
    uint4 x[sizeof(T) == 2 ? 1 : 2];
    fp4_to_row8<T>(*reinterpret_cast<const uint32_t*>(from + at * (D / 2) + lr * 4), from[(int64_t)c.ps * (D / 2) + at * (D / 32) + lr / 4], x);
    uint4* const to = reinterpret_cast<uint4*>(Ks + (((int64_t)s * c.Hkv + head) * n_spans + j) * D + lr * 8);
    to[0] = x[0];
    if constexpr (sizeof(T) == 4) to[1] = x[1];
  }
}

sl_status launched() { return hipGetLastError() == hipSuccess ? SL_OK : SL_ERR_LAUNCH; }

// call(T(), std::integral_constant<int, D>()) for the cache's rows
template <typename F>
void for_rows(const PageCache& c, F&& call) {
  if (c.dtype == SL_BF16) c.D == 128 ? call(bf16_t(), std::integral_constant<int, 128>()) : call(bf16_t(), std::integral_constant<int, 64>());
  else c.D == 128 ? call(float(), std::integral_constant<int, 128>()) : call(float(), std::integral_constant<int, 64>());
}
dim3 rows_grid(const PageCache& c, const PagedBatch& b) { return dim3((unsigned)((b.rows + kRows - 1) / kRows), c.Hkv); }

}  // namespace

sl_status paged_append_fp4(const PageCache& c, const PagedBatch& b, const void* K, const void* V, int64_t sh, int64_t st_, hipStream_t st) {
  for_rows(c, [&](auto t, auto d) {
    typedef decltype(t) T;
    append_fp4_kernel<T, d.value><<<rows_grid(c, b), 256, 0, st>>>(c, b, static_cast<const T*>(K), static_cast<const T*>(V), sh, st_);
  });
  return launched();
}

sl_status paged_read(const PageCache& c, const PagedBatch& b, void* K, void* V, int64_t sh, int64_t st_, hipStream_t st) {
  for_rows(c, [&](auto t, auto d) {
    typedef decltype(t) T;
    if (c.fp4) read_kernel<T, d.value, true><<<rows_grid(c, b), 256, 0, st>>>(c, b, static_cast<T*>(K), static_cast<T*>(V), sh, st_);
    else read_kernel<T, d.value, false><<<rows_grid(c, b), 256, 0, st>>>(c, b, static_cast<T*>(K), static_cast<T*>(V), sh, st_);
  });
  return launched();
}

sl_status paged_span_keys_fp4(const PageCache& c, const PagedBatch& b, int S, int n_spans, void* Ks, hipStream_t st) {
  for_rows(c, [&](auto t, auto d) {
    typedef decltype(t) T;
    const int chunks = (n_spans + kKeySpans - 1) / kKeySpans;
    span_keys_fp4_kernel<T, d.value><<<dim3(b.B, chunks, c.Hkv), 256, 0, st>>>(c, b, S, n_spans, static_cast<T*>(Ks));
  });
  return launched();
}

}  // namespace sl
