// Pages of a KV cache: given out, forked, freed, compacted; new tokens written, span keys gathered.
//
// All of it is data movement and small integers.  What decides who gets which page is one workgroup's
// prefix sums, so that the result does not depend on an order of atomics; what moves data is spread over the chip.
#include "paged.h"

namespace sl {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPerThread = 16;  // reference counts a thread looks at per pass: four 16-byte loads

// Sum of v over the threads before this one; total: over all.  (1024 threads)
template <typename I>
__device__ __forceinline__ I scan_before(I v, I* s_wave, I* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  I x = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const I y = __shfl_up(x, off, 64);
    if (lane >= off) x += y;
  }
  __syncthreads();  // (the last call's readers of s_wave are done)
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  I before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const I y = s_wave[w];
    if (w < wave) before += y;
    all += y;
  }
  *total = all;
  return before + x - v;
}

// refs[at .. at + 15], 1 where there is no page: such are not free
__device__ __forceinline__ void load_refs(const int32_t* __restrict__ refs, int at, int n, int (&r)[kPerThread]) {
  if (at + kPerThread <= n) {
#pragma unroll
    for (int i = 0; i < kPerThread / 4; ++i) {
      const int4 x = reinterpret_cast<const int4*>(refs + at)[i];
      r[4 * i] = x.x;
      r[4 * i + 1] = x.y;
      r[4 * i + 2] = x.z;
      r[4 * i + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) r[i] = at + i < n ? refs[at + i] : 1;
  }
}

// Entry i of a list (in LDS) is its sequence's first one.  Four entries a read, the same ones for the wavefront.
__device__ __forceinline__ bool listed_first(const int32_t* list, int i) {
  const int s = list[i], upto = __builtin_amdgcn_readfirstlane(i | 63);
  bool first = true;
#pragma unroll 4
  for (int k = 0; k < upto; k += 4) {
    const int4 x = *reinterpret_cast<const int4*>(list + k);
    first = first && !(x.x == s && k < i) && !(x.y == s && k + 1 < i) && !(x.z == s && k + 2 < i) && !(x.w == s && k + 3 < i);
  }
  return first;
}

// Pages for new tokens (FORK: for copies of partly filled pages).  end[i]: pages that entries 0 .. i need together; an
// entry is served if the free pages reach that far.  The counts are scanned from the front until the last page is found;
// what one workgroup reads of them at once (64 KB) takes about a microsecond.
template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void plan_pages_kernel(const PageCache c, const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ seqs, const int32_t* __restrict__ cu,
                                                                  int n, int32_t* __restrict__ ok) {
  __shared__ int64_t s_end[SL_MAX_PAGE_OPS];
  __shared__ __align__(16) int32_t s_seq[SL_MAX_PAGE_OPS];  // -1: not to be served
  __shared__ int32_t s_have[SL_MAX_PAGE_OPS];  // FORK: tokens of the source; else: pages held
  __shared__ int64_t s_wave64[kPlanThreads / 64];
  __shared__ int32_t s_wave[kPlanThreads / 64];
  const int most = c.max_pages * c.ps;
  for (int i = threadIdx.x; i < n; i += kPlanThreads) s_seq[i] = seqs[i];
  __syncthreads();
  bool good[SL_MAX_PAGE_OPS / kPlanThreads];
#pragma unroll
  for (int q = 0; q < SL_MAX_PAGE_OPS / kPlanThreads; ++q) {
    const int i = q * kPlanThreads + threadIdx.x;
    good[q] = i < n && (uint32_t)s_seq[i] < (uint32_t)c.n_seqs && listed_first(s_seq, i);
  }
  __syncthreads();
  int64_t before = 0;
#pragma unroll
  for (int q = 0; q < SL_MAX_PAGE_OPS / kPlanThreads; ++q) {
    if (q * kPlanThreads >= n) break;
    const int i = q * kPlanThreads + threadIdx.x;
    int need = 0;
    if (good[q]) {
      const int len = c.lens[s_seq[i]];
      if constexpr (FORK) {
        const int from = src[i];
        const int held = (uint32_t)from < (uint32_t)c.n_seqs && from != s_seq[i] ? c.lens[from] : -1;
        good[q] = len == 0 && held >= 0 && held <= most;
        if (good[q]) {
          s_have[i] = held;
          need = (uint32_t)held != (uint32_t)held / c.by_ps * c.ps;
        }
      } else {
        const int64_t add = (int64_t)cu[i + 1] - cu[i];
        good[q] = len >= 0 && add >= 0 && len + add <= most;
        if (good[q]) {
          s_have[i] = (uint32_t)(len + c.ps - 1) / c.by_ps;
          need = (int)((uint32_t)(len + (int)add + c.ps - 1) / c.by_ps) - s_have[i];
        }
      }
    }
    int64_t all;
    const int64_t at = before + scan_before<int64_t>(need, s_wave64, &all);
    if (i < n) {
      s_end[i] = at + need;
      if (!good[q]) s_seq[i] = -1;
    }
    before += all;
  }
  __syncthreads();
  const int64_t total = before;
  // free pages, in order, to the entries
  int64_t found = 0;
  int r[kPerThread];
  load_refs(c.refs, threadIdx.x * kPerThread, c.n_pages, r);
  for (int64_t base = 0; base < c.n_pages && found < total; base += kPlanThreads * kPerThread) {
    int next[kPerThread];
    const int64_t ahead = base + kPlanThreads * kPerThread;
    if (ahead < c.n_pages) load_refs(c.refs, (int)min(ahead + threadIdx.x * kPerThread, (int64_t)c.n_pages), c.n_pages, next);
    int mine = 0;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) mine += r[k] <= 0;
    int all;
    int64_t rank = found + scan_before<int>(mine, s_wave, &all);
    if (mine > 0 && rank < total) {
      int e = 0;
      {  // the entry that gets page `rank`: the first with end > rank
        int lo = 0, hi = n - 1;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (s_end[mid] > rank) hi = mid;
          else lo = mid + 1;
        }
        e = lo;
      }
#pragma unroll
      for (int k = 0; k < kPerThread; ++k) {
        if (r[k] > 0 || rank >= total) continue;
        while (s_end[e] <= rank) ++e;
        const int page = (int)base + threadIdx.x * kPerThread + k;
        const int64_t first = e ? s_end[e - 1] : 0;
        const int at = FORK ? (int)((uint32_t)s_have[e] / c.by_ps) : s_have[e] + (int)(rank - first);
        c.tables[(int64_t)s_seq[e] * c.max_pages + at] = page;
        c.refs[page] = 1;
        ++rank;
      }
    }
    found += all;
    if (ahead < c.n_pages) {
#pragma unroll
      for (int k = 0; k < kPerThread; ++k) r[k] = next[k];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int64_t first = i ? s_end[i - 1] : 0, end = s_end[i];
    const bool served = s_seq[i] >= 0 && (end == first || end <= found);
    if (served) {
      if (FORK) c.lens[s_seq[i]] = s_have[i];
      else c.lens[s_seq[i]] += cu[i + 1] - cu[i];
    } else if (!FORK && s_seq[i] >= 0) {  // the entry at which the pages ran out gives back what it got
      for (int64_t k = first; k < found && k < end; ++k) {
        int32_t* const t = c.tables + (int64_t)s_seq[i] * c.max_pages + s_have[i] + (k - first);
        c.refs[*t] = 0;
        *t = -1;
      }
    }
    ok[i] = served;
  }
}

// Copies rows [0, rows) of one head's part of a page, 16 bytes a lane.
__device__ __forceinline__ void copy_rows(const char* __restrict__ from, char* __restrict__ to, int64_t row_bytes, int pieces_log2,
                                          int rows, int thread, int threads) {
  const int n = rows << pieces_log2, mask = (1 << pieces_log2) - 1;
  constexpr int U = 4;
  int p = thread;
  for (; p + (U - 1) * threads < n; p += U * threads) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = p + u * threads;
      x[u] = load16(from + (q >> pieces_log2) * row_bytes + (q & mask) * 16);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = p + u * threads;
      *reinterpret_cast<uint4*>(to + (q >> pieces_log2) * row_bytes + (q & mask) * 16) = x[u];
    }
  }
  for (; p < n; p += threads)
    *reinterpret_cast<uint4*>(to + (p >> pieces_log2) * row_bytes + (p & mask) * 16) =
        load16(from + (p >> pieces_log2) * row_bytes + (p & mask) * 16);
}

__host__ __device__ inline int element_bytes(const PageCache& c) { return c.dtype == SL_BF16 ? 2 : 4; }
// 16-byte pieces of a row: 8, 16 or 32
__host__ __device__ inline int pieces_log2_of(const PageCache& c) { return (c.D == 128 ? 4 : 3) + (c.dtype == SL_BF16 ? 0 : 1); }

// One (layer, K or V, head) part of a page: unit in [0, layers * 2 * Hkv)
__device__ __forceinline__ void copy_part(const PageCache& c, int from, int to, int unit, int rows, int thread, int threads) {
  const int es = element_bytes(c);
  const int head = unit % c.Hkv, lt = unit / c.Hkv;
  char* const base = reinterpret_cast<char*>(lt & 1 ? c.V : c.K) + ((lt >> 1) * c.layer + head * c.head) * es;
  copy_rows(base + from * c.page * es, base + to * c.page * es, c.tok * es, pieces_log2_of(c), rows, thread, threads);
}

constexpr int kForkEntries = 1024;  // table entries of a workgroup

// What plan_pages_kernel<true> decided: dst's table from src's, references, the copied last page.
__global__ __launch_bounds__(256) void fork_kernel(const PageCache c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                   const int32_t* __restrict__ ok, int n, int chunks) {
  const int f = blockIdx.x, y = blockIdx.y;
  if (!ok[f]) return;
  const int s = src[f], d = dst[f], len = c.lens[d];
  const int full = (uint32_t)len / c.by_ps, part = len - full * c.ps;
  const int32_t* const from = c.tables + (int64_t)s * c.max_pages;
  int32_t* const to = c.tables + (int64_t)d * c.max_pages;
  if (y < chunks) {
    for (int k = y * kForkEntries + threadIdx.x; k < full && k < (y + 1) * kForkEntries; k += 256) {
      const int page = from[k];
      to[k] = page;
      if ((uint32_t)page < (uint32_t)c.n_pages) atomicAdd(&c.refs[page], 1);
    }
  } else if (part) {
    const int page = from[full];
    if ((uint32_t)page < (uint32_t)c.n_pages) copy_part(c, page, to[full], y - chunks, part, threadIdx.x, 256);
  }
}

__global__ __launch_bounds__(256) void free_kernel(const PageCache c, const int32_t* __restrict__ seqs) {
  const int s = seqs[blockIdx.x];
  if ((uint32_t)s >= (uint32_t)c.n_seqs) return;
  if (blockIdx.y == 0 && threadIdx.x == 0) c.lens[s] = 0;
  int32_t* const t = c.tables + (int64_t)s * c.max_pages;
  for (int k = blockIdx.y * kForkEntries + threadIdx.x; k < c.max_pages && k < ((int)blockIdx.y + 1) * kForkEntries; k += 256) {
    if (t[k] == -1) continue;
    const int page = atomicExch(&t[k], -1);  // (a sequence listed twice: one of the two gets the page)
    if ((uint32_t)page < (uint32_t)c.n_pages) atomicSub(&c.refs[page], 1);
  }
}

// The pages that move: pair k is moves[k] -> moves[half + k], k < *count.
__global__ __launch_bounds__(kPlanThreads) void plan_compact_kernel(const PageCache c, int32_t* __restrict__ map, int32_t* __restrict__ count,
                                                                    int32_t* __restrict__ moves, int half) {
  __shared__ int32_t s_wave[kPlanThreads / 64];
  int used = 0;
  int r[kPerThread];
  for (int64_t base = 0; base < c.n_pages; base += kPlanThreads * kPerThread) {
    load_refs(c.refs, (int)min(base + threadIdx.x * kPerThread, (int64_t)c.n_pages), c.n_pages, r);
    const int at = (int)min(base + threadIdx.x * kPerThread, (int64_t)c.n_pages);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) used += at + k < c.n_pages && r[k] > 0;
  }
  int n;
  scan_before<int>(used, s_wave, &n);
  int holes = 0, movers = 0;  // so far
  for (int64_t base = 0; base < c.n_pages; base += kPlanThreads * kPerThread) {
    const int at = (int)min(base + threadIdx.x * kPerThread, (int64_t)c.n_pages);
    load_refs(c.refs, at, c.n_pages, r);
    int h = 0, m = 0, hs, ms;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      h += at + k < n && r[k] <= 0;
      m += at + k >= n && at + k < c.n_pages && r[k] > 0;
    }
    int hk = holes + scan_before<int>(h, s_wave, &hs), mk = movers + scan_before<int>(m, s_wave, &ms);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int p = at + k;
      if (p >= c.n_pages) continue;
      if (p < n) {
        if (r[k] <= 0) moves[half + hk++] = p;
        else map[p] = p;
      } else if (r[k] > 0) {
        moves[mk++] = p;
      }
      if (r[k] <= 0) map[p] = -1;
    }
    holes += hs;
    movers += ms;
  }
  __syncthreads();  // (also orders the workgroup's own writes to moves before the reads)
  for (int k = threadIdx.x; k < movers; k += kPlanThreads) {
    const int from = moves[k], to = moves[half + k];
    map[from] = to;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
  }
  if (threadIdx.x == 0) *count = movers;
}

// The first `tables` workgroups rewrite the tables, the others move pages.
__global__ __launch_bounds__(256) void compact_kernel(const PageCache c, const int32_t* __restrict__ map, const int32_t* __restrict__ count,
                                                      const int32_t* __restrict__ moves, int half, int tables) {
  if ((int)blockIdx.x < tables) {
    const int64_t n = (int64_t)c.n_seqs * c.max_pages;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < n; k += (int64_t)tables * 256) {
      const int page = c.tables[k];
      if ((uint32_t)page >= (uint32_t)c.n_pages) continue;
      const int to = map[page];
      if (to != page) c.tables[k] = to;
    }
    return;
  }
  const int parts = c.layers * 2 * c.Hkv;
  const int64_t units = (int64_t)*count * parts;
  for (int64_t u = blockIdx.x - tables; u < units; u += gridDim.x - tables) {
    const int k = (int)(u / parts);
    copy_part(c, moves[k], moves[half + k], (int)(u - (int64_t)k * parts), c.ps, threadIdx.x, 256);
  }
}

// A lane takes 16 bytes of a row of K and of V; rows of one head follow each other.
__global__ __launch_bounds__(256) void append_kernel(const PageCache c, const PagedBatch b, const char* __restrict__ K,
                                                     const char* __restrict__ V, int64_t sh, int64_t st, int pieces_log2) {
  const int at = blockIdx.x * 256 + threadIdx.x, head = blockIdx.y;
  const int row = at >> pieces_log2, piece = at & ((1 << pieces_log2) - 1);
  if (row < b.cu[0] || row >= min(b.cu[b.B], b.rows)) return;
  const int e = entry_of_row(b.cu, b.B, row), s = b.seqs[e], len = length_of(c, s);
  const int t = len - (b.cu[e + 1] - row);
  if (t < 0 || t >= b.L || t >= len) return;
  const int k = (uint32_t)t / c.by_ps, page = c.tables[(int64_t)s * c.max_pages + k];
  if ((uint32_t)page >= (uint32_t)c.n_pages) return;
  const int es = element_bytes(c);
  const int64_t from = (head * sh + row * st) * es + piece * 16;
  const int64_t to = (b.layer * c.layer + page * c.page + head * c.head + (t - k * c.ps) * c.tok) * es + piece * 16;
  const uint4 x = load16(K + from), y = load16(V + from);
  *reinterpret_cast<uint4*>(reinterpret_cast<char*>(c.K) + to) = x;
  *reinterpret_cast<uint4*>(reinterpret_cast<char*>(c.V) + to) = y;
}

constexpr int kKeySpans = 64;  // spans of a workgroup

// Workgroup (b, y, head): those of entry b's completed spans that lie in [64 y, 64 y + 64).
__global__ __launch_bounds__(256) void span_keys_kernel(const PageCache c, const PagedBatch b, int S, int n_spans, char* __restrict__ Ks,
                                                        int pieces_log2) {
  const int e = blockIdx.x, head = blockIdx.z;
  const int s = b.seqs[e], len = length_of(c, s), n = b.cu[e + 1] - b.cu[e];
  if (n <= 0 || len <= 0) return;
  const int first = max(max(len - n, 0) / S, (int)blockIdx.y * kKeySpans);
  const int end = min(min(min(len, b.L) / S, n_spans), ((int)blockIdx.y + 1) * kKeySpans);
  const int es = element_bytes(c);
  for (int at = threadIdx.x; at < (end - first) << pieces_log2; at += 256) {
    const int j = first + (at >> pieces_log2), piece = at & ((1 << pieces_log2) - 1), t = j * S + (S - 1);
    const int k = (uint32_t)t / c.by_ps, page = c.tables[(int64_t)s * c.max_pages + k];
    if ((uint32_t)page >= (uint32_t)c.n_pages) continue;
    const int64_t from = (b.layer * c.layer + page * c.page + head * c.head + (t - k * c.ps) * c.tok) * es + piece * 16;
    const int64_t to = (((int64_t)s * c.Hkv + head) * n_spans + j) * c.D * es + piece * 16;
    *reinterpret_cast<uint4*>(Ks + to) = load16(reinterpret_cast<const char*>(c.K) + from);
  }
}

sl_status launched() { return hipGetLastError() == hipSuccess ? SL_OK : SL_ERR_LAUNCH; }

}  // namespace

sl_status pages_extend(const PageCache& c, const PagedBatch& b, int32_t* ok, hipStream_t st) {
  if (b.B == 0) return SL_OK;
  plan_pages_kernel<false><<<1, kPlanThreads, 0, st>>>(c, nullptr, b.seqs, b.cu, b.B, ok);
  return launched();
}

sl_status pages_fork(const PageCache& c, const int32_t* src, const int32_t* dst, int n, int32_t* ok, hipStream_t st) {
  if (n == 0) return SL_OK;
  plan_pages_kernel<true><<<1, kPlanThreads, 0, st>>>(c, src, dst, nullptr, n, ok);
  const int chunks = (c.max_pages + kForkEntries - 1) / kForkEntries;
  fork_kernel<<<dim3(n, chunks + c.layers * 2 * c.Hkv), 256, 0, st>>>(c, src, dst, ok, n, chunks);
  return launched();
}

sl_status pages_free(const PageCache& c, const int32_t* seqs, int n, hipStream_t st) {
  if (n == 0) return SL_OK;
  free_kernel<<<dim3(n, (c.max_pages + kForkEntries - 1) / kForkEntries), 256, 0, st>>>(c, seqs);
  return launched();
}

size_t pages_compact_ws_bytes(const PageCache& c) { return align_up(sizeof(int32_t) * (64 + 2 * ((size_t)c.n_pages / 2 + 1)), 256); }

sl_status pages_compact(const PageCache& c, int32_t* map, void* ws, hipStream_t st) {
  int32_t* const count = static_cast<int32_t*>(ws);
  int32_t* const moves = count + 64;
  const int half = c.n_pages / 2 + 1;  // pages that move are above the used ones' number, holes below: at most half of the pool
  plan_compact_kernel<<<1, kPlanThreads, 0, st>>>(c, map, count, moves, half);
  const int64_t entries = (int64_t)c.n_seqs * c.max_pages, units = (int64_t)(half - 1) * c.layers * 2 * c.Hkv;
  const int tables = (int)min((entries + 1023) / 1024, (int64_t)512), copies = (int)min(units, (int64_t)2048);
  compact_kernel<<<tables + copies, 256, 0, st>>>(c, map, count, moves, half, tables);
  return launched();
}

sl_status paged_append(const PageCache& c, const PagedBatch& b, const void* K, const void* V, int64_t sh, int64_t st_, hipStream_t st) {
  if (b.B == 0 || b.rows == 0) return SL_OK;
  const int pl = pieces_log2_of(c);
  const int64_t blocks = (((int64_t)b.rows << pl) + 255) / 256;
  append_kernel<<<dim3((unsigned)blocks, c.Hkv), 256, 0, st>>>(c, b, static_cast<const char*>(K), static_cast<const char*>(V), sh, st_, pl);
  return launched();
}

sl_status paged_span_keys(const PageCache& c, const PagedBatch& b, int S, int n_spans, void* Ks, hipStream_t st) {
  if (b.B == 0) return SL_OK;
  const int chunks = (n_spans + kKeySpans - 1) / kKeySpans;
  span_keys_kernel<<<dim3(b.B, chunks, c.Hkv), 256, 0, st>>>(c, b, S, n_spans, static_cast<char*>(Ks), pieces_log2_of(c));
  return launched();
}

}  // namespace sl
