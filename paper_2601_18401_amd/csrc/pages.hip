// Pages of a KV cache: given out, forked, freed, compacted; new tokens written, span keys gathered.
//
// All of it is data movement and small integers.  What decides who gets which page is one workgroup's
// prefix sums, so that the result does not depend on an order of atomics; what moves data is spread over the chip.
#include <climits>

#include "paged.h"

namespace sl {

namespace {

constexpr int kPlanThreads = 1024;

// Running sum over the lanes of a wavefront, own value included: rows of 16 lanes by shifts, then from row to row.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15 -> rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31 -> rows 2 and 3
  return v;
}
__device__ __forceinline__ int64_t wave_scan(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t y = __shfl_up(v, off, 64);
    if (lane >= off) v += y;
  }
  return v;
}

// Sum of v over the threads before this one; total: over all.  (1024 threads; turn alternates between calls, so that one
// barrier a call is enough: a turn's sums are written again behind the barrier of the call between.)
template <typename I>
__device__ __forceinline__ I scan_before(I v, I (*s_wave)[kPlanThreads / 64], int turn, I* total) {
  const int wave = threadIdx.x >> 6;
  const I x = wave_scan(v);
  if ((threadIdx.x & 63) == 63) s_wave[turn][wave] = x;
  __syncthreads();
  I before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const I y = s_wave[turn][w];
    if (w < wave) before += y;
    all += y;
  }
  *total = all;
  return before + x - v;
}

// Reference counts a thread looks at in a pass: 4 to begin with, 16 in large pools, whose passes are many.  (The planning kernels run
// once through their code, most of the time waiting for it: what is unrolled for nothing is paid for.  Eight forks in a
// cache of 3000 pages: 11.7 us with 16 and the list's loops unrolled, 20 KB of code.)
constexpr int kLargePool = 65536;

// refs[at .. at + PER - 1], 1 where there is no page: such are not free
template <int PER>
__device__ __forceinline__ void load_refs(const int32_t* __restrict__ refs, int at, int n, int (&r)[PER]) {
  if (at + PER <= n) {
#pragma unroll
    for (int i = 0; i < PER / 4; ++i) {
      const int4 x = reinterpret_cast<const int4*>(refs + at)[i];
      r[4 * i] = x.x;
      r[4 * i + 1] = x.y;
      r[4 * i + 2] = x.z;
      r[4 * i + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) r[i] = at + i < n ? refs[at + i] : 1;
  }
}

// Pages for new tokens (FORK: for copies of partly filled pages).  s_end[i]: pages that entries 0 .. i need together (I: a
// type that holds it); an entry is served if the free pages reach that far.  The counts are scanned from the front, a pass at a
// time, until the last page is found; a pass lists its free pages in LDS, and a thread then takes each to its entry.
// Chains of loads and barriers bound it, not bytes: the first counts are asked for before the entries, and an entry's lengths at once.
template <bool FORK, typename I, int PER>
__global__ __launch_bounds__(kPlanThreads) void plan_pages_kernel(const PageCache c, const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ seqs, const int32_t* __restrict__ cu,
                                                                  int n, int32_t* __restrict__ ok) {
  constexpr int kPass = kPlanThreads * PER;
  __shared__ I s_end[SL_MAX_PAGE_OPS];
  __shared__ int32_t s_seq[SL_MAX_PAGE_OPS];
  __shared__ int32_t s_have[SL_MAX_PAGE_OPS];  // tokens held (FORK: by the source); -1: not to be served
  __shared__ I s_sums[2][kPlanThreads / 64];
  __shared__ int32_t s_counts[2][kPlanThreads / 64];
  // The first entry of every sequence (an open hash of twice as many places as entries), then a pass's free pages.
  constexpr int kPlaces = 2 * SL_MAX_PAGE_OPS;
  __shared__ __align__(16) int32_t s_shared[2 * kPlaces > kPass ? 2 * kPlaces : kPass];
  int32_t *const s_key = s_shared, *const s_first = s_shared + kPlaces, *const s_free = s_shared;
  const int most = c.max_pages * c.ps;
  int r[PER];
  load_refs<PER>(c.refs, threadIdx.x * PER, c.n_pages, r);
#pragma unroll 1
  for (int k = threadIdx.x; k < 2 * kPlaces / 4; k += kPlanThreads) reinterpret_cast<int4*>(s_shared)[k] = make_int4(-1, -1, -1, -1);
  __syncthreads();
  auto place_of = [&](int s) {
    uint32_t at = (uint32_t)s * 2654435761u / (0x100000000ull / kPlaces);
    for (;; at = (at + 1) % kPlaces) {
      const int there = atomicCAS(&s_key[at], -1, s);
      if (there == -1 || there == s) return at;
    }
  };
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int s = seqs[i];
    s_seq[i] = s;
    if ((uint32_t)s < (uint32_t)c.n_seqs) atomicMin(reinterpret_cast<uint32_t*>(&s_first[place_of(s)]), (uint32_t)i);
  }
  __syncthreads();
  I total = 0;
  int turn = 0;
#pragma unroll 1
  for (int at = 0; at < n; at += kPlanThreads, turn ^= 1) {
    const int i = at + threadIdx.x;
    int have = -1, need = 0;
    if (i < n) {
      const int s = s_seq[i];
      if ((uint32_t)s < (uint32_t)c.n_seqs && s_first[place_of(s)] == i) {
        const int len = c.lens[s];
        if (FORK) {
          const int from = src[i];
          const int held = (uint32_t)from < (uint32_t)c.n_seqs && from != s ? c.lens[from] : -1;
          if (len == 0 && held <= most) have = held;
          need = (uint32_t)held != (uint32_t)held / c.by_ps * c.ps;
        } else {
          const int64_t add = (int64_t)cu[i + 1] - cu[i];
          if (len >= 0 && add >= 0 && len + add <= most) have = len;
          need = (int)((uint32_t)(len + (int)add + c.ps - 1) / c.by_ps - (uint32_t)(len + c.ps - 1) / c.by_ps);
        }
      }
    }
    if (have < 0) need = 0;
    I all;
    const I end = total + scan_before<I>(need, s_sums, turn, &all) + need;
    if (i < n) {
      s_end[i] = end;
      s_have[i] = have;
    }
    total += all;
  }
  // free pages, in order, to the entries
  I found = 0;
#pragma unroll 1
  for (int64_t base = 0; base < c.n_pages && found < total; base += kPass, turn ^= 1) {
    int next[PER];
    const int64_t ahead = base + kPass;
    if (ahead < c.n_pages) load_refs<PER>(c.refs, (int)min(ahead + threadIdx.x * PER, (int64_t)c.n_pages), c.n_pages, next);
    int mine = 0, all;
#pragma unroll
    for (int k = 0; k < PER; ++k) mine += r[k] <= 0;
    int rank = scan_before<int>(mine, s_counts, turn, &all);
    const I left = total - found;
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (r[k] <= 0) s_free[rank++] = (int)base + threadIdx.x * PER + k;
    __syncthreads();
    const int upto = left < all ? (int)left : all;
#pragma unroll 1
    for (int k = threadIdx.x; k < upto; k += kPlanThreads) {
      const I place = found + k;
      int lo = 0, hi = n - 1;
      while (lo < hi) {  // the entry that gets it: the first with end > place
        const int mid = (lo + hi) >> 1;
        if (s_end[mid] > place) hi = mid;
        else lo = mid + 1;
      }
      const I first = lo ? s_end[lo - 1] : 0;
      const int page = s_free[k], at = FORK ? (int)((uint32_t)s_have[lo] / c.by_ps) : (int)((uint32_t)(s_have[lo] + c.ps - 1) / c.by_ps) + (int)(place - first);
      c.tables[(int64_t)s_seq[lo] * c.max_pages + at] = page;
      c.refs[page] = 1;
    }
    found += all;
    if (ahead < c.n_pages) {
#pragma unroll
      for (int k = 0; k < PER; ++k) r[k] = next[k];
      __syncthreads();  // (s_free is filled again)
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const I first = i ? s_end[i - 1] : 0, end = s_end[i];
    const int have = s_have[i];
    const bool served = have >= 0 && (end == first || end <= found);
    if (served) {
      c.lens[s_seq[i]] = FORK ? have : have + cu[i + 1] - cu[i];
    } else if (!FORK && have >= 0) {  // the entry at which the pages ran out gives back what it got
      for (I k = first; k < found && k < end; ++k) {
        int32_t* const t = c.tables + (int64_t)s_seq[i] * c.max_pages + (uint32_t)(have + c.ps - 1) / c.by_ps + (int)(k - first);
        c.refs[*t] = 0;
        *t = -1;
      }
    }
    ok[i] = served;
  }
}

__global__ __launch_bounds__(256) void served_kernel(const int32_t* seqs, const int32_t* ok, int n, int32_t* served) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) served[i] = ok[i] ? seqs[i] : -1;
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
      x[u] = load16_stream(from + (q >> pieces_log2) * row_bytes + (q & mask) * 16);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = p + u * threads;
      store16_stream(to + (q >> pieces_log2) * row_bytes + (q & mask) * 16, x[u]);
    }
  }
  for (; p < n; p += threads)
    *reinterpret_cast<uint4*>(to + (p >> pieces_log2) * row_bytes + (p & mask) * 16) =
        load16(from + (p >> pieces_log2) * row_bytes + (p & mask) * 16);
}

__host__ __device__ inline int element_bytes(const PageCache& c) { return c.fp4 ? 1 : c.dtype == SL_BF16 ? 2 : 4; }
// 16-byte pieces of a row: 8, 16 or 32; of a row's codes 2 or 4
__host__ __device__ inline int pieces_log2_of(const PageCache& c) {
  return (c.D == 128 ? 4 : 3) + (c.fp4 ? -2 : c.dtype == SL_BF16 ? 0 : 1);
}

// One (layer, K or V, head) part of a page: unit in [0, layers * 2 * Hkv).  Pieces of kCopyRows rows count in 32 bits (pages may have 2^30).
constexpr int kCopyRows = 1 << 24;
__device__ __forceinline__ void copy_part(const PageCache& c, int from, int to, int unit, int rows, int thread, int threads) {
  const int es = element_bytes(c);
  const int head = unit % c.Hkv, lt = unit / c.Hkv;
  char* const base = reinterpret_cast<char*>(lt & 1 ? c.V : c.K) + ((lt >> 1) * c.layer + head * c.head) * es;
  const int64_t row_bytes = c.tok * es;
#pragma unroll 1
  for (int row = 0; row < rows; row += kCopyRows)
    copy_rows(base + from * c.page * es + row * row_bytes, base + to * c.page * es + row * row_bytes, row_bytes, pieces_log2_of(c),
              min(rows - row, kCopyRows), thread, threads);
  if (!c.fp4) return;
  // the rows' scales, which begin at a multiple of 32 bytes: pieces of 16, and what is left, two at a time
  const int64_t at = (int64_t)c.ps * c.tok;
  const char* const s = base + from * c.page + at;
  char* const d = base + to * c.page + at;
  const int64_t n = (int64_t)rows * (c.D / 32);
#pragma unroll 1
  for (int64_t p = thread; p < n >> 4; p += threads) *reinterpret_cast<uint4*>(d + p * 16) = load16(s + p * 16);
#pragma unroll 1
  for (int64_t p = (n >> 4 << 3) + thread; p < n >> 1; p += threads)
    *reinterpret_cast<uint16_t*>(d + p * 2) = *reinterpret_cast<const uint16_t*>(s + p * 2);
}

constexpr int kForkEntries = 1024;  // table entries of a workgroup

// What plan_pages_kernel<true> decided: dst's table from src's, references, the copied last page.  The first fork of a source adds the
// references of all (200 forks of 16 sequences: 240000 atomics otherwise, of which as many wait for each other as forks share a source).
__global__ __launch_bounds__(256) void fork_kernel(const PageCache c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                   const int32_t* __restrict__ ok, int n, int chunks) {
  const int f = blockIdx.x, y = blockIdx.y;
  if (!ok[f]) return;
  const int s = src[f], d = dst[f], len = c.lens[d];
  const int full = (uint32_t)len / c.by_ps, part = len - full * c.ps;
  const int32_t* const from = c.tables + (int64_t)s * c.max_pages;
  int32_t* const to = c.tables + (int64_t)d * c.max_pages;
  if (y < chunks) {
    if (y * kForkEntries >= full) return;
    __shared__ int s_forks, s_first;
    if (threadIdx.x == 0) {
      s_forks = 0;
      s_first = n;
    }
    __syncthreads();
    int forks = 0, first = n;
    for (int k = threadIdx.x; k < n; k += 256)
      if (src[k] == s && ok[k]) {
        ++forks;
        first = min(first, k);
      }
    if (forks) {
      atomicAdd(&s_forks, forks);
      atomicMin(&s_first, first);
    }
    __syncthreads();
    forks = s_first == f ? s_forks : 0;
    for (int k = y * kForkEntries + threadIdx.x; k < full && k < (y + 1) * kForkEntries; k += 256) {
      const int page = from[k];
      to[k] = page;
      if (forks && (uint32_t)page < (uint32_t)c.n_pages) atomicAdd(&c.refs[page], forks);
    }
  } else if (part) {
    const int page = from[full];
    if ((uint32_t)page < (uint32_t)c.n_pages) copy_part(c, page, to[full], y - chunks, part, threadIdx.x, 256);
  }
}

// A sequence listed twice is emptied by its first entry.
__global__ __launch_bounds__(256) void free_kernel(const PageCache c, const int32_t* __restrict__ seqs) {
  const int s = seqs[blockIdx.x];
  if ((uint32_t)s >= (uint32_t)c.n_seqs) return;
  bool earlier = false;
  for (int k = threadIdx.x; k < (int)blockIdx.x; k += 256) earlier = earlier || seqs[k] == s;
  if (__syncthreads_or(earlier)) return;
  if (blockIdx.y == 0 && threadIdx.x == 0) c.lens[s] = 0;
  int32_t* const t = c.tables + (int64_t)s * c.max_pages;
  for (int k = blockIdx.y * kForkEntries + threadIdx.x; k < c.max_pages && k < ((int)blockIdx.y + 1) * kForkEntries; k += 256) {
    const int page = t[k];
    if (page == -1) continue;
    t[k] = -1;
    if ((uint32_t)page < (uint32_t)c.n_pages) atomicSub(&c.refs[page], 1);
  }
}

// The pages that move: pair k is moves[k] -> moves[half + k], k < *count.  The first pass's counts stay in registers between the two
// looks at them, and up to 4096 pairs in LDS: a round trip to memory is a tenth of a small cache's plan.
constexpr int kKeptMoves = 4096;
template <int PER>
__global__ __launch_bounds__(kPlanThreads) void plan_compact_kernel(const PageCache c, int32_t* __restrict__ map, int32_t* __restrict__ count,
                                                                    int32_t* __restrict__ moves, int half) {
  __shared__ int32_t s_sums[2][kPlanThreads / 64];
  __shared__ int32_t s_from[kKeptMoves], s_to[kKeptMoves], s_refs[kKeptMoves];
  constexpr int64_t kPass = kPlanThreads * PER;
  int first[PER], r[PER];
  auto place = [&](int64_t base) { return (int)min(base + threadIdx.x * PER, (int64_t)c.n_pages); };
  load_refs<PER>(c.refs, place(0), c.n_pages, first);
  int used = 0, n, turn = 0;
#pragma unroll 1
  for (int64_t base = 0; base < c.n_pages; base += kPass) {
    const int at = place(base);
    if (base > 0) load_refs<PER>(c.refs, at, c.n_pages, r);
#pragma unroll
    for (int k = 0; k < PER; ++k) used += at + k < c.n_pages && (base > 0 ? r[k] : first[k]) > 0;
  }
  scan_before<int>(used, s_sums, turn, &n);
  int holes = 0, movers = 0;  // so far
#pragma unroll
  for (int k = 0; k < PER; ++k) r[k] = first[k];
#pragma unroll 1
  for (int64_t base = 0; base < c.n_pages; base += kPass) {
    const int at = place(base);
    if (base > 0) load_refs<PER>(c.refs, at, c.n_pages, r);
    int both = 0, all;  // holes, and movers in the upper half: 16384 of a pass at most
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      both += at + k < n && r[k] <= 0;
      both += (at + k >= n && at + k < c.n_pages && r[k] > 0) << 16;
    }
    const uint32_t before = (uint32_t)scan_before<int>(both, s_sums, turn ^= 1, &all);
    int hk = holes + (int)(before & 0xffff), mk = movers + (int)(before >> 16);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int p = at + k;
      if (p >= c.n_pages) continue;
      const bool on = r[k] > 0;
      if (!on || p < n) map[p] = on ? p : -1;
      if (p < n && !on) {
        if (hk < kKeptMoves) s_to[hk] = p;
        moves[half + hk++] = p;
      }
      if (p >= n && on) {
        if (mk < kKeptMoves) {
          s_from[mk] = p;
          s_refs[mk] = r[k];
        }
        moves[mk++] = p;
      }
    }
    holes += (uint32_t)all & 0xffff;
    movers += (uint32_t)all >> 16;
  }
  if (threadIdx.x == 0) *count = movers;
  __syncthreads();  // (also orders the workgroup's own writes to moves before the reads)
#pragma unroll 1
  for (int k = threadIdx.x; k < movers; k += kPlanThreads) {
    const bool near = k < kKeptMoves;
    const int from = near ? s_from[k] : moves[k], to = near ? s_to[k] : moves[half + k], refs = near ? s_refs[k] : c.refs[from];
    map[from] = to;
    c.refs[to] = refs;
    c.refs[from] = 0;
  }
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

// A workgroup takes 32 rows of a head: a lane for each row finds its place, then all lanes copy, 16 bytes at a time.  Bound by memory:
// 120000 rows of 8 heads at 5.1 TB/s, where a large copy reaches 4.9 to 5.2; without the non-temporal hint 4.9, with every 16 bytes finding
// their own place 4.6.
constexpr int kAppendRows = 32;
__global__ __launch_bounds__(256) void append_kernel(const PageCache c, const PagedBatch b, const char* __restrict__ K,
                                                     const char* __restrict__ V, int64_t sh, int64_t st, int pieces_log2) {
  __shared__ int64_t s_to[kAppendRows];
  const int first = blockIdx.x * kAppendRows, head = blockIdx.y, es = element_bytes(c);
  if (threadIdx.x < kAppendRows) {
    const int row = first + threadIdx.x;
    int64_t to = -1;
    if (row < b.rows && row >= b.cu[0] && row < b.cu[b.B]) {
      const int e = entry_of_row(b.cu, b.B, row), s = b.seqs[e], len = length_of(c, s), t = len - (b.cu[e + 1] - row);
      if (t >= 0 && t < b.L && t < len) {
        const int k = (uint32_t)t / c.by_ps, page = c.tables[(int64_t)s * c.max_pages + k];
        // (a page of several sequences holds tokens of each, whatever the batch says of this one)
        if ((uint32_t)page < (uint32_t)c.n_pages && c.refs[page] <= 1)
          to = (b.layer * c.layer + page * c.page + head * c.head + (t - k * c.ps) * c.tok) * es;
      }
    }
    s_to[threadIdx.x] = to;
  }
  __syncthreads();
  const char *const k0 = K + (head * sh + first * st) * es, *const v0 = V + (head * sh + first * st) * es;
  const int n = kAppendRows << pieces_log2, mask = (1 << pieces_log2) - 1;
  constexpr int U = 2;  // of K and as many of V: rows have 8, 16 or 32 pieces, so that n is a multiple of 256, if not of 512
  for (int p = threadIdx.x; p < n; p += U * 256) {
    uint4 x[U], y[U];
    int64_t to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = p + u * 256, row = q >> pieces_log2;
      to[u] = q < n ? s_to[row] : -1;
      if (to[u] < 0) continue;
      const int64_t from = row * st * es + (q & mask) * 16;
      x[u] = load16_stream(k0 + from);
      y[u] = load16_stream(v0 + from);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (to[u] < 0) continue;
      const int64_t at = to[u] + ((p + u * 256) & mask) * 16;
      store16_stream(reinterpret_cast<char*>(c.K) + at, x[u]);
      store16_stream(reinterpret_cast<char*>(c.V) + at, y[u]);
    }
  }
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

template <bool FORK, typename I>
static void plan_pages(const PageCache& c, const int32_t* src, const int32_t* seqs, const int32_t* cu, int n, int32_t* ok, hipStream_t st) {
  if (c.n_pages > kLargePool) plan_pages_kernel<FORK, I, 16><<<1, kPlanThreads, 0, st>>>(c, src, seqs, cu, n, ok);
  else plan_pages_kernel<FORK, I, 4><<<1, kPlanThreads, 0, st>>>(c, src, seqs, cu, n, ok);
}

sl_status pages_extend(const PageCache& c, const PagedBatch& b, int32_t* ok, hipStream_t st) {
  if (b.B == 0) return SL_OK;
  // (an entry's need is at most a table's width)
  if ((int64_t)b.B * c.max_pages < INT_MAX) plan_pages<false, int>(c, nullptr, b.seqs, b.cu, b.B, ok, st);
  else plan_pages<false, int64_t>(c, nullptr, b.seqs, b.cu, b.B, ok, st);
  return launched();
}

sl_status pages_served(const int32_t* seqs, const int32_t* ok, int n, int32_t* served, hipStream_t st) {
  if (n == 0) return SL_OK;
  served_kernel<<<(n + 255) / 256, 256, 0, st>>>(seqs, ok, n, served);
  return launched();
}

sl_status pages_fork(const PageCache& c, const int32_t* src, const int32_t* dst, int n, int32_t* ok, hipStream_t st) {
  if (n == 0) return SL_OK;
  plan_pages<true, int>(c, src, dst, nullptr, n, ok, st);
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
  if (c.n_pages > kLargePool) plan_compact_kernel<16><<<1, kPlanThreads, 0, st>>>(c, map, count, moves, half);
  else plan_compact_kernel<4><<<1, kPlanThreads, 0, st>>>(c, map, count, moves, half);
  const int64_t entries = (int64_t)c.n_seqs * c.max_pages, units = (int64_t)(half - 1) * c.layers * 2 * c.Hkv;
  const int tables = (int)min((entries + 1023) / 1024, (int64_t)512), copies = (int)min(units, (int64_t)8192);
  compact_kernel<<<tables + copies, 256, 0, st>>>(c, map, count, moves, half, tables);
  return launched();
}

sl_status paged_append(const PageCache& c, const PagedBatch& b, const void* K, const void* V, int64_t sh, int64_t st_, hipStream_t st) {
  if (b.B == 0 || b.rows == 0) return SL_OK;
  if (c.fp4) return paged_append_fp4(c, b, K, V, sh, st_, st);
  const int pl = pieces_log2_of(c);
  append_kernel<<<dim3((unsigned)((b.rows + kAppendRows - 1) / kAppendRows), c.Hkv), 256, 0, st>>>(c, b, static_cast<const char*>(K), static_cast<const char*>(V), sh, st_, pl);
  return launched();
}

sl_status paged_span_keys(const PageCache& c, const PagedBatch& b, int S, int n_spans, void* Ks, hipStream_t st) {
  if (b.B == 0) return SL_OK;
  if (c.fp4) return paged_span_keys_fp4(c, b, S, n_spans, Ks, st);
  const int chunks = (n_spans + kKeySpans - 1) / kKeySpans;
  span_keys_kernel<<<dim3(b.B, chunks, c.Hkv), 256, 0, st>>>(c, b, S, n_spans, static_cast<char*>(Ks), pieces_log2_of(c));
  return launched();
}

}  // namespace sl
