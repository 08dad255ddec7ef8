// Span-attention of new tokens over a paged cache.
//
// A row's keys are the tokens of its selected spans and of its window.  They are cut into pieces; a piece's softmax gives
// a normalised output and a log-sum-exp (in log2 units), and a merge joins a row's pieces: exp2(lse_p - lse) of each for the
// joint form, and for the gated one alpha_t * exp2(lse_p - lse_t) summed over the slots t that the piece belongs to.
#include <climits>
#include <mutex>
#include <type_traits>

#include "paged.h"

namespace sl {

namespace {

struct Pieces {
  int routed, routed_tokens;  // of a span, and tokens of one
  int window, window_tokens;  // of the window
  int count;                  // of a row: topk * routed + window
};

struct PagedArgs {
  PageCache c;
  PagedBatch b;
  PagedAttention a;
  Pieces p;
  const void* Q;
  const int32_t* idx;
  const float* scores;
  void* O;
  float* LSE;
  void* part_o;       // [Hq * rows][count][D], see Record
  float* part_lse;    // [Hq * rows][count] log2-sum-exp2; -inf: no token, and no output
  float* part_scale;  // [Hq * rows][count] of bf16 calls
  float scale_log2e;
  bool marks;  // tiles write the records, and may have marked some
};

// Tiles of the matrix-core form.
struct TilePlan {
  int tiles;             // window tiles of a kv head
  int64_t window_units;  // tiles * pieces of a window * Hkv
  int64_t units;         // ... and the spans' pieces: workgroups that have something to do
  int spans, buckets;    // spans of the longest sequence; B * Hkv * spans
  int32_t *counts, *first_tile;  // [buckets]
  int most_tiles;  // of the buckets; a multiple of 8
  int4* records;   // [most_tiles] in the order of the workgroups: {span, entry * Hkv + kv head, place of the tile, items; 0: no tile}
  int32_t *ranks;  // [Hq * rows * topk] an item's place in its bucket, -1 for empty slots
  int32_t *items;  // [most_tiles][cols] (row and head) * 32 + slot
};

__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }  // NaN stays
// exp2(a - b) where a = -inf means nothing, also beside b = -inf
__device__ __forceinline__ float weight_of(float a, float b) { return a == -INFINITY ? 0.f : fast_exp2(a - b); }

// Grids of more than 2^20 workgroups go on in y (a launch holds fewer than 2^32 threads in x).
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// A piece's normalised output: fp32, or for bf16 calls fp16 beside a power of two above the row's largest value: half the
// bytes, off by up to 2^-11 of the largest value, where rounding the result to bf16 costs 2^-8 (and bf16 here would cost as much again).
template <typename T>
struct Record {
  typedef float Value;
};
template <>
struct Record<bf16_t> {
  typedef _Float16 Value;
};
// a power of two from the largest of a row's finite values on (half of it at the end of fp32's range)
__device__ __forceinline__ float scale_above(float largest) {
  const int e = __builtin_amdgcn_frexp_expf(largest);
  return largest > 0.f ? ldexpf(1.f, e < -100 ? -100 : e > 127 ? 127 : e) : 1.f;
}

// An entry of the batch as a wavefront sees it (all lanes alike).
struct Entry {
  int e, s, len;  // entry, sequence and its length (-1: no such sequence)
  int r0, r1;     // cu[e], cu[e + 1]
};
// The last entry e with before(cu[e], e), which holds for entry 0 and up to some entry: 64 of them are looked at at once, with all that
// is asked of the one that is found.  (A binary search is a chain of loads: a piece of 64 tokens took as long to find as to attend.)
template <typename F>
__device__ __forceinline__ Entry find_entry(const PagedArgs& x, F&& before) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = x.b.B;
  while (n > 64) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    const bool in = at < lo + n && before(x.b.cu[min(at, x.b.B - 1)], at);
    const int k = max(__popcll(__builtin_amdgcn_ballot_w64(in)) - 1, 0);
    n = min(step, n - k * step);
    lo += k * step;
  }
  const int at = min(lo + lane, x.b.B - 1);
  const int cu = x.b.cu[at], r0 = max(cu, 0), r1 = x.b.cu[at + 1], s = x.b.seqs[at], len = length_of(x.c, s);
  const int k = max(__popcll(__builtin_amdgcn_ballot_w64(lane < n && before(cu, at))) - 1, 0);
  return {lo + k, __builtin_amdgcn_readlane(s, k), __builtin_amdgcn_readlane(len, k), __builtin_amdgcn_readlane(r0, k),
          __builtin_amdgcn_readlane(r1, k)};
}
__device__ __forceinline__ Entry entry_with_row(const PagedArgs& x, int row) {
  return find_entry(x, [=](int r0, int) { return r0 <= row; });
}
// position of a row; < 0: a row without a token
__device__ __forceinline__ int position_of(const PagedArgs& x, const Entry& e, int row) {
  const int pos = e.len - (e.r1 - row);
  return pos >= e.len || pos >= x.b.L ? -1 : pos;
}

// ------------------------------------------------------------------ row by row
// One wavefront, one query, one piece: LPR lanes cover a row of K or V with 16 bytes each, RPW rows per instruction, every
// row group with its own running maximum and sum.
template <typename T, int D>
struct RowState {
  static constexpr int EPL = RowLayout<T, D>::EPL, LPR = RowLayout<T, D>::LPR, RPW = RowLayout<T, D>::RPW;
  float m, l, o[EPL];
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[e] = 0.f;
  }
  __device__ __forceinline__ void scale_to(float to) {
    const float f = weight_of(m, to);
    l *= f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[e] *= f;
    m = to;
  }
  // tokens [t0, t1) of the sequence whose table is given
  template <int U>
  __device__ __forceinline__ void attend(const PageCache& c, const T* K, const T* V, const int32_t* table, const float (&q)[EPL], int t0,
                                         int t1, int lane) {
    const int g = lane / LPR, lr = lane % LPR;
    int page[U];
    auto look_up = [&](int tb) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = tb + u * RPW + g;
        page[u] = t < t1 ? table[(uint32_t)t / c.by_ps] : -1;
      }
    };
    look_up(t0);
    for (int tb = t0; tb < t1; tb += RPW * U) {
      uint4 kr[U], vr[U];
      bool on[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = tb + u * RPW + g;
        on[u] = t < t1 && (uint32_t)page[u] < (uint32_t)c.n_pages;
        kr[u] = vr[u] = make_uint4(0, 0, 0, 0);
        if (on[u]) {
          const int64_t at = page[u] * c.page + (int64_t)((uint32_t)t - (uint32_t)t / c.by_ps * c.ps) * c.tok + lr * EPL;
          kr[u] = load16_stream(K + at);
          vr[u] = load16_stream(V + at);
        }
      }
      if (tb + RPW * U < t1) look_up(tb + RPW * U);
      float s[U], top = m;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float kf[EPL], acc = 0.f;
        Elem<T>::unpack(kr[u], kf);
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc = fmaf(q[e], kf[e], acc);
        acc = group_sum<LPR>(acc);
        s[u] = on[u] ? acc : -INFINITY;
        top = max_of(top, s[u]);
      }
      if (top == -INFINITY) continue;
      scale_to(top);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float p = fast_exp2(s[u] - m);
        l += p;
        float vf[EPL];
        Elem<T>::unpack(vr[u], vf);
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[e] = fmaf(p, vf[e], o[e]);
      }
    }
  }
  // the row groups' states into one, in every lane
  __device__ __forceinline__ void join_groups() {
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1) {
      const float mo = __shfl_xor(m, off, 64);
      const float to = max_of(m, mo);
      if (to == -INFINITY) continue;
      scale_to(to);
      l += __shfl_xor(l, off, 64);
#pragma unroll
      for (int e = 0; e < EPL; ++e) o[e] += __shfl_xor(o[e], off, 64);
    }
  }
};

// Piece `part` of a row as tokens [t0, t1); slots that hold no span have none.
struct PieceRange {
  int t0, t1;
};
__device__ __forceinline__ PieceRange range_of_piece(const PagedArgs& x, int pos, int part, const int32_t* slots) {
  const int S = x.a.S, c = pos / S;
  const int slot = part / x.p.routed;
  if (slot < x.a.topk) {
    const int j = slots[slot];
    if (j < 0 || j >= c) return {0, 0};
    const int t0 = j * S + (part - slot * x.p.routed) * x.p.routed_tokens, end = (j + 1) * S;
    return {t0, min(t0 + x.p.routed_tokens, end)};
  }
  const int64_t t0 = (int64_t)c * S + (int64_t)(part - x.a.topk * x.p.routed) * x.p.window_tokens;
  return {(int)min(t0, (int64_t)pos + 1), (int)min(t0 + x.p.window_tokens, (int64_t)pos + 1)};
}

// One piece of a row and head by `WAVES` wavefronts of a workgroup, a run of its tokens each, to its record (or, DIRECT, to the
// row's result).  s_o, s_ml: [WAVES][D] and [WAVES][2] of LDS.
template <typename T, int D, int WAVES, bool DIRECT>
__device__ __forceinline__ void take_piece(const PagedArgs& x, int s, int rh, const PieceRange& r, int64_t rec, float* s_o, float* s_ml) {
  using RS = RowState<T, D>;
  const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : threadIdx.x >> 6;
  const int h = rh / x.b.rows, row = rh - h * x.b.rows;
  constexpr int RUN = 4 * RS::RPW;
  const int run = ((r.t1 - r.t0 + WAVES - 1) / WAVES + RUN - 1) / RUN * RUN;
  const int t0 = r.t0 + wave * run, t1 = min(t0 + run, r.t1);
  RS st;
  st.clear();
  if (t0 < t1) {
    float q[RS::EPL];
    Elem<T>::unpack(load16(static_cast<const T*>(x.Q) + h * x.a.qsh + row * x.a.qst + lane % RS::LPR * RS::EPL), q);
#pragma unroll
    for (int e = 0; e < RS::EPL; ++e) q[e] *= x.scale_log2e;
    const int64_t base = x.b.layer * x.c.layer + h / x.a.G * x.c.head;
    st.template attend<4>(x.c, static_cast<const T*>(x.c.K) + base, static_cast<const T*>(x.c.V) + base,
                          x.c.tables + (int64_t)s * x.c.max_pages, q, t0, t1, lane);
    st.join_groups();
  }
  float m = st.m, l = st.l;
  if (WAVES > 1) {
    if (lane == 0) {
      s_ml[2 * wave] = m;
      s_ml[2 * wave + 1] = l;
    }
    if (lane < RS::LPR) {
#pragma unroll
      for (int e = 0; e < RS::EPL; ++e) s_o[wave * D + lane * RS::EPL + e] = st.o[e];
    }
    __syncthreads();
    if (wave != 0) return;
    m = s_ml[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = max_of(m, s_ml[2 * w]);
    l = 0.f;
#pragma unroll
    for (int e = 0; e < RS::EPL; ++e) st.o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = weight_of(s_ml[2 * w], m);
      if (s_ml[2 * w] == -INFINITY) continue;
      l = fmaf(f, s_ml[2 * w + 1], l);
#pragma unroll
      for (int e = 0; e < RS::EPL; ++e) st.o[e] = fmaf(f, s_o[w * D + lane % RS::LPR * RS::EPL + e], st.o[e]);
    }
  }
  const bool none = m == -INFINITY;
  const float lse = none ? m : m + __log2f(l), inv = none ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < RS::EPL; ++e) st.o[e] *= inv;
  if (DIRECT) {
    if (lane == 0 && x.LSE) x.LSE[rh] = lse * kLn2;
    if (lane < RS::LPR)
#pragma unroll
      for (int e = 0; e < RS::EPL; ++e) Elem<T>::store1(static_cast<T*>(x.O) + (int64_t)rh * D + lane * RS::EPL + e, none ? 0.f : st.o[e]);
    return;
  }
  if (lane == 0) x.part_lse[rec] = lse;
  if (none) return;
  typedef typename Record<T>::Value Value;
  typedef Value Values __attribute__((ext_vector_type(RS::EPL)));
  float by = 1.f;
  if (sizeof(Value) == 2) {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < RS::EPL; ++e) top = fmaxf(top, fabsf(st.o[e]) < INFINITY ? fabsf(st.o[e]) : 0.f);
#pragma unroll
    for (int off = 1; off < RS::LPR; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const float scale = scale_above(top);
    if (lane == 0) x.part_scale[rec] = scale;
    by = 1.f / scale;
  }
  Values v;
#pragma unroll
  for (int e = 0; e < RS::EPL; ++e) v[e] = (Value)(st.o[e] * by);
  if (lane < RS::LPR) *reinterpret_cast<Values*>(static_cast<Value*>(x.part_o) + rec * D + lane * RS::EPL) = v;
}

// Workgroup u takes piece u % count of row-and-head u / count.
template <typename T, int D>
__global__ __launch_bounds__(256) void rows_kernel(const PagedArgs x) {
  __shared__ float s_o[4 * D], s_ml[8];
  const int64_t u = workgroup();
  if (u >= (int64_t)x.a.Hq * x.b.rows * x.p.count) return;
  const int rh = (int)(u / x.p.count), part = (int)(u - (int64_t)rh * x.p.count);
  const int h = rh / x.b.rows, row = rh - h * x.b.rows;
  const Entry at = entry_with_row(x, row);
  if (row < at.r0 || row >= at.r1) return;
  const int pos = position_of(x, at, row);
  const PieceRange r = pos < 0 ? PieceRange{0, 0} : range_of_piece(x, pos, part, x.idx + h * x.a.ish + row * x.a.ist);
  take_piece<T, D, 4, false>(x, at.s, rh, r, (int64_t)rh * x.p.count + part, s_o, s_ml);
}

// All pieces of a row and head by one workgroup, whose four wavefronts share out the spans and cut the window in four: no
// records, no merge.  Where there are rows enough to fill the chip (1000 rows and heads of 290 tokens: 33 -> 25 us).
template <typename T, int D>
__global__ __launch_bounds__(256) void whole_rows_kernel(const PagedArgs x) {
  using RS = RowState<T, D>;
  constexpr int RUN = 4 * RS::RPW;
  __shared__ float s_o[4][D], s_ml[4][2];
  if (workgroup() >= (int64_t)x.a.Hq * x.b.rows) return;
  const int rh = (int)workgroup(), lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane % RS::LPR;
  const int h = rh / x.b.rows, row = rh - h * x.b.rows;
  // asked for at once: the query, the slots and their scores, the row's entry
  float q[RS::EPL];
  Elem<T>::unpack(load16(static_cast<const T*>(x.Q) + h * x.a.qsh + row * x.a.qst + lr * RS::EPL), q);
  const int64_t at_slots = h * x.a.ish + row * x.a.ist;
  int slot = lane < x.a.topk ? x.idx[at_slots + lane] : -1;
  float score = x.a.combined && lane < x.a.topk ? x.scores[at_slots + lane] : -INFINITY;
  const Entry at = entry_with_row(x, row);
  if (row < at.r0 || row >= at.r1) return;
  const int pos = position_of(x, at, row), c = pos < 0 ? 0 : pos / x.a.S;
  if (slot >= c) slot = -1;
#pragma unroll
  for (int e = 0; e < RS::EPL; ++e) q[e] *= x.scale_log2e;
  const int64_t base = x.b.layer * x.c.layer + h / x.a.G * x.c.head;
  const T *const K = static_cast<const T*>(x.c.K) + base, *const V = static_cast<const T*>(x.c.V) + base;
  const int32_t* const table = x.c.tables + (int64_t)max(at.s, 0) * x.c.max_pages;
  RS st;
  st.clear();
  auto spans = [&](int k) {  // slot k's span, by this wavefront
    const int j = __builtin_amdgcn_readlane(slot, k);
    if (j >= 0) st.template attend<4>(x.c, K, V, table, q, j * x.a.S, (j + 1) * x.a.S, lane);
  };
  if (!x.a.combined)
    for (int k = wave; k < x.a.topk; k += 4) spans(k);
  if (pos >= 0) {
    const int t0 = c * x.a.S, run = ((pos + 1 - t0 + 3) / 4 + RUN - 1) / RUN * RUN, from = t0 + wave * run;
    st.template attend<4>(x.c, K, V, table, q, from, min(from + run, pos + 1), lane);
  }
  st.join_groups();
  // the wavefronts' states into one, in every wavefront
  if (lane == 0) {
    s_ml[wave][0] = st.m;
    s_ml[wave][1] = st.l;
  }
  if (lane < RS::LPR)
#pragma unroll
    for (int e = 0; e < RS::EPL; ++e) s_o[wave][lr * RS::EPL + e] = st.o[e];
  __syncthreads();
  float m = s_ml[0][0], l = 0.f, o[RS::EPL];
#pragma unroll
  for (int w = 1; w < 4; ++w) m = max_of(m, s_ml[w][0]);
#pragma unroll
  for (int e = 0; e < RS::EPL; ++e) o[e] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (s_ml[w][0] == -INFINITY) continue;
    const float f = weight_of(s_ml[w][0], m);
    l = fmaf(f, s_ml[w][1], l);
#pragma unroll
    for (int e = 0; e < RS::EPL; ++e) o[e] = fmaf(f, s_o[w][lr * RS::EPL + e], o[e]);
  }
  const bool gated = x.a.combined && __builtin_amdgcn_ballot_w64(slot >= 0) != 0;
  if (!gated) {
    if (wave != 0) return;
    const bool none = m == -INFINITY;
    const float inv = none ? 0.f : 1.f / l;
    if (lane == 0 && x.LSE) x.LSE[rh] = none ? -INFINITY : (m + __log2f(l)) * kLn2;
    if (lane < RS::LPR)
#pragma unroll
      for (int e = 0; e < RS::EPL; ++e)
        Elem<T>::store1(static_cast<T*>(x.O) + (int64_t)rh * D + lr * RS::EPL + e, none ? 0.f : o[e] * inv);
    return;
  }
  // m, l, o: the window.  Each slot's softmax goes over its span and the window.
  if (slot < 0) score = -INFINITY;
  float top = score;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) top = max_of(top, __shfl_xor(top, off, 64));
  const float gate = slot >= 0 ? fast_exp2((score - top) * kLog2e) : 0.f;
  float sum = gate, acc[RS::EPL];
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
#pragma unroll
  for (int e = 0; e < RS::EPL; ++e) acc[e] = 0.f;
  for (int k = wave; k < x.a.topk; k += 4) {
    const float alpha = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(gate / sum), k));
    if (alpha == 0.f) continue;
    st.clear();
    spans(k);
    st.join_groups();
    const float to = max_of(st.m, m);
    if (to == -INFINITY) continue;
    const float mine = weight_of(st.m, to), near = weight_of(m, to), by = alpha / (mine * st.l + near * l);
#pragma unroll
    for (int e = 0; e < RS::EPL; ++e) acc[e] = fmaf(by, mine * st.o[e] + near * o[e], acc[e]);
  }
  __syncthreads();
  if (lane < RS::LPR)
#pragma unroll
    for (int e = 0; e < RS::EPL; ++e) s_o[wave][lr * RS::EPL + e] = acc[e];
  __syncthreads();
  if (threadIdx.x < D)
    Elem<T>::store1(static_cast<T*>(x.O) + (int64_t)rh * D + threadIdx.x,
                    (s_o[0][threadIdx.x] + s_o[1][threadIdx.x]) + (s_o[2][threadIdx.x] + s_o[3][threadIdx.x]));
}

// ------------------------------------------------------------------ tiles on the matrix cores
// A tile is up to NW * 32 * CB query columns that attend one run of the sequence's tokens, each in a range of its own: rows and heads
// of a kv head's group on their windows, or the rows that list a span.  Both products are taken transposed, so that a lane
// owns a column:
//   S^T[token][column] = K . Q^T      A = K rows from LDS, B = queries in registers
//   O^T[d][column] += V^T . P^T       A = V through transposing LDS reads, B = P^T straight from the S^T accumulators
// (Lane l of a 32x32 result holds column l % 32 and rows 8 (r / 4) + 4 (l / 32) + r % 4.  bf16, 32x32x16: K rows are fed with bits 2 and 3
// of their number swapped, which makes a lane's eight consecutive accumulators eight consecutive tokens.  fp32, 32x32x2: accumulator r of
// the two halves is the pair of tokens that one product of V^T takes.)
// K and V rows come by direct global -> LDS loads, 64 tokens a step in two stages, 16-byte pieces swizzled against bank conflicts.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// Swizzle of a staged row's 16-byte pieces, so that those that lanes read together lie in different banks.
template <typename T, int D>
__device__ __forceinline__ int k_swizzle(int row) {
  return sizeof(T) == 4 ? row & (D / 4 - 1) : D == 128 ? row & 15 : (row >> 1) & 7;
}
template <typename T, int D>
__device__ __forceinline__ int v_swizzle(int row) {
  return sizeof(T) == 4 ? 0 : D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
}

__device__ __forceinline__ float across_halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return max_of(__int_as_float(r[0]), __int_as_float(r[1]));
}
__device__ __forceinline__ float across_halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(r[0]) + __int_as_float(r[1]);
}

// The lane's number, derived where it is used: two blocks of columns leave no register for what can be had again.
__device__ __forceinline__ int lane_now() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(x));
  return x;
}

__device__ uint4 g_zeros[32];  // what a row without a page is read from

#define SL_LDS(p) ((__attribute__((address_space(3))) void*)(p))

// Sixteen rows of a K (TENSOR 0) or V (1) stage: global -> LDS, 1 KB an instruction.
template <typename T, int D>
struct RowLanes {
  static constexpr int LPR = D * (int)sizeof(T) / 16, RPI = 64 / LPR;  // lanes of a row, rows of an instruction
};
template <typename T, int D, int TENSOR>
__device__ __forceinline__ int piece_of(int row, int lane) {
  return lane % RowLanes<T, D>::LPR ^ (TENSOR == 0 ? k_swizzle<T, D>(row) : v_swizzle<T, D>(row));
}
// STREAM: with the non-temporal hint, where a row is read once (one token behind a million 62 -> 56 us, 24 caches of up to 120000 tokens
// 116 -> 103; prompts, whose rows are read by many tiles, 760 -> 802).
// base: row 0 of the sixteen, which lie in one page; rows from `rows` on become zeros (what lies there may be anything, and zero times
// that need not be zero).
template <typename T, int D, int TENSOR, bool STREAM>
__device__ __forceinline__ void stage_rows(T* to, int first_row, const T* base, int rows, int row_bytes, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)  // (the host pass does not know the resource's type)
  constexpr int LPR = RowLanes<T, D>::LPR, RPI = RowLanes<T, D>::RPI;
  const __amdgpu_buffer_rsrc_t from =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, rows <= 0 ? 0 : (rows - 1) * row_bytes + D * (int)sizeof(T), 0x00020000);
#pragma unroll
  for (int i = 0; i < 16 / RPI; ++i) {
    const int row = i * RPI + lane / LPR;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, SL_LDS(reinterpret_cast<char*>(to) + i * 1024), 16,
                                             row * row_bytes + piece_of<T, D, TENSOR>(first_row + row, lane) * 16, 0, 0, STREAM ? 2 : 0);
  }
#endif
}
// Pages of any size: `at` of lane l is the element offset of row l of the stage, < 0: zeros.
template <typename T, int D, int TENSOR, bool STREAM>
__device__ __forceinline__ void stage_rows_any(T* to, int first_row, const T* base, int64_t at, int lane) {
  constexpr int LPR = RowLanes<T, D>::LPR, RPI = RowLanes<T, D>::RPI;
#pragma unroll
  for (int i = 0; i < 16 / RPI; ++i) {
    const int row = first_row + i * RPI + lane / LPR;
    const int lo = __shfl((int)(uint32_t)at, row, 64), hi = __shfl((int)(at >> 32), row, 64);
    const char* const from =
        hi < 0 ? reinterpret_cast<const char*>(g_zeros) : reinterpret_cast<const char*>(base + (((int64_t)hi << 32) | (uint32_t)lo));
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + piece_of<T, D, TENSOR>(row, lane) * 16),
                                     SL_LDS(reinterpret_cast<char*>(to) + i * 1024), 16, 0, STREAM ? 2 : 0);
  }
}

// An LDS address that the compiler knows nothing of: where it sees that staged rows are read, it waits for every staging load
// in flight, the next step's among them.
template <typename T>
__device__ __forceinline__ uint32_t lds_address(const T* p, int offset) {
  uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) T*)p + offset;
  asm volatile("" : "+v"(at));
  return at;
}

// Two transposing reads: the lane's column of rows 0 .. 3 and 4 .. 7 behind p.
template <int D>
__device__ __forceinline__ bf16x8 transposed8(const bf16_t* __restrict__ p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* LdsPtr;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)p);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(p + 4 * D));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A wavefront's CB blocks of 32 columns; it takes 32 * KB tokens at a time.
// LIVE: which of the tokens have a page: a bit for each sixteen of them (uint32_t), or, where pages end anywhere, for each (uint64_t).
template <int D, int CB, int KB>
struct Softmax {
  static constexpr int DT = D / 32;
  f32x16 o[CB][DT], s[CB][KB];
  float m[CB], l[CB];

  __device__ __forceinline__ void clear_sums() {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      m[cb] = -INFINITY;
      l[cb] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[cb][dt][r] = 0.f;
    }
  }
  __device__ __forceinline__ void clear_scores() {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[cb][kb][r] = 0.f;
  }
  // token_of(r, half): token of accumulator r of a block of 32; lo, last (LDS): what each column attends
  template <typename LIVE, typename F>
  __device__ __forceinline__ void mask(int t0, LIVE live, const int* lo, const int* last, F&& token_of) {
    const int ln = lane_now(), hf = ln >> 5;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const int from = lo[32 * cb + (ln & 31)], width = last[32 * cb + (ln & 31)] - from;  // (nothing: INT_MAX, and below 0)
      const int at = t0 + token_of(0, hf) - from;
      const LIVE bits = sizeof(LIVE) == 8 ? live >> token_of(0, hf) : live;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int ahead = 32 * kb + token_of(r, 0) - token_of(0, 0), t = at + ahead;
          // (sixteen tokens at a time: token_of(r, 1) lies in the sixteen of token_of(r, 0))
          const bool there = bits >> (sizeof(LIVE) == 8 ? ahead : (32 * kb + token_of(r, 0)) / 16) & 1;
          s[cb][kb][r] = t >= 0 && t <= width && there ? s[cb][kb][r] : -INFINITY;
        }
    }
  }
  // Weights are taken against a bound, which moves, to the maximum + 8, only when a score passes it.
  __device__ __forceinline__ void move_bounds(float sc) {
    bool grow[CB], any = false;
    float top[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      top[cb] = s[cb][0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) top[cb] = max_of(top[cb], s[cb][kb][r]);
      top[cb] = across_halves_max(top[cb]) * sc;
      grow[cb] = !(top[cb] <= m[cb]);
      any = any || grow[cb];
    }
    if (__builtin_amdgcn_ballot_w64(any) == 0) return;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const float to = grow[cb] ? top[cb] + 8.f : m[cb];
      const float f = grow[cb] ? weight_of(m[cb], to) : 1.f;
      m[cb] = to;
      l[cb] *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[cb][dt][r] *= f;
    }
  }
  __device__ __forceinline__ float minus_bound(int cb) const { return m[cb] == -INFINITY ? 0.f : -m[cb]; }
};

template <typename T, int D, int CB, int KB>
struct Tile;

template <int D, int CB, int KB>
struct Tile<bf16_t, D, CB, KB> : Softmax<D, CB, KB> {
  typedef Softmax<D, CB, KB> Base;
  using Base::DT;
  using Base::l;
  using Base::o;
  using Base::s;
  static constexpr int KK = D / 16;
  bf16x8 q[CB][KK];
  int kbase, vbase;

  __device__ __forceinline__ void clear(int lane) {
    const int col = lane & 31, hf = lane >> 5;
    const int krow = (col & 0x13) | ((col & 4) << 1) | ((col & 8) >> 1);
    kbase = 2 * (krow * D + ((hf ^ k_swizzle<bf16_t, D>(krow)) << 3));
    const int vrow = (lane & 15) >> 2;
    vbase = 2 * ((8 * hf + vrow) * D + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_swizzle<bf16_t, D>(vrow)) << 3) + 4 * (lane & 1));
    Base::clear_sums();
  }
  __device__ __forceinline__ void load_q(int cb, const bf16_t* row, int lane) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[cb][kk] = *reinterpret_cast<const bf16x8*>(row + (lane >> 5) * 8 + kk * 16);
  }
  // 32 * KB tokens from t0 on, K rows at kt, V rows at vt (LDS)
  template <typename LIVE>
  __device__ __forceinline__ void attend(const bf16_t* kt, const bf16_t* vt, int t0, bool masked, LIVE live, float sc, const int* lo,
                                         const int* last) {
    Base::clear_scores();
    const uint32_t ka = lds_address(kt, kbase);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const bf16x8 a = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>((uintptr_t)((ka ^ (kk << 5)) + 64 * D * kb));
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) s[cb][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[cb][kk], s[cb][kb], 0, 0, 0);
      }
    // fragment reads run four products ahead (0x100 = LDS read, 0x008 = MFMA)
    __builtin_amdgcn_sched_group_barrier(0x100, 4 / CB, 0);
#pragma unroll
    for (int i = 0; i < KK * KB - 4 / CB; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, CB, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    __builtin_amdgcn_s_setprio(3);  // (few of the vector instructions fit beside another wavefront's products)
    if (masked) Base::mask(t0, live, lo, last, [](int r, int hf) { return 8 * hf + 16 * (r >> 3) + (r & 7); });
    Base::move_bounds(sc);
    bf16x8 p[CB][2 * KB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const float minus = Base::minus_bound(cb);
#pragma unroll
      for (int ks = 0; ks < 2 * KB; ++ks) {
        f32x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = fast_exp2(fmaf(s[cb][ks >> 1][8 * (ks & 1) + e], sc, minus));
        // the unrounded weights' sum: lse is exact to fp32
        l[cb] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        // Rounded to bf16 for the product with V: an error of up to 2^-8 of each weight, as large as rounding the result makes.
        p[cb][ks] = __builtin_convertvector(w, bf16x8);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    const uint32_t va = lds_address(vt, vbase);
#pragma unroll
    for (int ks = 0; ks < 2 * KB; ++ks)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint32_t at = (va ^ (dt << 6)) + 32 * ks * D;
        const bf16x8 a = transposed8<D>((const bf16_t*)(const __attribute__((address_space(3))) bf16_t*)(uintptr_t)at);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p[cb][ks], o[cb][dt], 0, 0, 0);
      }
    __builtin_amdgcn_sched_group_barrier(0x100, 8 / CB, 1);
#pragma unroll
    for (int i = 0; i < 2 * KB * DT - 4 / CB; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, CB, 1);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4, 1);
  }
};

// fp32: a lane reads 16 bytes of a K row, elements 8 c + 4 (l / 32) + 0 .. 3, which feed four products of two elements each.
template <int D>
struct Tile<float, D, 1, 1> : Softmax<D, 1, 1> {
  typedef Softmax<D, 1, 1> Base;
  using Base::DT;
  using Base::l;
  using Base::o;
  using Base::s;
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  f32x4 q[D / 8];
  int kbase, vbase;

  __device__ __forceinline__ void clear(int lane) {
    const int row = lane & 31, hf = lane >> 5;
    kbase = row * D * 4 + ((hf ^ k_swizzle<float, D>(row)) << 4);
    vbase = 4 * hf * D * 4 + row * 4;
    Base::clear_sums();
  }
  __device__ __forceinline__ void load_q(int, const float* row, int lane) {
#pragma unroll
    for (int c = 0; c < D / 8; ++c) q[c] = *reinterpret_cast<const f32x4*>(row + 8 * c + (lane >> 5) * 4);
  }
  template <typename LIVE>
  __device__ __forceinline__ void attend(const float* kt, const float* vt, int t0, bool masked, LIVE live, float sc, const int* lo,
                                         const int* last) {
    Base::clear_scores();
    const uint32_t ka = lds_address(kt, kbase);
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
      const f32x4 a = *reinterpret_cast<const __attribute__((address_space(3))) f32x4*>((uintptr_t)(ka ^ (c << 5)));
#pragma unroll
      for (int e = 0; e < 4; ++e) s[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], q[c][e], s[0][0], 0, 0, 0);
    }
    if (masked) Base::mask(t0, live, lo, last, [](int r, int hf) { return 8 * (r >> 2) + 4 * hf + (r & 3); });
    Base::move_bounds(sc);
    const float minus = Base::minus_bound(0);
    f32x16 w;
#pragma unroll
    for (int r = 0; r < 16; ++r) w[r] = fast_exp2(fmaf(s[0][0][r], sc, minus));
#pragma unroll
    for (int r = 0; r < 16; r += 4) l[0] += (w[r] + w[r + 1]) + (w[r + 2] + w[r + 3]);
    const uint32_t va = lds_address(vt, vbase);
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const float a = *reinterpret_cast<const __attribute__((address_space(3))) float*>(
            (uintptr_t)(va + (8 * (r >> 2) + (r & 3)) * D * 4 + dt * 128));
        o[0][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w[r], o[0][dt], 0, 0, 0);
      }
  }
};

// The columns of a tile: rows and heads of one kv head's group, rows first.  Entry e's tiles start at floor(cu[e] * G / cols) + e, which
// leaves room for ceil(new rows * G / cols) of them, since ceil(y - x) <= floor(y) - floor(x) + 1.
struct ColumnRun {
  Entry at;
  int u0, n;  // columns u0 .. u0 + n - 1 of the entry: row r0 + u / G, head u % G of the group
};
// (G: columns of a row)
__device__ __forceinline__ ColumnRun columns_of(const PagedArgs& x, int tile, int cols, int G) {
  auto first = [&](int r0, int e) { return (int)((int64_t)max(r0, 0) * G / cols) + e; };
  ColumnRun r;
  r.at = find_entry(x, [&](int r0, int e) { return first(r0, e) <= tile; });
  const int64_t u0 = (int64_t)(tile - first(r.at.r0, r.at.e)) * cols;
  const int64_t n = (int64_t)(min(r.at.r1, x.b.rows) - r.at.r0) * G - u0;
  r.u0 = (int)u0;
  r.n = u0 < 0 || n <= 0 ? 0 : (int)min(n, (int64_t)cols);
  return r;
}

// Waits for the wavefront's loads, staging ones too, and LDS operations.
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// NW wavefronts of 32 * CB columns, two stages of STEP tokens.  Measured (bf16, D = 128): four prompts of 2500 to 6000 tokens, 32:8 heads,
// 770 us = 1.05 PFLOP/s, where a large library product reaches 1.2; 2000 rows behind 64K tokens, 32:4 heads, eight spans of 512, 215 us =
// 0.66 PFLOP/s (tiles of 8 steps, whose beginnings and ends are a quarter of them); one token behind a million 49 us = 5.2 TB/s, 24 caches
// of up to 120000 tokens 93 us = 5.6 TB/s, where a pure read reaches 6.4.
//   4 wavefronts: the matrix cores are what bounds these
//   1 wavefront: few columns, so that memory does; four workgroups (D = 128) of a compute unit have 16 KB each on the way
//                (three and four stages leave room for fewer: 24 caches of up to 120000 tokens 119 -> 122, 153 us)
// Workgroups of the window come first, then, of the spans' pieces,
//   4 wavefronts: the buckets' tiles
//   1 wavefront: one for every (row, head, slot).  Other heads and rows of its 32 columns may list the same span: the first one
//                that does takes it for all, so that a span is read once for the group.
//   ANY: pages of a size that is no multiple of 16: every row has a page of its own, at twice the instructions for its address
//   PAST: records go past the caches
template <typename T, int D, int NW, int CB, int STEP, bool ANY, bool PAST>
__global__ __launch_bounds__(64 * NW, NW == 1 || sizeof(T) == 4 ? 1 : 2) void tile_kernel(const PagedArgs x, const TilePlan plan) {
  constexpr int COLS = NW * 32 * CB;
  extern __shared__ __align__(1024) char s_dynamic[];  // (static, the compiler would wait for staging loads at every read)
  T(*const s_kv)[2][STEP * D] = reinterpret_cast<T(*)[2][STEP * D]>(s_dynamic);
  __shared__ int s_rh[COLS], s_lo[COLS], s_last[COLS];
  const int lane = threadIdx.x & 63, wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = workgroup();
  if (unit >= plan.units) return;  // (grid_of rounds up)
  const bool window = unit < plan.window_units;
  int seq, head, part;         // sequence, kv head, piece
  int begin, end;              // tokens [begin, end) of the tile
  int any_lo, any_last;        // ... that any of the wavefront's columns attends
  int all_lo, all_last;        // ... that all of them attend
  // The pages of the first rows are asked for as soon as a tile knows its sequence and tokens.
  // !ANY: lane g has the page of the g-th sixteen tokens from `batch` on; the next 64 pages are looked up while those are in use.
  // ANY: lane l has the page of row l of the next stage.
  int page = -1;
  auto look_up = [&](int t0) {
    const int ln = lane_now(), t = t0 + (ANY ? ln % STEP : ln * 16);
    return t < end ? x.c.tables[(int64_t)seq * x.c.max_pages + (uint32_t)t / x.c.by_ps] : -1;
  };
  auto ask_pages = [&] {
    seq = __builtin_amdgcn_readfirstlane(seq);
    begin = __builtin_amdgcn_readfirstlane(begin);
    end = __builtin_amdgcn_readfirstlane(end);
    if (begin < end) page = look_up(begin / 16 * 16);
  };
  // columns
  if (window) {
    // (tile, piece) of the kv heads in turn; the last tiles first, whose ranges are the longest
    head = (int)(unit % x.c.Hkv);
    const int at = (int)(unit / x.c.Hkv);
    if (at >= plan.tiles * x.p.window) return;
    const int tile = plan.tiles - 1 - at / x.p.window, piece = at % x.p.window;
    part = x.a.topk * x.p.routed + piece;
    const ColumnRun run = columns_of(x, tile, COLS, x.a.G);
    if (run.n <= 0) return;
    const int r0 = run.at.r0, u0 = run.u0, len = run.at.len, pos0 = len - (run.at.r1 - r0);
    seq = run.at.s;
    const int first = max(pos0 + u0 / x.a.G, 0);  // position of the tile's first row that has a token
    const int most = min(len, x.b.L) - 1;         // of the last row that has one
    const int64_t origin = (int64_t)(first / x.a.S) * x.a.S / 16 * 16 + (int64_t)piece * x.p.window_tokens;
    const int from = (int)min(origin, (int64_t)INT_MAX), upto = (int)min(origin + x.p.window_tokens - 1, (int64_t)INT_MAX);
    auto lo_of = [&](int pos) { return max(pos / x.a.S * x.a.S, from); };
    auto last_of = [&](int pos) { return min(pos, upto); };
    // Later rows begin and end no earlier.
    const int last = min(pos0 + (u0 + run.n - 1) / x.a.G, most);
    begin = lo_of(first);
    end = first > last ? begin : last_of(last) + 1;
    ask_pages();
    for (int c = threadIdx.x; c < COLS; c += 64 * NW) {
      const int u = u0 + c, row = r0 + u / x.a.G, pos = pos0 + u / x.a.G;
      int rh = -1, clo = INT_MAX, clast = -1;
      if (c < run.n) {
        rh = (head * x.a.G + u % x.a.G) * x.b.rows + row;
        if (pos >= 0 && pos <= most && lo_of(pos) <= last_of(pos)) {
          clo = lo_of(pos);
          clast = last_of(pos);
        }
      }
      s_rh[c] = rh;
      s_lo[c] = clo;
      s_last[c] = clast;
    }
    const int c0 = wave * 32 * CB, c1 = min(c0 + 32 * CB, run.n) - 1;
    const int p0 = pos0 + (u0 + c0) / x.a.G, p1 = pos0 + (u0 + c1) / x.a.G, q0 = max(p0, 0), q1 = min(p1, most);
    const bool some = c0 <= c1 && q0 <= q1;
    any_lo = some ? lo_of(q0) : INT_MAX;
    any_last = some ? last_of(q1) : -1;
    all_lo = p0 < 0 || p1 > most ? INT_MAX : lo_of(q1);  // (a row without a token attends nothing)
    all_last = last_of(q0);
  } else if (NW > 1) {
    // eight tiles, one for each XCD, and their pieces in turn
    const int64_t u = unit - plan.window_units, group8 = u / (8 * x.p.routed);
    const int in_group = (int)(u - group8 * 8 * x.p.routed);
    part = in_group >> 3;
    const int4 rec = plan.records[group8 * 8 + (in_group & 7)];
    const int count = rec.w, j = rec.x;
    if (count == 0) return;
    head = rec.y % x.c.Hkv;
    seq = x.b.seqs[rec.y / x.c.Hkv];
    begin = j * x.a.S + part * x.p.routed_tokens;
    end = min(begin + x.p.routed_tokens, (j + 1) * x.a.S);
    ask_pages();
    for (int c = threadIdx.x; c < COLS; c += 64 * NW) {
      const int item = c < count ? plan.items[(int64_t)rec.z * COLS + c] : -1;  // (row and head) * 32 + slot
      // (where cu_rows decreases, some that are counted have no row: their items hold anything)
      s_rh[c] = item >= 0 && item >> 5 < x.a.Hq * x.b.rows && (item & 31) < x.a.topk ? item : -1;
      s_lo[c] = c < count ? begin : INT_MAX;
      s_last[c] = c < count ? end - 1 : -1;
    }
    const bool some = wave * 32 * CB < count;
    all_lo = begin;
    all_last = end - 1;
    any_lo = some ? all_lo : INT_MAX;
    any_last = some ? all_last : -1;
  } else {
    const int64_t u = unit - plan.window_units;
    part = (int)(u % x.p.routed);
    const int64_t item = u / x.p.routed;
    const int slot = (int)(item % x.a.topk), rh = (int)(item / x.a.topk);
    const int h = rh / x.b.rows, row = rh - h * x.b.rows;
    const int j = x.idx[h * x.a.ish + row * x.a.ist + slot];
    const Entry at = entry_with_row(x, row);
    if (row < at.r0 || row >= at.r1) return;
    head = h / x.a.G;
    seq = at.s;
    const int own = (row - at.r0) * x.a.G + h - head * x.a.G, u0 = own & ~31;  // columns u0 .. u0 + 31 of the entry
    const int pos = position_of(x, at, row);
    if (pos < 0 || j < 0 || j >= pos / x.a.S) {
      if (lane == 0) x.part_lse[(int64_t)rh * x.p.count + slot * x.p.routed + part] = -INFINITY;
      return;
    }
    const int cols = min((min(at.r1, x.b.rows) - at.r0) * x.a.G - u0, 32);
    begin = any_lo = all_lo = j * x.a.S + part * x.p.routed_tokens;
    end = min(begin + x.p.routed_tokens, (j + 1) * x.a.S);
    any_last = all_last = end - 1;
    ask_pages();  // (before the other columns' lists: a unit is short, and a chain of loads)
    if (lane < 32) {
      s_rh[lane] = -1;
      s_lo[lane] = INT_MAX;
      s_last[lane] = -1;
    }
    bool earlier = false;
    for (int i = lane; i < cols * x.a.topk; i += 64) {
      const int c = i / x.a.topk, k = i - c * x.a.topk;
      const int row2 = at.r0 + (u0 + c) / x.a.G, h2 = head * x.a.G + (u0 + c) % x.a.G;
      const int pos2 = position_of(x, at, row2);
      if (pos2 >= 0 && j < pos2 / x.a.S && x.idx[h2 * x.a.ish + row2 * x.a.ist + k] == j) {
        earlier = earlier || u0 + c < own || (u0 + c == own && k < slot);
        s_rh[c] = (h2 * x.b.rows + row2) * 32 + k;
        s_lo[c] = begin;
        s_last[c] = end - 1;
      }
    }
    if (__builtin_amdgcn_ballot_w64(earlier) != 0) return;
  }
  __syncthreads();
  constexpr int KB = CB == 2 || STEP == 32 || sizeof(T) == 4 ? 1 : 2;
  Tile<T, D, CB, KB> tile;
  tile.clear(lane);
  any_lo = __builtin_amdgcn_readfirstlane(any_lo);
  any_last = __builtin_amdgcn_readfirstlane(any_last);
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_last = __builtin_amdgcn_readfirstlane(all_last);
  begin = begin / 16 * 16;
  head = __builtin_amdgcn_readfirstlane(head);
  const int64_t base = x.b.layer * x.c.layer + head * x.c.head;
  const T *const K = static_cast<const T*>(x.c.K), *const V = static_cast<const T*>(x.c.V);
  constexpr int GROUPS = STEP / 16;
  auto there = [&](int page) { return (uint64_t)__builtin_amdgcn_ballot_w64((uint32_t)page < (uint32_t)x.c.n_pages); };
  int batch = begin, next_page = -1;
  uint64_t alive = 0;       // which of the looked up pages there are
  uint64_t live[2] = {};    // of the stages: a bit for each sixteen rows (ANY: for each)
  auto stage = [&](int t0, int b) {
    const int ln = lane_now();
    if constexpr (ANY) {
      const int t = t0 + ln % STEP;
      live[b] = there(page);
      const int64_t at = (uint32_t)page < (uint32_t)x.c.n_pages
                             ? base + page * x.c.page + (int64_t)((uint32_t)t - (uint32_t)t / x.c.by_ps * x.c.ps) * x.c.tok
                             : -1;
#pragma unroll
      for (int i = 0; i < GROUPS / NW; ++i) {
        const int r0 = (NW == 1 ? i : wave) * 16;
        stage_rows_any<T, D, 0, NW == 1>(&s_kv[b][0][r0 * D], r0, K, at, ln);
        stage_rows_any<T, D, 1, NW == 1>(&s_kv[b][1][r0 * D], r0, V, at, ln);
      }
      page = look_up(t0 + STEP);
    } else {
      if (t0 - batch >= 1024) {
        batch += 1024;
        page = next_page;
        alive = there(page);
        next_page = look_up(batch + 1024);
      }
      const int first = (t0 - batch) / 16, row_bytes = (int)x.c.tok * (int)sizeof(T);
      live[b] = alive >> first;
#pragma unroll
      for (int i = 0; i < GROUPS / NW; ++i) {
        const int g = NW == 1 ? i : wave, r0 = g * 16, t = __builtin_amdgcn_readfirstlane(t0 + r0);
        const bool on = live[b] >> g & 1;
        const int rows = on ? min(end - t, 16) : 0;
        const int in_page = __builtin_amdgcn_readfirstlane((uint32_t)t - (uint32_t)t / x.c.by_ps * x.c.ps);
        const int64_t from = on ? uniform64(base + __builtin_amdgcn_readlane(page, first + g) * x.c.page + in_page * x.c.tok) : 0;
        stage_rows<T, D, 0, NW == 1>(&s_kv[b][0][r0 * D], r0, K + from, rows, row_bytes, ln);
        stage_rows<T, D, 1, NW == 1>(&s_kv[b][1][r0 * D], r0, V + from, rows, row_bytes, ln);
      }
    }
  };
  if (begin < end) {
    alive = there(page);
    if (!ANY && end - batch > 1024) next_page = look_up(batch + 1024);
    stage(begin, 0);
  }
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const int item = s_rh[wave * 32 * CB + cb * 32 + (lane & 31)];
    const int rh = max(window ? item : item >> 5, 0);  // (a column of nobody reads some row: nothing is made of it)
    const int h = rh / x.b.rows, row = rh - h * x.b.rows;
    tile.load_q(cb, static_cast<const T*>(x.Q) + h * x.a.qsh + row * x.a.qst, lane);
  }
  int b = 0;
  for (int t0 = begin; t0 < end; t0 += STEP, b ^= 1) {
    wait_loads();
    if (NW > 1) {
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
    if (t0 + STEP < end) stage(t0 + STEP, b ^ 1);
#pragma unroll 1
    for (int at = 0; at < STEP; at += 32 * KB) {
      const int t = t0 + at, upto = t + 32 * KB - 1;
      if (upto < any_lo || t > any_last) continue;
      typedef std::conditional_t<ANY, uint64_t, uint32_t> Live;
      constexpr Live kAll = ANY ? (KB == 2 ? ~(Live)0 : (Live)0xffffffffu) : (Live)((1 << 2 * KB) - 1);
      const Live now = (Live)(live[b] >> (ANY ? at : at / 16)) & kAll;
      tile.attend(&s_kv[b][0][at * D], &s_kv[b][1][at * D], t, t < all_lo || upto > all_last || now != kAll, now, x.scale_log2e,
                  s_lo + wave * 32 * CB, s_last + wave * 32 * CB);
    }
  }
  // Results.  A column with a value that is not finite is marked by an lse that is not a number: it may have come from a
  // token that the column does not attend, and the merge takes such a piece again, row by row.
  // Values go out by way of the stages, whose rows are free by now: a lane has four of them of one column, 8 or 16 bytes of a row's 256.
  if (NW > 1) __syncthreads();
  const bool direct = x.p.count == 1;
  typedef typename Record<T>::Value Value;
  typedef std::conditional_t<sizeof(T) == 2, __bf16, float> Out;
  constexpr int LPR = D * (int)sizeof(Value) / 16, RPI = 64 / LPR;  // lanes of a row, rows of an instruction
  char* const s_out = s_dynamic + wave * (32 * D * (int)sizeof(Value));
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const int ln = lane_now(), own = wave * 32 * CB + cb * 32 + (ln & 31), item = s_rh[own];
    const float sum = across_halves_sum(tile.l[cb]);
    const float inv = 1.f / sum;
    float check = 0.f, top = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        check = fmaf(tile.o[cb][dt][r], 0.f, check);
        top = max_of(top, fabsf(tile.o[cb][dt][r]));
      }
    check = across_halves_sum(check);
    top = across_halves_max(top);
    const bool none = tile.m[cb] == -INFINITY;
    const float lse = none ? -INFINITY : check == 0.f ? tile.m[cb] + __log2f(sum) : NAN;
    auto record = [&](int item) {
      return (int64_t)(window ? item : item >> 5) * x.p.count + (window ? part : (item & 31) * x.p.routed + part);
    };
    const float scale = direct || sizeof(T) == 4 ? 1.f : scale_above(top * inv);
    if (item >= 0 && ln < 32) {
      const int64_t rec = record(item);
      x.part_lse[rec] = lse;
      if (direct && x.LSE) x.LSE[rec] = lse * kLn2;
      if (!direct && sizeof(T) == 2) x.part_scale[rec] = scale;
    }
    // d = 32 dt + 8 g + 4 (ln / 32) on: a 16-byte unit, or half of one, swizzled by the row
    auto put = [&](auto zero, float by) {
      typedef decltype(zero) V;
      typedef V Four __attribute__((ext_vector_type(4)));
      const int row = ln & 31, hf = ln >> 5;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          Four v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (V)(none ? 0.f : tile.o[cb][dt][4 * g + e] * by);
          const int unit = sizeof(V) == 2 ? 4 * dt + g : 8 * dt + 2 * g + hf;
          *reinterpret_cast<Four*>(s_out + (row * LPR + (unit ^ row % LPR)) * 16 + (sizeof(V) == 2 ? 8 * hf : 0)) = v;
        }
    };
    if (direct) put(Out(), inv);
    else put(Value(), inv / scale);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    char* const to = static_cast<char*>(direct ? x.O : x.part_o);
    const uint64_t write = __builtin_amdgcn_ballot_w64(item >= 0 && (direct || !none));
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) {
      const int row = i * RPI + ln / LPR, piece = ln % LPR;
      if (!(write >> row & 1)) continue;
      const uint4 v = *reinterpret_cast<const uint4*>(s_out + (row * LPR + (piece ^ row % LPR)) * 16);
      char* const at = to + record(s_rh[wave * 32 * CB + cb * 32 + row]) * (D * (int)sizeof(Value)) + piece * 16;
      if (PAST) store16_stream(at, v);
      else *reinterpret_cast<uint4*>(at) = v;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- the rows that list a span: buckets (entry, kv head, span), each cut into tiles of `cols` items
__global__ __launch_bounds__(256) void zero_kernel(int32_t* __restrict__ to, int n) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) to[i] = 0;
}

// An item's place in its bucket.  A workgroup takes kCountRows rows of an entry with the heads of a kv head's group: it counts their items
// in LDS, adds its counts to the buckets', and hands out the places that it got; their order among workgroups may differ from run to run,
// which no result depends on.  Atomics on the buckets alone took 188 us for 512000 items of 512 buckets.
// Pieces of empty slots are marked here: no tile writes them.
constexpr int kCountRows = 64, kCountSpans = 12288;
__global__ __launch_bounds__(1024) void count_kernel(const PagedArgs x, const TilePlan plan) {
  extern __shared__ int32_t s_count[];  // [spans], if they fit
  const int head = blockIdx.y;
  const ColumnRun run = columns_of(x, blockIdx.x, kCountRows, 1);
  if (run.n <= 0) return;
  const bool local = plan.spans <= kCountSpans;
  if (local)
    for (int j = threadIdx.x; j < plan.spans; j += 1024) s_count[j] = 0;
  __syncthreads();
  int32_t* const counts = plan.counts + ((int64_t)run.at.e * x.c.Hkv + head) * plan.spans;
  const int of_head = run.n * x.a.topk, items = of_head * x.a.G;
  for (int pass = local ? 0 : 1; pass < 2; ++pass) {
#pragma unroll 4
    for (int i = threadIdx.x; i < items; i += 1024) {
      const int g = i / of_head, at = i - g * of_head, r = at / x.a.topk, k = at - r * x.a.topk;
      const int h = head * x.a.G + g, row = run.at.r0 + run.u0 + r;
      const int pos = position_of(x, run.at, row), c = pos < 0 ? 0 : pos / x.a.S;
      const int64_t rh = (int64_t)h * x.b.rows + row;
      const int j = x.idx[h * x.a.ish + row * x.a.ist + k];
      if (j >= 0 && j < c) {
        if (pass == 0) atomicAdd(&s_count[j], 1);
        else plan.ranks[rh * x.a.topk + k] = local ? atomicAdd(&s_count[j], 1) : atomicAdd(&counts[j], 1);
      } else if (pass == 1) {
        plan.ranks[rh * x.a.topk + k] = -1;
        for (int q = 0; q < x.p.routed; ++q) x.part_lse[rh * x.p.count + k * x.p.routed + q] = -INFINITY;
      }
    }
    if (pass == 0) {
      __syncthreads();
      for (int j = threadIdx.x; j < plan.spans; j += 1024)
        if (s_count[j]) s_count[j] = atomicAdd(&counts[j], s_count[j]);
      __syncthreads();
    }
  }
}

// Tiles of each bucket in the buckets' order; one workgroup.  Tiles of one bucket read the same rows: workgroups u = x (mod 8) run on
// XCD x, which has an L2 of its own, and are given the x-th eighth of the list, in its order.
// (Where cu_rows decreases, rows may be counted once for each of 65535 entries: sums stop at most_tiles, which is below 2^30, and what the
// list has no room for is left out.)
__global__ __launch_bounds__(1024) void tiles_kernel(const TilePlan plan, int cols_log2) {
  __shared__ int s_wave[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto tiles_of = [&](int i) {
    const int n = i < plan.buckets ? (plan.counts[i] + (1 << cols_log2) - 1) >> cols_log2 : 0;
    return min(max(n, 0), plan.most_tiles);
  };
  auto sum = [&](int a, int b) { return min(a + b, plan.most_tiles); };
  int total = 0;
#pragma unroll 1
  for (int base = 0; base < plan.buckets; base += 1024) {
    const int i = base + threadIdx.x;
    int v = tiles_of(i);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(v, off, 64);
      if (lane >= off) v = sum(v, y);
    }
    const int before = __shfl_up(v, 1, 64);
    __syncthreads();
    if (lane == 63) s_wave[wave] = v;
    __syncthreads();
    int at = total;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (k < wave) at = sum(at, s_wave[k]);
      total = sum(total, s_wave[k]);
    }
    if (lane > 0) at = sum(at, before);
    if (i < plan.buckets) plan.first_tile[i] = at;
  }
  const int share = (total + 7) / 8;
#pragma unroll 1
  for (int base = 0; base < plan.buckets; base += 1024) {
    const int i = base + threadIdx.x, n = tiles_of(i);
    if (n == 0) continue;
    const int first = plan.first_tile[i], count = plan.counts[i];
    for (int k = 0; k < n && first + k < total; ++k) {
      const int tile = first + k, x = tile / share;
      plan.records[(tile - x * share) * 8 + x] = make_int4(i % plan.spans, i / plan.spans, tile, min(count - (k << cols_log2), 1 << cols_log2));
    }
  }
  for (int k = threadIdx.x; k < plan.most_tiles; k += 1024)
    if ((k & 7) * share + (k >> 3) >= total || (k >> 3) >= share) plan.records[k].w = 0;
}

__global__ __launch_bounds__(256) void items_kernel(const PagedArgs x, const TilePlan plan, int cols_log2) {
  const int64_t i = workgroup() * 256 + threadIdx.x;
  const int rh = (int)(i / x.a.topk), k = (int)(i - (int64_t)rh * x.a.topk);
  if (rh >= x.a.Hq * x.b.rows) return;
  const int h = rh / x.b.rows, row = rh - h * x.b.rows;
  if (row < x.b.cu[0] || row >= x.b.cu[x.b.B]) return;
  const int rank = plan.ranks[i];
  if (rank < 0) return;
  const int e = entry_of_row(x.b.cu, x.b.B, row), j = x.idx[h * x.a.ish + row * x.a.ist + k];
  // (Where cu_rows decreases, count_kernel may have passed this row over, or given it to another entry: its rank is then anything, and so is j.)
  if ((uint32_t)j >= (uint32_t)plan.spans) return;
  const int64_t at = ((int64_t)plan.first_tile[(e * x.c.Hkv + h / x.a.G) * plan.spans + j] << cols_log2) + rank;
  if (at >= 0 && at < (int64_t)plan.most_tiles << cols_log2) plan.items[at] = rh * 32 + k;
}

// ------------------------------------------------------------------ merge
// Pieces of a row and head that a tile marked, once more, row by row, by one wavefront: of the window, whose tiles cut it where they
// like, all into its first record.  DIRECT: one piece a row, whose result the tile has written.
template <typename T, int D, bool DIRECT>
__device__ __forceinline__ void mend_row(const PagedArgs& x, int rh) {
  const int h = rh / x.b.rows, row = rh - h * x.b.rows, P = x.p.count, routed = x.a.topk * x.p.routed;
  const Entry at = entry_with_row(x, row);
  const int pos = position_of(x, at, row);
  // (a row without a token is marked only where cu_rows decreases and no tile took it)
  const PieceRange window = pos < 0 ? PieceRange{0, 0} : PieceRange{pos / x.a.S * x.a.S, pos + 1};
  if (DIRECT) {
    take_piece<T, D, 1, true>(x, at.s, rh, window, 0, nullptr, nullptr);
    return;
  }
  const int64_t rec = (int64_t)rh * P;
  const int32_t* const slots = x.idx + h * x.a.ish + row * x.a.ist;
  bool near = false;
  for (int k = 0; k < P; ++k) {
    const float lse = x.part_lse[rec + k];
    if (lse == lse) continue;
    if (k < routed) take_piece<T, D, 1, false>(x, at.s, rh, range_of_piece(x, pos, k, slots), rec + k, nullptr, nullptr);
    else near = true;
  }
  if (near) {
    take_piece<T, D, 1, false>(x, at.s, rh, window, rec + routed, nullptr, nullptr);
    for (int k = routed + 1 + (threadIdx.x & 63); k < P; k += 64) x.part_lse[rec + k] = -INFINITY;
  }
}

// A wavefront looks at the records of 64 rows and heads.
template <typename T, int D, bool DIRECT>
__global__ __launch_bounds__(256) void mend_kernel(const PagedArgs x) {
  const int64_t n = (int64_t)x.a.Hq * x.b.rows;
  const int P = x.p.count;
  const int64_t first = (workgroup() * 4 + (threadIdx.x >> 6)) * 64, mine = first + (threadIdx.x & 63);
  const int row = (int)(mine % x.b.rows);
  bool bad = false;
  if (mine < n && row >= x.b.cu[0] && row < x.b.cu[x.b.B])
    for (int k = 0; k < P; ++k) {
      const float lse = x.part_lse[mine * P + k];
      bad = bad || lse != lse;
    }
  for (uint64_t marked = __builtin_amdgcn_ballot_w64(bad); marked; marked &= marked - 1)
    mend_row<T, D, DIRECT>(x, (int)first + __builtin_ctzll(marked));
}

// N lanes of a workgroup's 256 join the pieces of one row and head: weights to LDS, then D / 8 (fp32: D / 4) lanes a piece.  Nothing they
// ask for depends on what they have read: the first outputs are on their way before there are weights.  Bound by memory where rows fill
// the chip: 64000 rows and heads of 10 pieces of 256 bytes, 185 MB, in 42 us (4.4 TB/s; with a wavefront a row 47: its instructions).
// MEND: marked pieces are mended here.  (Where there are rows enough to fill the chip, that would cost half its occupancy.)
template <typename T, int D, int N, bool MEND>
__global__ __launch_bounds__(256) void merge_kernel(const PagedArgs x) {
  typedef typename Record<T>::Value Value;
  constexpr int EPL = 16 / sizeof(Value), LANES = D / EPL, GROUPS = N / LANES, U = N == 32 ? 8 : 4, ROWS = 256 / N;
  static_assert(N == 32 || N == 64 || N == 256, "half a wavefront, one, or four");
  typedef Value Values __attribute__((ext_vector_type(EPL)));
  extern __shared__ float s_dyn[];  // [ROWS][count] weights
  __shared__ float s_red[4];
  __shared__ float s_gates[ROWS][SL_MAX_TOPK], s_lses[ROWS][SL_MAX_TOPK];
  __shared__ float s_out[N < 256 ? 1 : GROUPS * D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x % N, sub = threadIdx.x / N, P = x.p.count;
  const int64_t unit = workgroup() * ROWS + sub;
  if (unit >= (int64_t)x.a.Hq * x.b.rows) return;
  const int rh = (int)unit;
  const int h = rh / x.b.rows, row = rh - h * x.b.rows;
  const int g = tid / LANES, c = tid % LANES;
  const Values* const po = reinterpret_cast<const Values*>(static_cast<const Value*>(x.part_o) + (int64_t)rh * P * D) + c;
  const float* const lse = x.part_lse + (int64_t)rh * P;
  const float* const scales = x.part_scale + (int64_t)rh * P;
  Values v[U];
  float lse0, scale0 = 1.f;  // of piece tid; the others are read again where there are so many
  auto ask = [&] {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + u * GROUPS < P) v[u] = __builtin_nontemporal_load(po + (int64_t)(g + u * GROUPS) * LANES);
    lse0 = tid < P ? lse[tid] : -INFINITY;
    if (sizeof(Value) == 2 && tid < P) scale0 = scales[tid];
  };
  ask();
  if (row < x.b.cu[0] || row >= x.b.cu[x.b.B]) return;
  float* const s_w = s_dyn + sub * P;
  float *const s_gate = s_gates[sub], *const s_lse = s_lses[sub];
  auto barrier = [] {
    if (N == 256) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  auto all_max = [&](float v) {
#pragma unroll
    for (int off = N < 64 ? N / 2 : 32; off >= 1; off >>= 1) v = max_of(v, __shfl_xor(v, off, 64));
    if (N < 256) return v;
    __syncthreads();
    if (lane == 0) s_red[wave] = v;
    __syncthreads();
    return max_of(max_of(s_red[0], s_red[1]), max_of(s_red[2], s_red[3]));
  };
  auto all_sum = [&](float v) {
#pragma unroll
    for (int off = N < 64 ? N / 2 : 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    if (N < 256) return v;
    __syncthreads();
    if (lane == 0) s_red[wave] = v;
    __syncthreads();
    return (s_red[0] + s_red[1]) + (s_red[2] + s_red[3]);
  };
  // log2-sum-exp2 of the pieces from `from` on
  auto lse_of = [&](int from) {
    float v = tid >= from ? lse0 : -INFINITY;
    for (int k = tid + N; k < P; k += N)
      if (k >= from) v = max_of(v, lse[k]);
    const float m = all_max(v);
    if (m == -INFINITY) return m;
    float l = tid >= from ? weight_of(lse0, m) : 0.f;
    for (int k = tid + N; k < P; k += N)
      if (k >= from) l += weight_of(lse[k], m);
    return m + __log2f(all_sum(l));
  };
  const int routed = x.a.topk * x.p.routed;
  bool any = false;  // a slot holds a span
  float total = lse_of(0);
  if (MEND && total != total && x.marks) {
    if (N == 64 || wave == 0) mend_row<T, D, false>(x, rh);
    __threadfence_block();
    barrier();
    ask();
    total = lse_of(0);
  }
  if (x.a.combined) {
    int pos;
    if constexpr (N == 32) {  // (rows of a wavefront differ)
      const int e = entry_of_row(x.b.cu, x.b.B, row);
      pos = position_of(x, {e, 0, length_of(x.c, x.b.seqs[e]), 0, x.b.cu[e + 1]}, row);
    } else {
      pos = position_of(x, entry_with_row(x, row), row);
    }
    const float near = lse_of(routed);
    float score = -INFINITY;
    bool mine = false;
    if (tid < x.a.topk) {
      const int64_t i = h * x.a.ish + row * x.a.ist + tid;
      const int j = x.idx[i];
      mine = pos >= 0 && j >= 0 && j < pos / x.a.S;
      if (mine) score = x.scores[i];
      float m = near;
      for (int k = 0; k < x.p.routed; ++k) m = max_of(m, lse[tid * x.p.routed + k]);
      float l = weight_of(near, m);
      for (int k = 0; k < x.p.routed; ++k) l += weight_of(lse[tid * x.p.routed + k], m);
      s_lse[tid] = m == -INFINITY ? m : m + __log2f(l);
    }
    if (N == 256) any = __syncthreads_or(mine);
    else any = (N == 64 ? __builtin_amdgcn_ballot_w64(mine) : __builtin_amdgcn_ballot_w64(mine) >> (lane & 32) & 0xffffffffu) != 0;
    if (any) {
      const float top = all_max(score);
      const float e = mine ? fast_exp2((score - top) * kLog2e) : 0.f;
      const float sum = all_sum(e);
      if (tid < x.a.topk) s_gate[tid] = e / sum;
      barrier();
    } else {
      total = near;
    }
  } else if (tid == 0 && x.LSE) {
    x.LSE[rh] = total * kLn2;
  }
  for (int k = tid; k < P; k += N) {
    const float mine = k == tid ? lse0 : lse[k];
    float w = 0.f;
    if (!any) {
      if (!x.a.combined || k >= routed) w = weight_of(mine, total);
    } else if (k < routed) {
      const int t = k / x.p.routed;
      if (s_gate[t] != 0.f) w = s_gate[t] * weight_of(mine, s_lse[t]);
    } else {
      for (int t = 0; t < x.a.topk; ++t)
        if (s_gate[t] != 0.f) w += s_gate[t] * weight_of(mine, s_lse[t]);
    }
    // (a piece without tokens has written neither output nor scale)
    if (sizeof(Value) == 2 && w != 0.f) w *= k == tid ? scale0 : scales[k];
    s_w[k] = w;
  }
  barrier();
  float acc[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = 0.f;
  for (int k0 = g; k0 < P; k0 += U * GROUPS) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * GROUPS;
      const float w = k < P ? s_w[k] : 0.f;
      if (w != 0.f) {
        if (k0 != g) v[u] = __builtin_nontemporal_load(po + (int64_t)k * LANES);
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[e] = fmaf(w, (float)v[u][e], acc[e]);
      }
    }
  }
  if constexpr (N < 256) {
#pragma unroll
    for (int off = LANES; off < N; off <<= 1)
#pragma unroll
      for (int e = 0; e < EPL; ++e) acc[e] += __shfl_xor(acc[e], off, 64);
    if (g == 0) {
      T* const to = static_cast<T*>(x.O) + (int64_t)rh * D + c * EPL;
      if constexpr (sizeof(T) == 2) {
        typedef __bf16 Out __attribute__((ext_vector_type(EPL)));
        Out o;
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[e] = (__bf16)acc[e];
        *reinterpret_cast<Out*>(to) = o;
      } else {
        *reinterpret_cast<float4*>(to) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < EPL; ++e) s_out[g * D + c * EPL + e] = acc[e];
    __syncthreads();
    if (tid < D) {
      float o = 0.f;
#pragma unroll
      for (int k = 0; k < GROUPS; ++k) o += s_out[k * D + tid];
      Elem<T>::store1(static_cast<T*>(x.O) + (int64_t)rh * D + tid, o);
    }
  }
}

// ------------------------------------------------------------------ host
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
dim3 grid_of(int64_t workgroups) {
  constexpr int64_t kMost = 1 << 20;
  return workgroups <= kMost ? dim3((unsigned)workgroups) : dim3((unsigned)kMost, (unsigned)div_up(workgroups, kMost));
}

// Records that the Infinity Cache (256 MB) would not keep until they are merged are written past the caches.  By the MiB reserved for them
// (32:4 heads, eight spans; us of the call, and past the caches): 193 (1900 rows, spans of 512) 248 and 252, 203 262 and 265, 232 (2700 rows, spans of
// 128) 239.9 and 238.7, 258 254.5 and 253.4, 344 335.5 and 332.7, 740 833 and 775, 4800 (64K rows, spans of 256) 5570 and 5260.
constexpr size_t kStreamedRecords = (size_t)230 << 20;

// How a call is taken.
struct Form {
  Pieces p;
  bool tiles;      // the matrix-core form
  bool buckets;    // ... with the spans' rows in buckets
  bool whole;      // row by row, a row a workgroup
  int cols_log2;   // columns of a tile
  TilePlan plan;   // (pointers unset)
  int64_t most_tiles;  // of the buckets
  size_t o_bytes, lse_bytes, plan_bytes;
};

Form form_of(const PageCache& c, const PagedBatch& b, const PagedAttention& a) {
  const int64_t rh = (int64_t)a.Hq * b.rows, window = a.S < b.L ? a.S : b.L;
  Form f = {};
  const int64_t spans = div_up(b.L, a.S), buckets = (int64_t)b.B * c.Hkv * spans, items = rh * a.topk;
  const int64_t columns = (int64_t)b.rows * a.G;  // of a kv head
  // Buckets read a span once for its rows, behind four launches that sort them.  us, 32:4 heads, top-8 of spans of 128, buckets and
  // without: bf16, 2.2 items a bucket 56 and 51, 4.4 65 and 91, 17 77 and 321; fp32, where a tile costs as much as 128 items however
  // few it has, 4.4 222 and 159, 8.7 228 and 312, 17 234 and 633.
  // (fp32 calls below 2^19 keys: 250 rows of 4 heads, top-4 of spans of 64, 33 and 25)
  f.buckets = a.topk > 0 && (c.dtype == SL_BF16 ? items >= 3 * buckets : items >= 6 * buckets && items * a.S >= 1 << 19);
  // fp32: row by row where tiles of 128 columns would be all but empty.
  f.tiles = c.dtype == SL_BF16 || f.buckets || (a.topk == 0 && columns > 32 * (int64_t)b.B);
  f.cols_log2 = (columns <= 32 * (int64_t)b.B || a.topk > 0) && !f.buckets          ? 5
                : c.dtype == SL_BF16 && columns * c.Hkv + items >= 256 * 1024 ? 8
                                                                             : 7;
  const int cols = 1 << f.cols_log2;
  f.whole = !f.tiles && rh >= 1024;
  if (f.whole) {
    f.p.count = 1;
    return f;
  }
  auto cut = [](int64_t tokens, int64_t units, int64_t wanted, int64_t most) {
    int64_t n = div_up(wanted, units);
    if (n > most) n = most;
    if (n > div_up(tokens, 64)) n = div_up(tokens, 64);
    return n < 1 ? 1 : n;
  };
  Pieces& p = f.p;
  p = {1, a.S, 1, (int)window, 0};
  if (a.topk > 0 && a.S <= b.L) {  // (no row has a longer span among its candidates)
    const int64_t units = f.buckets ? items / cols + 1 : items;
    p.routed_tokens = (int)div_up(div_up(a.S, cut(a.S, units, 1024, 64)), 16) * 16;
    p.routed = (int)div_up(a.S, p.routed_tokens);
  }
  if (f.tiles) {
    f.plan.tiles = (int)(columns / cols) + b.B;
    const int64_t longest = window + cols / a.G + 17;  // a tile's rows may lie in two windows; it begins at a multiple of 16
    // Enough workgroups of the narrow form for what fits the chip at once, four or (D = 64) nine to a compute unit: 32 caches of 1000
    // tokens, 32:8 heads, 39 us with four times as many, 33 so; of the wide one, twice.
    const int64_t n = cut(longest, (int64_t)f.plan.tiles * c.Hkv, cols == 32 && c.D == 64 ? 2048 : 1024, 256);
    p.window_tokens = (int)div_up(div_up(longest, n), 64) * 64;
    p.window = (int)div_up(longest, p.window_tokens);
    f.plan.window_units = div_up((int64_t)f.plan.tiles * p.window * c.Hkv, 8) * 8;
  } else {
    p.window_tokens = (int)div_up(window, cut(window, rh, 4096, 256));
    p.window = (int)div_up(window, p.window_tokens);
  }
  p.count = a.topk * p.routed + p.window;
  // (one piece a row: the tiles write results, and what the merge would ask for is not there)
  const bool direct = f.tiles && p.count == 1;
  f.o_bytes = direct ? 0 : align_up((size_t)rh * p.count * c.D * (c.dtype == SL_BF16 ? sizeof(_Float16) : sizeof(float)), 256);
  f.lse_bytes = align_up((size_t)rh * p.count * sizeof(float), 256);
  f.plan.units = f.plan.window_units;
  if (f.buckets) {
    f.plan.spans = (int)spans;
    f.plan.buckets = (int)buckets;
    // (a share of eight may be a tile short of its length)
    f.most_tiles = div_up(items / cols + (buckets < items ? buckets : items), 8) * 8;
    f.plan.units += f.most_tiles * p.routed;
    f.plan_bytes = align_up(sizeof(int32_t) * (align_up(2 * (size_t)buckets, 64) + 4 * (size_t)f.most_tiles + (size_t)items + (size_t)f.most_tiles * cols), 256);
  } else {
    f.plan.units += items * p.routed;
  }
  return f;
}

// The stages fill up to 128 KB of dynamic LDS beside the static arrays: more than a kernel has without asking.
template <typename T, int D, int NW, int CB, int STEP, bool ANY, bool PAST>
bool launch_tiles_as(const PagedArgs& x, const TilePlan& plan, hipStream_t st) {
  constexpr int kBytes = 2 * 2 * STEP * D * (int)sizeof(T);
  static std::mutex mu;
  static bool asked[64];
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return false;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!asked[dev])
      asked[dev] = hipFuncSetAttribute(reinterpret_cast<const void*>(tile_kernel<T, D, NW, CB, STEP, ANY, PAST>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, kBytes) == hipSuccess;
    if (!asked[dev]) return false;
  }
  tile_kernel<T, D, NW, CB, STEP, ANY, PAST><<<grid_of(plan.units), 64 * NW, kBytes, st>>>(x, plan);
  return true;
}
template <typename T, int D, int NW, int CB, int STEP>
bool launch_tiles(const PagedArgs& x, const Form& f, const TilePlan& plan, hipStream_t st) {
  const bool any = x.c.ps % 16 != 0;
  if constexpr (NW > 1)
    if (f.o_bytes >= kStreamedRecords)
      return any ? launch_tiles_as<T, D, NW, CB, STEP, true, true>(x, plan, st) : launch_tiles_as<T, D, NW, CB, STEP, false, true>(x, plan, st);
  return any ? launch_tiles_as<T, D, NW, CB, STEP, true, false>(x, plan, st) : launch_tiles_as<T, D, NW, CB, STEP, false, false>(x, plan, st);
}

template <typename T, int D>
sl_status launch(const PagedArgs& x, const Form& f, char* ws, hipStream_t st) {
  const int64_t rh = (int64_t)x.a.Hq * x.b.rows;
  if (f.tiles) {
    TilePlan plan = f.plan;
    if (f.buckets) {
      plan.most_tiles = (int)f.most_tiles;
      plan.counts = reinterpret_cast<int32_t*>(ws + f.o_bytes + 2 * f.lse_bytes);
      plan.first_tile = plan.counts + plan.buckets;
      plan.records = reinterpret_cast<int4*>(plan.counts + align_up(2 * (size_t)plan.buckets, 64));
      plan.ranks = reinterpret_cast<int32_t*>(plan.records + f.most_tiles);
      plan.items = plan.ranks + rh * x.a.topk;
      const int64_t blocks = div_up(plan.buckets, 1024);
      zero_kernel<<<(unsigned)(blocks < 1024 ? blocks : 1024), 256, 0, st>>>(plan.counts, plan.buckets);
      const int64_t runs = (int64_t)x.b.rows / kCountRows + x.b.B;
      count_kernel<<<dim3((unsigned)runs, x.c.Hkv), 1024, plan.spans <= kCountSpans ? plan.spans * sizeof(int32_t) : 0, st>>>(x, plan);
      tiles_kernel<<<1, 1024, 0, st>>>(plan, f.cols_log2);
      items_kernel<<<grid_of(div_up(rh * x.a.topk, 256)), 256, 0, st>>>(x, plan, f.cols_log2);
    }
    bool done;
    if constexpr (sizeof(T) == 2)
      done = f.cols_log2 == 5   ? launch_tiles<T, D, 1, 1, 32>(x, f, plan, st)
             : f.cols_log2 == 7 ? launch_tiles<T, D, 4, 1, 64>(x, f, plan, st)
                                : launch_tiles<T, D, 4, 2, 64>(x, f, plan, st);
    else
      done = launch_tiles<T, D, 4, 1, 64>(x, f, plan, st);
    if (!done) return SL_ERR_LAUNCH;
  }
  if constexpr (sizeof(T) == 4) {
    if (f.whole) {
      whole_rows_kernel<T, D><<<grid_of(rh), 256, 0, st>>>(x);
      return hipGetLastError() == hipSuccess ? SL_OK : SL_ERR_LAUNCH;
    }
    if (!f.tiles) rows_kernel<T, D><<<grid_of(rh * x.p.count), 256, 0, st>>>(x);
  }
  if (x.p.count == 1 && f.tiles) {
    mend_kernel<T, D, true><<<grid_of(div_up(rh, 256)), 256, 0, st>>>(x);
  } else {
    // A wavefront a row, or half of one, where there are rows enough, or pieces few enough to be asked for at once (16 dense sequences,
    // 1100 rows and heads of 30 pieces: 7.0 us by four wavefronts, 4.0 so).
    constexpr int kAtOnce = 4 * 64 / (D * (int)sizeof(typename Record<T>::Value) / 16);
    if (rh >= 4096 && x.p.count <= 1024) {
      if (f.tiles) mend_kernel<T, D, false><<<grid_of(div_up(rh, 256)), 256, 0, st>>>(x);
      if (x.p.count <= 32) merge_kernel<T, D, 32, false><<<grid_of(div_up(rh, 8)), 256, 8 * x.p.count * sizeof(float), st>>>(x);
      else merge_kernel<T, D, 64, false><<<grid_of(div_up(rh, 4)), 256, 4 * x.p.count * sizeof(float), st>>>(x);
    } else if (x.p.count <= kAtOnce) {
      merge_kernel<T, D, 64, true><<<grid_of(div_up(rh, 4)), 256, 4 * x.p.count * sizeof(float), st>>>(x);
    } else {
      merge_kernel<T, D, 256, true><<<grid_of(rh), 256, x.p.count * sizeof(float), st>>>(x);
    }
  }
  return hipGetLastError() == hipSuccess ? SL_OK : SL_ERR_LAUNCH;
}

}  // namespace

size_t paged_attention_ws_bytes(const PageCache& c, const PagedBatch& b, const PagedAttention& a) {
  const Form f = form_of(c, b, a);
  return f.o_bytes + 2 * f.lse_bytes + f.plan_bytes;
}

sl_status paged_attention(const PageCache& c, const PagedBatch& b, const PagedAttention& a, const void* Q, const int32_t* idx,
                          const float* scores, void* O, float* LSE, void* ws, hipStream_t st) {
  const Form f = form_of(c, b, a);
  char* const at = static_cast<char*>(ws);
  PagedArgs x = {c, b, a, f.p, Q, idx, scores, O, LSE, ws, reinterpret_cast<float*>(at + f.o_bytes),
                 reinterpret_cast<float*>(at + f.o_bytes + f.lse_bytes), a.scale * kLog2e,
                 f.tiles};
  if (c.dtype == SL_BF16) return c.D == 128 ? launch<bf16_t, 128>(x, f, at, st) : launch<bf16_t, 64>(x, f, at, st);
  return c.D == 128 ? launch<float, 128>(x, f, at, st) : launch<float, 64>(x, f, at, st);
}

}  // namespace sl
