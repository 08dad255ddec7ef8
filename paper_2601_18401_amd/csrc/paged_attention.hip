// Span-attention of new tokens over a paged cache.
//
// A row's keys are the tokens of its selected spans and of its window.  They are cut into pieces; a piece's softmax gives
// a normalised output and a log-sum-exp (in log2 units), and a merge joins a row's pieces: exp2(lse_p - lse) of each for the
// joint form, and for the gated one alpha_t * exp2(lse_p - lse_t) summed over the slots t that the piece belongs to.
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
  float* part_o;    // [Hq * rows][count][D]
  float* part_lse;  // [Hq * rows][count]
  float scale_log2e;
};

__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }  // NaN stays
// exp2(a - b) where a = -inf means nothing, also beside b = -inf
__device__ __forceinline__ float weight_of(float a, float b) { return a == -INFINITY ? 0.f : fast_exp2(a - b); }

// Grids of more than 2^20 workgroups go on in y (a launch holds fewer than 2^32 threads in x).
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

struct RowPlace {
  int s, pos;  // sequence and position; pos < 0: a row without a token
};
__device__ __forceinline__ RowPlace place_of_row(const PagedArgs& x, int e, int row) {
  const int s = x.b.seqs[e], len = length_of(x.c, s), pos = len - (x.b.cu[e + 1] - row);
  return {s, pos >= len || pos >= x.b.L ? -1 : pos};
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

// Wavefront u takes piece u % count of row-and-head u / count.
template <typename T, int D>
__global__ __launch_bounds__(256) void rows_kernel(const PagedArgs x) {
  using RS = RowState<T, D>;
  const int lane = threadIdx.x & 63;
  const int64_t u = workgroup() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= (int64_t)x.a.Hq * x.b.rows * x.p.count) return;
  const int rh = (int)(u / x.p.count), part = (int)(u - (int64_t)rh * x.p.count);
  const int h = rh / x.b.rows, row = rh - h * x.b.rows;
  if (row < x.b.cu[0] || row >= x.b.cu[x.b.B]) return;
  const RowPlace at = place_of_row(x, entry_of_row(x.b.cu, x.b.B, row), row);
  RS st;
  st.clear();
  if (at.pos >= 0) {
    const PieceRange r = range_of_piece(x, at.pos, part, x.idx + h * x.a.ish + row * x.a.ist);
    if (r.t0 < r.t1) {
      float q[RS::EPL];
      Elem<T>::unpack(load16(static_cast<const T*>(x.Q) + h * x.a.qsh + row * x.a.qst + lane % RS::LPR * RS::EPL), q);
#pragma unroll
      for (int e = 0; e < RS::EPL; ++e) q[e] *= x.scale_log2e;
      const int64_t base = x.b.layer * x.c.layer + h / x.a.G * x.c.head;
      st.template attend<4>(x.c, static_cast<const T*>(x.c.K) + base, static_cast<const T*>(x.c.V) + base,
                            x.c.tables + (int64_t)at.s * x.c.max_pages, q, r.t0, r.t1, lane);
      st.join_groups();
    }
  }
  if (lane == 0) x.part_lse[u] = st.m == -INFINITY ? -INFINITY : st.m + __log2f(st.l);
  if (lane < RS::LPR && !(st.m == -INFINITY)) {
    const float inv = 1.f / st.l;
#pragma unroll
    for (int e = 0; e < RS::EPL; e += 4)
      *reinterpret_cast<float4*>(x.part_o + u * D + lane * RS::EPL + e) =
          make_float4(st.o[e] * inv, st.o[e + 1] * inv, st.o[e + 2] * inv, st.o[e + 3] * inv);
  }
}

// ------------------------------------------------------------------ merge
// A workgroup joins the pieces of one row and head: weights to LDS, then D / 4 lanes a piece.
template <typename T, int D>
__global__ __launch_bounds__(256) void merge_kernel(const PagedArgs x) {
  extern __shared__ float s_w[];  // [count]
  __shared__ float s_red[8];
  __shared__ float s_gate[SL_MAX_TOPK], s_lse[SL_MAX_TOPK];
  constexpr int LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ float4 s_o[GROUPS][LANES];
  if (workgroup() >= (int64_t)x.a.Hq * x.b.rows) return;
  const int rh = (int)workgroup(), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, P = x.p.count;
  const int h = rh / x.b.rows, row = rh - h * x.b.rows;
  if (row < x.b.cu[0] || row >= x.b.cu[x.b.B]) return;
  const float* const lse = x.part_lse + (int64_t)rh * P;
  auto all_max = [&](float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = max_of(v, __shfl_xor(v, off, 64));
    __syncthreads();
    if (lane == 0) s_red[wave] = v;
    __syncthreads();
    return max_of(max_of(s_red[0], s_red[1]), max_of(s_red[2], s_red[3]));
  };
  auto all_sum = [&](float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if (lane == 0) s_red[wave] = v;
    __syncthreads();
    return (s_red[0] + s_red[1]) + (s_red[2] + s_red[3]);
  };
  // log2-sum-exp2 of pieces [from, to)
  auto lse_of = [&](int from, int to) {
    float v = -INFINITY;
    for (int k = from + tid; k < to; k += 256) v = max_of(v, lse[k]);
    const float m = all_max(v);
    if (m == -INFINITY) return m;
    float l = 0.f;
    for (int k = from + tid; k < to; k += 256) l += weight_of(lse[k], m);
    return m + __log2f(all_sum(l));
  };
  const int routed = x.a.topk * x.p.routed;
  float total = -INFINITY;
  bool any = false;  // a slot holds a span
  if (x.a.combined) {
    const RowPlace at = place_of_row(x, entry_of_row(x.b.cu, x.b.B, row), row);
    const float near = lse_of(routed, P);
    float score = -INFINITY;
    bool mine = false;
    if (tid < x.a.topk) {
      const int64_t i = h * x.a.ish + row * x.a.ist + tid;
      const int j = x.idx[i];
      mine = at.pos >= 0 && j >= 0 && j < at.pos / x.a.S;
      if (mine) score = x.scores[i];
      float m = near;
      for (int k = 0; k < x.p.routed; ++k) m = max_of(m, lse[tid * x.p.routed + k]);
      float l = weight_of(near, m);
      for (int k = 0; k < x.p.routed; ++k) l += weight_of(lse[tid * x.p.routed + k], m);
      s_lse[tid] = m == -INFINITY ? m : m + __log2f(l);
    }
    any = __syncthreads_or(mine);
    if (any) {
      const float top = all_max(score);
      const float e = mine ? fast_exp2((score - top) * kLog2e) : 0.f;
      const float sum = all_sum(e);
      if (tid < x.a.topk) s_gate[tid] = e / sum;
      __syncthreads();
      for (int k = tid; k < P; k += 256) {
        float w = 0.f;
        if (k < routed) {
          const int t = k / x.p.routed;
          if (s_gate[t] != 0.f) w = s_gate[t] * weight_of(lse[k], s_lse[t]);
        } else {
          for (int t = 0; t < x.a.topk; ++t)
            if (s_gate[t] != 0.f) w += s_gate[t] * weight_of(lse[k], s_lse[t]);
        }
        s_w[k] = w;
      }
    }
  }
  if (!any) {
    total = lse_of(x.a.combined ? routed : 0, P);
    for (int k = tid; k < P; k += 256) s_w[k] = x.a.combined && k < routed ? 0.f : weight_of(lse[k], total);
    if (tid == 0 && x.LSE) x.LSE[rh] = total * kLn2;
  }
  __syncthreads();
  const int g = tid / LANES, c = tid % LANES;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const float4* const po = reinterpret_cast<const float4*>(x.part_o + (int64_t)rh * P * D) + c;
  for (int k = g; k < P; k += GROUPS) {
    const float w = s_w[k];
    if (w == 0.f) continue;  // (a piece without tokens has written no output)
    const float4 v = po[(int64_t)k * LANES];
    acc.x = fmaf(w, v.x, acc.x);
    acc.y = fmaf(w, v.y, acc.y);
    acc.z = fmaf(w, v.z, acc.z);
    acc.w = fmaf(w, v.w, acc.w);
  }
  s_o[g][c] = acc;
  __syncthreads();
  if (tid < D) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) v += reinterpret_cast<const float*>(s_o[k])[tid];
    Elem<T>::store1(static_cast<T*>(x.O) + (int64_t)rh * D + tid, v);
  }
}

// ------------------------------------------------------------------ host
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
dim3 grid_of(int64_t workgroups) {
  constexpr int64_t kMost = 1 << 20;
  return workgroups <= kMost ? dim3((unsigned)workgroups) : dim3((unsigned)kMost, (unsigned)div_up(workgroups, kMost));
}

// Pieces of at least 64 tokens, enough of them for 4096 wavefronts.
Pieces pieces_of(const PagedBatch& b, const PagedAttention& a) {
  const int64_t rh = (int64_t)a.Hq * b.rows, window = a.S < b.L ? a.S : b.L;
  Pieces p = {1, a.S, 1, (int)window, 0};
  auto cut = [](int64_t tokens, int64_t units, int64_t most) {
    int64_t n = div_up(4096, units);
    if (n > most) n = most;
    if (n > div_up(tokens, 64)) n = div_up(tokens, 64);
    return n < 1 ? 1 : n;
  };
  if (a.topk > 0) {
    p.routed_tokens = (int)div_up(a.S, cut(a.S, rh * a.topk, 64));
    p.routed = (int)div_up(a.S, p.routed_tokens);
  }
  p.window_tokens = (int)div_up(window, cut(window, rh, 256));
  p.window = (int)div_up(window, p.window_tokens);
  p.count = a.topk * p.routed + p.window;
  return p;
}

template <typename T, int D>
sl_status launch(const PagedArgs& x, hipStream_t st) {
  const int64_t rh = (int64_t)x.a.Hq * x.b.rows;
  rows_kernel<T, D><<<grid_of(div_up(rh * x.p.count, 4)), 256, 0, st>>>(x);
  merge_kernel<T, D><<<grid_of(rh), 256, x.p.count * sizeof(float), st>>>(x);
  return hipGetLastError() == hipSuccess ? SL_OK : SL_ERR_LAUNCH;
}

}  // namespace

size_t paged_attention_ws_bytes(const PageCache& c, const PagedBatch& b, const PagedAttention& a) {
  const Pieces p = pieces_of(b, a);
  const size_t records = (size_t)a.Hq * b.rows * p.count;
  return align_up(records * c.D * sizeof(float), 256) + align_up(records * sizeof(float), 256);
}

sl_status paged_attention(const PageCache& c, const PagedBatch& b, const PagedAttention& a, const void* Q, const int32_t* idx,
                          const float* scores, void* O, float* LSE, void* ws, hipStream_t st) {
  PagedArgs x = {c, b, a, pieces_of(b, a), Q, idx, scores, O, LSE, static_cast<float*>(ws), nullptr, a.scale * kLog2e};
  x.part_lse = reinterpret_cast<float*>(static_cast<char*>(ws) +
                                        align_up((size_t)a.Hq * b.rows * x.p.count * c.D * sizeof(float), 256));
  if (c.dtype == SL_BF16) return c.D == 128 ? launch<bf16_t, 128>(x, st) : launch<bf16_t, 64>(x, st);
  return c.D == 128 ? launch<float, 128>(x, st) : launch<float, 64>(x, st);
}

}  // namespace sl
