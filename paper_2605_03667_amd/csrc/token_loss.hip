// Log-probabilities of tokens from logits and the losses on them, with their gradients
// (the formulas are in include/elas_loss.h).
//
// Bound by HBM: about 8 instructions and an exponential or two a value against one read and one write of it.  So a row
// is read once: a team of 1 to 16 waves holds it in registers, finds its maximum and the sum of
// exp2((x - max) scale log2(e)), then the token's own terms, and writes the gradient.  The maximum is of the
// logits themselves, so that a row of nothing but a type's lowest value is a uniform distribution at
// any scale.  Statistics are 64-bit sums per workgroup over its rows, added up by a second launch.  65536 x 32000
// bf16 with gradient: 1514 to 1538 us, 5.5 TB/s (read twice: 2153); 16381 x 32000 bf16, an eighth padding
// and a sixth of weight 0: 329; 2000 x 32000 float32: 86; 4093 x 32003 float32 without one: 72.
#include <math.h>

#include <algorithm>

#include "../../include/elas_loss.h"
#include "internal.h"
#include "spans.h"

namespace elas {

namespace {

// Most workgroups that take rows.  More than the card holds at once, so that those with masked rows do not
// leave it idle at the end (16381 x 32000, a quarter masked: 373 us with 1024, 366 with 2048, 352 with 4096, 333 with 8192).
constexpr int kGroups = 8192;
constexpr int kSums = 3;                 // statistics of a workgroup
constexpr float kLowest = -0x1.fffffep127f;
constexpr float kLog2E = 0x1.715476p0f;

// Operands of a launch.
struct Rows {
  const void *logits, *ids;
  void* dlogits;
  const float *weight, *advantage, *old_logp, *ref_logp;
  float *logp, *lse;
  double* part;
  int64_t T, ld, ld_out;
  int32_t V;
  float scale, reduce, z_coef, low, high, kl_coef;
  bool ids_i64;
};

__device__ __forceinline__ int64_t id_of(const void* ids, bool i64, int64_t t) {
  return i64 ? ((const int64_t*)ids)[t] : (int64_t)((const int32_t*)ids)[t];
}

// A maximum and the sum of exp2((x - max) c) of the values it is of.
struct MaxSum {
  float m = kLowest, s = 0.f;
  __device__ __forceinline__ void rescale(float to, float c) {
    s *= __builtin_amdgcn_exp2f((m - to) * c);
    m = to;
  }
};

// exp(q) - 1 - q without cancellation: near 0 by its series, the next term of which is 2^-28 of the sum at 1/2.
__device__ __forceinline__ float exp_minus_line(float q) {
  if (fabsf(q) < 0.5f) {
    float s = 1.f / 9.f;
    s = fmaf(s, q, 1.f) * (1.f / 8.f);
    s = fmaf(s, q, 1.f) * (1.f / 7.f);
    s = fmaf(s, q, 1.f) * (1.f / 6.f);
    s = fmaf(s, q, 1.f) * (1.f / 5.f);
    s = fmaf(s, q, 1.f) * (1.f / 4.f);
    s = fmaf(s, q, 1.f) * (1.f / 3.f);
    s = fmaf(s, q, 1.f) * (1.f / 2.f);
    return s * q * q;
  }
  return q == INFINITY ? q : expm1f(q) - q;
}

// ln of a sum of exponentials; its two parts are added in 64 bits.
__device__ __forceinline__ double log_of(float s) {
  int k;
  float f = frexpf(s, &k);
  if (f < 0x1.6a09e6p-1f) f *= 2.f, --k;
  return fma((double)k, 0x1.62e42fefa39efp-1, (double)logf(f));
}

// What a row's label and every value of it get: dlogits_j = label [j = id] + all exp2((x_j - max) c),
// and the row's statistics.
struct Terms {
  float label, all;
  double sum[kSums];
};

template <int KIND>
__device__ __forceinline__ Terms row_terms(const Rows& a, int64_t t, float w, float x, const MaxSum& row, float* logp_out, float* lse_out) {
  const double ln = log_of(row.s);
  const double logp = ((double)x - (double)row.m) * (double)a.scale - ln, lse = (double)row.m * (double)a.scale + ln;
  *logp_out = (float)logp;
  *lse_out = (float)lse;
  Terms r{};
  if (KIND == LogitsArgs::LOGP) return r;
  const float c = a.reduce * w;
  float at_label, everywhere;
  if (KIND == LogitsArgs::TOKEN) {
    // (a coefficient of 0 takes no part, infinite as lse may be)
    const bool zed = a.z_coef != 0.f;
    const double z = zed ? (double)c * (double)a.z_coef * lse * lse : 0.0;
    r.sum[0] = z - (double)c * logp;
    r.sum[1] = z;
    at_label = -c;
    everywhere = zed ? c * (1.f + 2.f * a.z_coef * (float)lse) : c;
  } else {
    const float adv = a.advantage[t];
    const float ratio = a.old_logp ? expf((float)(logp - (double)a.old_logp[t])) : 1.f;
    const bool held = adv > 0.f ? ratio > a.high : adv < 0.f && ratio < a.low;
    const float bounded = fminf(fmaxf(ratio, a.low), a.high);
    // (an advantage or a coefficient of 0 takes no part where the exponential beside it passes float32's range)
    const float gain = adv == 0.f && ratio == INFINITY ? 0.f : ratio * adv;
    float loss = -(held ? bounded * adv : gain), g = held ? 0.f : -gain, k = 0.f;
    if (a.ref_logp) {
      const float q = (float)((double)a.ref_logp[t] - logp);
      k = exp_minus_line(q);
      if (a.kl_coef != 0.f) {
        loss = fmaf(a.kl_coef, k, loss);
        g = fmaf(-a.kl_coef, expm1f(q), g);
      }
    }
    r.sum[0] = (double)c * (double)loss;
    r.sum[1] = (double)c * (double)k;
    r.sum[2] = held ? (double)c : 0.0;
    at_label = c * g;
    everywhere = -at_label;
  }
  r.label = a.scale * at_label;
  r.all = a.scale * everywhere / row.s;
  return r;
}

// How a row is cut: pieces of 16 bytes from `lead` on, the first that is aligned in the matrix
// that is written (or, without one, read), `full` of them; and the values in front of and behind them,
// one to a thread.  (8000 rows of 50257 bf16 logits, half of them not even 4-byte aligned: 358 us, 402 with pieces
// from the row's first value on; without a gradient 140 and 170.)
template <class E>
struct Cut {
  static constexpr int N = Span<E>::N;
  int lead, full, edges;
  __device__ __forceinline__ Cut(const E* row, int V) {
    lead = (int)(-(uintptr_t)row % 16 / sizeof(E));
    if (lead > V) lead = V;
    full = (V - lead) / N;
    edges = V - full * N;
  }
  // place of a thread's value outside the pieces; only the first `edges` threads have one
  __device__ __forceinline__ int edge(int tid) const { return tid < lead ? tid : full * N + tid; }
};

// A thread's place `i` values behind a row's uniform one: a 32-bit offset, so that the address stays in scalar registers.
template <class E>
__device__ __forceinline__ E* at_value(E* uniform, int i) {
  return (E*)((char*)uniform + (uint32_t)i * (uint32_t)sizeof(E));
}
template <class E>
__device__ __forceinline__ const E* at_value(const E* uniform, int i) {
  return (const E*)((const char*)uniform + (uint32_t)i * (uint32_t)sizeof(E));
}

// Maximum and sum of a thread's pieces i, i + stride .. of a row, 2 pieces at a time (200000 x 1000 bf16
// without a gradient 80 us, with 4 at a time 98, the others alike).
template <class E, bool STREAM>
__device__ __forceinline__ void add_pieces(MaxSum& r, float c, const E* pieces, int i, int full, int stride) {
  constexpr int N = Span<E>::N, AT_ONCE = 2;
  for (; i < full; i += AT_ONCE * stride) {
    Span<E> p[AT_ONCE];
#pragma unroll
    for (int q = 0; q < AT_ONCE; ++q) {
      p[q].clear();
      if (i + q * stride < full) p[q].template load<STREAM>(at_value(pieces, (i + q * stride) * N));
    }
    float m = r.m;
#pragma unroll
    for (int q = 0; q < AT_ONCE; ++q)
#pragma unroll
      for (int k = 0; k < N; ++k) m = fmaxf(m, p[q].get(k));
    r.rescale(m, c);
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < AT_ONCE; ++q)
#pragma unroll
      for (int k = 0; k < N; ++k) s += __builtin_amdgcn_exp2f((p[q].get(k) - m) * c);
    r.s += s;
  }
}
// The same by a team of few waves, whose threads have long chains of groups: added up in sixteens, and those in turn, so that
// there are at most 16 + V / 16384 one behind another and not V / 1024, each of which may lose half a step beside a large first one.
// (4093 x 32003 float32 91 us either way, 8192 x 50257 bf16 142; a team of 16 waves has V / 8192 without it.)
template <class E>
__device__ __forceinline__ void add_long_pieces(MaxSum& r, float c, const E* pieces, int i, int full, int stride) {
  const int run = 16 * 2 * stride;
  for (; i < full; i += run) {
    MaxSum near;
    near.m = r.m;
    add_pieces<E, false>(near, c, pieces, i, full - i > run ? i + run : full, stride);
    r.rescale(near.m, c);
    r.s += near.s;
  }
}
__device__ __forceinline__ void add_value(MaxSum& r, float c, float v) {
  r.rescale(fmaxf(r.m, v), c);
  r.s += __builtin_amdgcn_exp2f((v - r.m) * c);
}
__device__ __forceinline__ void add(MaxSum& r, float c, const MaxSum& o) {
  const float m = fmaxf(r.m, o.m);
  r.rescale(m, c);
  r.s += o.s * __builtin_amdgcn_exp2f((o.m - m) * c);
}

// The threads' maxima and sums to the row's, in every thread; returns the label's logit.  `lds` holds
// 2 WAVES + 1 floats; used in turn, two of them need no other barrier.
template <int WAVES, class E>
__device__ __forceinline__ float whole_row(MaxSum& r, float c, const E* label, float* lds) {
  const int tid = threadIdx.x;
  r.rescale(wave_max(r.m), c);
  r.s = wave_sum(r.s);
  if constexpr (WAVES == 1) return span_value(*label);
  if ((tid & 63) == 0) lds[tid >> 6] = r.m, lds[WAVES + (tid >> 6)] = r.s;
  if (tid == 0) lds[2 * WAVES] = span_value(*label);   // before any wave writes the row in place
  __syncthreads();
  float m = lds[0], s = 0.f;
#pragma unroll
  for (int k = 1; k < WAVES; ++k) m = fmaxf(m, lds[k]);
#pragma unroll
  for (int k = 0; k < WAVES; ++k) s += lds[WAVES + k] * __builtin_amdgcn_exp2f((lds[k] - m) * c);
  r.m = m, r.s = s;
  return lds[2 * WAVES];
}

// Waves to a row; a workgroup of rows of one wave takes kRowsOfOne of them.
constexpr int kRowsOfOne = 4;
template <int WAVES>
struct Team {
  static constexpr int THREADS = WAVES * 64, ROWS = WAVES == 1 ? kRowsOfOne : 1;
};

// Which of its workgroup's rows a wave's team takes, in a scalar register.
template <int WAVES>
__device__ __forceinline__ int wave_row() {
  return WAVES == 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0;
}

// A team's statistics, in shared memory: its first thread adds to them, and the workgroup's
// first threads add up the teams'.
template <int WAVES>
struct Sums {
  double (*all)[kSums];
  __device__ __forceinline__ explicit Sums(double (*lds)[kSums]) : all(lds + wave_row<WAVES>()) {
    if (threadIdx.x % Team<WAVES>::THREADS == 0)
#pragma unroll
      for (int k = 0; k < kSums; ++k) (*all)[k] = 0.0;
  }
  __device__ __forceinline__ void add(const double (&v)[kSums]) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) (*all)[k] += v[k];
  }
  static __device__ __forceinline__ void write(const double (*lds)[kSums], double* part) {
    __syncthreads();
    if (threadIdx.x < kSums) {
      double v = lds[0][threadIdx.x];
#pragma unroll
      for (int w = 1; w < Team<WAVES>::ROWS; ++w) v += lds[w][threadIdx.x];
      part[(int64_t)blockIdx.x * kSums + threadIdx.x] = v;
    }
  }
};

__device__ __forceinline__ void write_row(const Rows& a, int64_t t, float logp, float lse) {
  if (a.logp) a.logp[t] = logp;
  if (a.lse) a.lse[t] = lse;
}

// Without a gradient: a row once through its team.
template <int KIND, class E, int WAVES>
__global__ __launch_bounds__(Team<WAVES>::THREADS * Team<WAVES>::ROWS) void rows_kernel(const Rows a) {
  constexpr int TH = Team<WAVES>::THREADS, ROWS = Team<WAVES>::ROWS;
  __shared__ float red[2][2 * WAVES + 1];
  __shared__ double sums[ROWS][kSums];
  const int tid = threadIdx.x % TH;
  const float c = a.scale * kLog2E;
  Sums<WAVES> sum(sums);
  int turn = 0;
  for (int64_t t = (int64_t)blockIdx.x * ROWS + wave_row<WAVES>(); t < a.T; t += (int64_t)gridDim.x * ROWS) {
    const int64_t id = id_of(a.ids, a.ids_i64, t);
    const float w = KIND != LogitsArgs::LOGP && a.weight ? a.weight[t] : 1.f;
    if (id < 0 || id >= a.V || w == 0.f) {
      if (tid == 0) write_row(a, t, 0.f, 0.f);
      continue;
    }
    const E* x = (const E*)a.logits + t * a.ld;
    const Cut<E> cut(x, a.V);
    MaxSum r;
    if constexpr (WAVES == 4)
      add_long_pieces(r, c, x + cut.lead, tid, cut.full, TH);
    else
      add_pieces<E, false>(r, c, x + cut.lead, tid, cut.full, TH);
    if (tid < cut.edges) add_value(r, c, span_value(x[cut.edge(tid)]));
    const float label = whole_row<WAVES>(r, c, x + id, red[turn]);
    turn ^= 1;
    float logp, lse;
    const Terms o = row_terms<KIND>(a, t, w, label, r, &logp, &lse);
    if (tid == 0) {
      write_row(a, t, logp, lse);
      if (KIND != LogitsArgs::LOGP) sum.add(o.sum);
    }
  }
  if (KIND != LogitsArgs::LOGP) sum.write(sums, a.part);
}

// A loss with its gradient, the row in the registers of its team: PARTS pieces to a thread, what lies
// behind the row -inf.  BEYOND: a longer row, whose pieces behind those are read twice (4000 x 160000 bf16: 565 to 599 us, with 12
// held, which spill, 865; 4000 x 131072 float32: 853 us, 1300 with all of it read twice; of these teams' 128 registers up to
// 8 still go to scratch memory).  Loads and stores are non-temporal (65536 x 32000 bf16: 1488 us, with plain
// loads 1548; before them, plain stores too, 1597 for 1537).
template <int KIND, class E, int WAVES, int PARTS, bool BEYOND>
__global__ __launch_bounds__(Team<WAVES>::THREADS * Team<WAVES>::ROWS) void held_kernel(const Rows a) {
  using S = Span<E>;
  constexpr int N = S::N, TH = Team<WAVES>::THREADS, ROWS = Team<WAVES>::ROWS;
  constexpr bool KEEP = N == 4;      // float32: the exponentials take the logits' place
  __shared__ float red[2][2 * WAVES + 1];
  __shared__ double sums[ROWS][kSums];
  const int tid = threadIdx.x % TH;
  const float c = a.scale * kLog2E;
  Sums<WAVES> sum(sums);
  int turn = 0;
  for (int64_t t = (int64_t)blockIdx.x * ROWS + wave_row<WAVES>(); t < a.T; t += (int64_t)gridDim.x * ROWS) {
    const int64_t id = id_of(a.ids, a.ids_i64, t);
    const float w = a.weight ? a.weight[t] : 1.f;
    const E* x = (const E*)a.logits + t * a.ld;
    E* d = (E*)a.dlogits + t * a.ld_out;
    const Cut<E> cut(d, a.V);
    const E* xp = x + cut.lead;
    E* dp = d + cut.lead;
    if (id < 0 || id >= a.V || w == 0.f) {
      const float zero[N] = {};
      for (int i = tid; i < cut.full; i += TH) S::template store<true>(dp + i * N, zero);
      if (tid < cut.edges) set_span_value(d + cut.edge(tid), 0.f);
      if (tid == 0) write_row(a, t, 0.f, 0.f);
      continue;
    }
    S p[PARTS];
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
      p[q].clear();
      if (tid + q * TH < cut.full) p[q].template load<true>(at_value(xp + q * TH * N, tid * N));
    }
    const float edge = tid < cut.edges ? span_value(x[cut.edge(tid)]) : -INFINITY;
    MaxSum r;
    r.m = fmaxf(r.m, edge);
#pragma unroll
    for (int q = 0; q < PARTS; ++q)
#pragma unroll
      for (int k = 0; k < N; ++k) r.m = fmaxf(r.m, p[q].get(k));
    const float own = r.m;
    r.s = __builtin_amdgcn_exp2f((edge - own) * c);
#pragma unroll
    for (int q = 0; q < PARTS; ++q) p[q].keep_packed();
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float e = __builtin_amdgcn_exp2f((p[q].get(k) - own) * c);
        if constexpr (KEEP) p[q].set(k, e);
        s += e;
      }
      r.s += s;
    }
#pragma unroll
    for (int q = 0; q < PARTS; ++q) p[q].keep_packed();
    if constexpr (BEYOND) {
      MaxSum more;
      add_pieces<E, false>(more, c, xp, tid + PARTS * TH, cut.full, TH);
      add(r, c, more);
    }
    const float label = whole_row<WAVES>(r, c, x + id, red[turn]);
    turn ^= 1;
    float logp, lse;
    const Terms o = row_terms<KIND>(a, t, w, label, r, &logp, &lse);
    if (tid == 0) {
      write_row(a, t, logp, lse);
      sum.add(o.sum);
    }
    const int at = (int)id - cut.lead;      // the label's place among the pieces
    const auto put = [&](int first, float (&v)[N]) __attribute__((always_inline)) {     // piece first + tid
      const int in = at - first * N - tid * N;
      if ((unsigned)in < (unsigned)N) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += in == k ? o.label : 0.f;
      }
      if (first + tid < cut.full) S::template store<true>(at_value(dp + first * N, tid * N), v);
    };
    const float all = KEEP ? o.all * __builtin_amdgcn_exp2f((own - r.m) * c) : o.all;
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
      float v[N];
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = (KEEP ? p[q].get(k) : __builtin_amdgcn_exp2f((p[q].get(k) - r.m) * c)) * all;
      put(q * TH, v);
    }
    if constexpr (BEYOND) {
#pragma unroll 4
      for (int first = PARTS * TH; first + tid < cut.full; first += TH) {
        S more;
        more.template load<true>(at_value(xp + first * N, tid * N));
        float v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = __builtin_amdgcn_exp2f((more.get(k) - r.m) * c) * o.all;
        put(first, v);
      }
    }
    if (tid < cut.edges) {
      const float v = __builtin_amdgcn_exp2f((edge - r.m) * c) * o.all;
      set_span_value(d + cut.edge(tid), cut.edge(tid) == (int)id ? v + o.label : v);
    }
  }
  sum.write(sums, a.part);
}

// Few rows: each is split over workgroups, in two launches.  The first leaves every part's maximum and sum, and the
// label's logit (a gradient may take the logits' place); the second joins them, every workgroup for itself, and
// writes its part of the gradient, and one more workgroup, a row to a thread, the rows' results and the statistics.
// 16 rows in a graph: 32000 bf16 6.5 us (9.2 by the kernels above and their sum), 65000 bf16 8.0 (13.0),
// 131072 float32 9.2 (19.5).
struct Split {
  float2* part;       // [T][parts]: maximum, sum
  float* label;       // [T]
  float* stats;
  int parts, per;     // parts of a row (kParts at most), pieces of one
};

// Whether a row takes part.
__device__ __forceinline__ bool row_of(const Rows& a, int64_t t, int64_t& id, float& w) {
  id = id_of(a.ids, a.ids_i64, t);
  w = a.weight ? a.weight[t] : 1.f;
  return id >= 0 && id < a.V && w != 0.f;
}

template <class E>
__global__ __launch_bounds__(256) void split_kernel(const Rows a, const Split sp) {
  __shared__ float red[2 * 4 + 1];
  const int tid = threadIdx.x, part = blockIdx.x;
  const int64_t t = blockIdx.y;
  int64_t id;
  float w;
  if (!row_of(a, t, id, w)) return;
  const float c = a.scale * kLog2E;
  const E* x = (const E*)a.logits + t * a.ld;
  const Cut<E> cut(a.dlogits ? (const E*)a.dlogits + t * a.ld_out : x, a.V);
  MaxSum r;
  const int first = part * sp.per, end = first + sp.per;
  add_pieces<E, false>(r, c, x + cut.lead, first + tid, end < cut.full ? end : cut.full, 256);
  if (part == 0 && tid < cut.edges) add_value(r, c, span_value(x[cut.edge(tid)]));
  const float label = whole_row<4>(r, c, x + id, red);
  if (tid == 0) {
    sp.part[t * sp.parts + part] = make_float2(r.m, r.s);
    if (part == 0) sp.label[t] = label;
  }
}

template <int KIND, class E>
__global__ __launch_bounds__(256) void join_kernel(const Rows a, const Split sp) {
  using S = Span<E>;
  constexpr int N = S::N;
  __shared__ double red[4][kSums];
  const int tid = threadIdx.x, lane = tid & 63, part = blockIdx.x;
  const float c = a.scale * kLog2E;
  if (blockIdx.y == gridDim.y - 1) {
    if (part > 0) return;
    double sum[kSums] = {0.0, 0.0, 0.0};
    for (int64_t t = tid; t < a.T; t += 256) {
      int64_t id;
      float w, logp = 0.f, lse = 0.f;
      if (row_of(a, t, id, w)) {
        MaxSum r;
        for (int k = 0; k < sp.parts; ++k) {
          const float2 v = sp.part[t * sp.parts + k];
          add(r, c, MaxSum{v.x, v.y});
        }
        const Terms o = row_terms<KIND>(a, t, w, sp.label[t], r, &logp, &lse);
#pragma unroll
        for (int k = 0; k < kSums; ++k) sum[k] += o.sum[k];
      }
      write_row(a, t, logp, lse);
    }
    const double v = block_sums<4>(sum, red);
    if (tid < (KIND == LogitsArgs::TOKEN ? 2 : 3)) sp.stats[tid] = (float)v;
    return;
  }
  const int64_t t = blockIdx.y;
  int64_t id;
  float w;
  const bool on = row_of(a, t, id, w);
  const E* x = (const E*)a.logits + t * a.ld;
  E* d = (E*)a.dlogits + t * a.ld_out;
  const Cut<E> cut(d, a.V);
  const int first = part * sp.per + tid, end = (part + 1) * sp.per < cut.full ? (part + 1) * sp.per : cut.full;
  const bool edge = part == 0 && tid < cut.edges;
  MaxSum r;
  Terms o{};
  if (on) {
    if (lane < sp.parts) {
      const float2 v = sp.part[t * sp.parts + lane];
      r.m = v.x, r.s = v.y;
    }
    r.rescale(wave_max(r.m), c);
    r.s = wave_sum(r.s);
    float logp, lse;
    o = row_terms<KIND>(a, t, w, sp.label[t], r, &logp, &lse);
  }
  const int at = on ? (int)id - cut.lead : -1;
  for (int i = first; i < end; i += 256) {
    float v[N] = {};
    if (on) {
      S p;
      p.template load<false>(at_value(x + cut.lead, i * N));
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = __builtin_amdgcn_exp2f((p.get(k) - r.m) * c) * o.all;
      if ((unsigned)(at - i * N) < (unsigned)N) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += at - i * N == k ? o.label : 0.f;
      }
    }
    S::template store<false>(at_value(d + cut.lead, i * N), v);
  }
  if (edge) {
    const int i = cut.edge(tid);
    float v = 0.f;
    if (on) {
      v = __builtin_amdgcn_exp2f((span_value(x[i]) - r.m) * c) * o.all;
      if (i == (int)id) v += o.label;
    }
    set_span_value(d + i, v);
  }
}

__global__ __launch_bounds__(1024) void loss_sum_kernel(const double* part, int groups, int count, float* stats) {
  __shared__ double red[16][kSums];
  double s[kSums] = {0.0, 0.0, 0.0};
  for (int g = threadIdx.x; g < groups; g += 1024) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) s[k] += part[(int64_t)g * kSums + k];
  }
  const double v = block_sums<16>(s, red);
  if ((int)threadIdx.x < count) stats[threadIdx.x] = (float)v;
}

// Gradient from those of logp and lse: every value by itself, kChunk pieces of a row to a thread at a time (8192 x 32000
// bf16, by 4 waves: 168 us with 2, 174 with 4, 176 with 8 or 16).  Bound by HBM: 6.3 TB/s.  A lse is rounded to 2^-24 of itself, and
// exp(z - lse) is off by as much as lse is: up to 64 no more than by the exponent's own roundings at e^-20 (3 of 2^-24 of it each).
// Beyond, the row's sum is taken anew, from one more read of it (8192 x 32000 float32: 618 us, 335 at a lse of 12; always by the row's
// first workgroup, and so on one die in 8: 6025).  A bf16 gradient's own rounding, 2^-9, hides 2^-12, which is 4096.  (Among
// logits of a type's lowest value a lse holds nothing of the sum at all.)
template <class E>
constexpr float kLargeLse = sizeof(E) == 2 ? 4096.f : 64.f;
constexpr int kChunk = 2;

struct BwdRows {
  const void *logits, *ids;
  void* dlogits;
  const float *dlogp, *dlse, *lse;
  int64_t T, ld, ld_out;
  int32_t V, chunks;
  float scale;
  bool ids_i64;
};

template <class E, int TH>
__global__ __launch_bounds__(TH) void logp_bwd_kernel(const BwdRows a) {
  using S = Span<E>;
  constexpr int N = S::N;
  __shared__ float red[2 * (TH / 64) + 1];
  const int tid = threadIdx.x;
  const int64_t items = a.T * a.chunks;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t t = item / a.chunks;
    const int chunk = (int)(item - t * a.chunks);
    const int64_t id = id_of(a.ids, a.ids_i64, t);
    const E* x = (const E*)a.logits + t * a.ld;
    E* d = (E*)a.dlogits + t * a.ld_out;
    const Cut<E> cut(d, a.V);
    const E* xp = x + cut.lead;
    E* dp = d + cut.lead;
    const int first = chunk * kChunk * TH + tid;
    const bool edge = chunk == 0 && tid < cut.edges;
    if (id < 0 || id >= a.V) {
      const float zero[N] = {};
#pragma unroll
      for (int q = 0; q < kChunk; ++q)
        if (first + q * TH < cut.full) S::template store<true>(dp + (first + q * TH) * N, zero);
      if (edge) set_span_value(d + cut.edge(tid), 0.f);
      continue;
    }
    const float g = a.dlogp[t], e = a.dlse ? a.dlse[t] : 0.f, lse = a.lse[t];
    const float at_label = a.scale * g, all = a.scale * (e - g);
    const int at = (int)id - cut.lead;
    if (!(fabsf(lse) <= kLargeLse<E>)) {
      // the whole row by one of its workgroups, which finds its maximum and sum anew: another one from row to row, as workgroups
      // are dealt out to the dies in turn
      if (chunk != (int)((uint32_t)t % (uint32_t)a.chunks)) continue;
      const bool edge = tid < cut.edges;
      const float c = a.scale * kLog2E;
      MaxSum r;
      add_long_pieces(r, c, xp, tid, cut.full, TH);
      if (edge) add_value(r, c, span_value(x[cut.edge(tid)]));
      __syncthreads();      // (`red` may still be read from another such row)
      whole_row<TH / 64>(r, c, x + id, red);
      const float share = all / r.s;
      for (int i = tid; i < cut.full; i += TH) {
        S q;
        q.template load<false>(at_value(xp, i * N));
        float v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = __builtin_amdgcn_exp2f((q.get(k) - r.m) * c) * share + (at - i * N == k ? at_label : 0.f);
        S::template store<false>(at_value(dp, i * N), v);
      }
      if (edge) {
        const int i = cut.edge(tid);
        set_span_value(d + i, __builtin_amdgcn_exp2f((span_value(x[i]) - r.m) * c) * share + (i == (int)id ? at_label : 0.f));
      }
      continue;
    }
    S p[kChunk];
#pragma unroll
    for (int q = 0; q < kChunk; ++q)
      if (first + q * TH < cut.full) p[q].template load<true>(at_value(xp, (first + q * TH) * N));
#pragma unroll
    for (int q = 0; q < kChunk; ++q) {
      const int i = first + q * TH;
      if (i >= cut.full) break;
      float v[N];
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = __builtin_amdgcn_exp2f((p[q].get(k) * a.scale - lse) * kLog2E) * all;
      if ((unsigned)(at - i * N) < (unsigned)N) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += at - i * N == k ? at_label : 0.f;
      }
      S::template store<true>(at_value(dp, i * N), v);
    }
    if (edge) {
      const int i = cut.edge(tid);
      const float v = __builtin_amdgcn_exp2f((span_value(x[i]) * a.scale - lse) * kLog2E) * all;
      set_span_value(d + i, i == (int)id ? v + at_label : v);
    }
  }
}

// ---- host -----------------------------------------------------------------------------

int groups_of(int64_t T) { return (int)std::min<int64_t>(T, kGroups); }

// Whether rows are split, and how: rows of 16 KB and more, of which there are too few for a workgroup each to fill the card.
// In us, split and not: 48 x 32000 bf16 6.8 and 9.4, 128 of them 8.6 and 9.8, 160 x 64000 14.4 and 13.6, 256 x 16000 8.3
// and 7.7; float32, whose second read is twice as long, 48 x 32000 8.0 and 9.0, 96 x 90791 19.0 and 22.1, 128 x 64000 19.1
// and 16.4.  Rows alone do not say it all: 96 x 32000 float32 loses 0.8 us by it (10.2 and 9.4), where 96 x 90791 gains 3.1.  At
// most 16 parts, which one thread joins for the statistics (16 x 131072 float32: 9.2 us with 16, 11.5 with 8, 10.3 with 32).
constexpr int64_t kSplitRowsBf16 = 128, kSplitRowsF32 = 96, kSplitRow = 16384;
constexpr int kParts = 16;
constexpr int64_t split_rows(bool f32) { return f32 ? kSplitRowsF32 : kSplitRowsBf16; }
struct SplitPlan {
  bool split;
  int parts, per;
  SplitPlan(int64_t T, int64_t V, bool f32) {
    const int64_t n = f32 ? 4 : 8, pieces = (V + n - 1) / n, bytes = pieces * 16;
    split = T > 0 && T <= split_rows(f32) && bytes >= kSplitRow;
    const int64_t at_least = (pieces + kParts * 256 - 1) / (kParts * 256);
    per = (int)(256 * std::max<int64_t>(at_least, 2));
    parts = (int)((pieces + per - 1) / per);
  }
  size_t bytes(int64_t T) const { return (size_t)T * ((size_t)parts * sizeof(float2) + sizeof(float)); }
};

template <int KIND, class E>
hipError_t launch_split(const Rows& r, const SplitPlan& plan, void* ws, float* stats, const char* tag, hipStream_t stream) {
  Split sp{};
  sp.part = (float2*)ws;
  sp.label = (float*)(sp.part + r.T * plan.parts);
  sp.stats = stats;
  sp.parts = plan.parts;
  sp.per = plan.per;
  {
    TimedLaunch tl("loss_split", stream);
    hipLaunchKernelGGL(split_kernel<E>, dim3((unsigned)plan.parts, (unsigned)r.T), dim3(256), 0, stream, r, sp);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 grid = r.dlogits ? dim3((unsigned)plan.parts, (unsigned)r.T + 1) : dim3(1, 1);
  TimedLaunch tl(tag, stream);
  hipLaunchKernelGGL((join_kernel<KIND, E>), grid, dim3(256), 0, stream, r, sp);
  return hipGetLastError();
}

template <int WAVES>
dim3 grid_of(int64_t T) {
  return dim3((unsigned)std::min<int64_t>((T + Team<WAVES>::ROWS - 1) / Team<WAVES>::ROWS, kGroups));
}
template <int KIND, class E, int WAVES, int PARTS, bool BEYOND = false>
unsigned launch_held(const Rows& r, hipStream_t stream) {
  const dim3 grid = grid_of<WAVES>(r.T);
  hipLaunchKernelGGL((held_kernel<KIND, E, WAVES, PARTS, BEYOND>), grid, dim3(Team<WAVES>::THREADS * Team<WAVES>::ROWS), 0, stream, r);
  return grid.x;
}
template <int KIND, class E, int WAVES>
unsigned launch_rows(const Rows& r, hipStream_t stream) {
  const dim3 grid = grid_of<WAVES>(r.T);
  hipLaunchKernelGGL((rows_kernel<KIND, E, WAVES>), grid, dim3(Team<WAVES>::THREADS * Team<WAVES>::ROWS), 0, stream, r);
  return grid.x;
}

// The team that holds a row with the fewest idle lanes, of as few waves as leave a SIMD 4 or more of them.  In us, with the
// next team beside it: 100000 x 2900 bf16 224 (4 waves of 2 pieces: 320), 60000 x 6000 262 (4 of 3: 280), 60000 x 8000 343
// (8 of 2: 386), 60000 x 12000 538 (4 of 6: 570), 30000 x 16000 333 (4 of 8: 342), 65536 x 32000 1488 (4 of 16: 1591,
// 16 of 4: 1689), 10000 x 48000 342 (16 of 6: 387), 8000 x 50257 292 (16 of 8: 358), 8000 x 61000
// 370 (16 of 8: 408), 16000 x 32000 float32 680 (8 of 16: 695).  Returns the workgroups.
template <int KIND, class E>
unsigned launch_gradient(const Rows& r, hipStream_t stream) {
  const int pieces = (r.V + Span<E>::N - 1) / Span<E>::N, whole = (pieces + 63) / 64;      // pieces to a lane of one wave
  if (whole <= 2) return launch_held<KIND, E, 1, 2>(r, stream);
  if (whole <= 4) return launch_held<KIND, E, 1, 4>(r, stream);
  if (whole <= 6) return launch_held<KIND, E, 1, 6>(r, stream);
  if (whole <= 8) return launch_held<KIND, E, 1, 8>(r, stream);
  if (whole <= 12) return launch_held<KIND, E, 1, 12>(r, stream);
  if (whole <= 16) return launch_held<KIND, E, 4, 4>(r, stream);
  if (whole <= 24) return launch_held<KIND, E, 8, 3>(r, stream);
  if (whole <= 32) return launch_held<KIND, E, 8, 4>(r, stream);
  if (whole <= 48) return launch_held<KIND, E, 8, 6>(r, stream);
  if (whole <= 56) return launch_held<KIND, E, 8, 7>(r, stream);
  if (whole <= 64) return launch_held<KIND, E, 8, 8>(r, stream);
  if (whole <= 96) return launch_held<KIND, E, 8, 12>(r, stream);
  if (whole <= 112) return launch_held<KIND, E, 8, 14>(r, stream);
  if (whole <= 120) return launch_held<KIND, E, 8, 15>(r, stream);
  if (whole <= 128) return launch_held<KIND, E, 16, 8>(r, stream);
  if (whole <= 192) return launch_held<KIND, E, 16, 12>(r, stream);
  if (whole <= 256) return launch_held<KIND, E, 16, 16>(r, stream);
  return launch_held<KIND, E, 16, sizeof(E) == 2 ? 6 : 16, true>(r, stream);
}
template <int KIND, class E>
unsigned launch_rows(const Rows& r, hipStream_t stream) {
  if constexpr (KIND != LogitsArgs::LOGP)
    if (r.dlogits) return launch_gradient<KIND, E>(r, stream);
  const int64_t bytes = (int64_t)r.V * sizeof(E);
  // (100000 x 5000 bf16: 176 us by a wave a row, 209 by 4; 16 x 131072 float32: 9.1 by 16 waves, 24.3 by 4; 512 x 32000
  // bf16: 6.5 and 7.0; 1000 x 32000: 13.3 and 12.6)
  if (bytes <= 16384) return launch_rows<KIND, E, 1>(r, stream);
  if (r.T <= 512) return launch_rows<KIND, E, 16>(r, stream);
  return launch_rows<KIND, E, 4>(r, stream);
}
template <int KIND>
hipError_t launch_rows(const Rows& r, bool f32, const char* tag, unsigned* groups, hipStream_t stream) {
  TimedLaunch tl(tag, stream);
  *groups = f32 ? launch_rows<KIND, float>(r, stream) : launch_rows<KIND, uint16_t>(r, stream);
  return hipGetLastError();
}

}  // namespace

// (never less for fewer tokens, so that what the largest batch needs will do for all)
size_t token_loss_workspace_bytes(int64_t T, int64_t V, bool f32) {
  const int64_t few = std::min(T, split_rows(f32));
  const SplitPlan plan(few, V, f32);
  return std::max(plan.split ? plan.bytes(few) : 0, (size_t)groups_of(T) * kSums * sizeof(double));
}

hipError_t run_token_loss(const LogitsArgs& a, hipStream_t stream) {
  Rows r{};
  r.logits = a.logits; r.ids = a.ids; r.dlogits = a.dlogits; r.weight = a.weight; r.advantage = a.advantage; r.old_logp = a.old_logp;
  r.ref_logp = a.ref_logp; r.logp = a.logp; r.lse = a.lse; r.part = (double*)a.ws; r.T = a.T; r.ld = a.ld; r.ld_out = a.ld_out;
  r.V = (int32_t)a.V; r.scale = a.scale; r.reduce = a.reduce; r.z_coef = a.z_coef; r.low = a.low; r.high = a.high; r.kl_coef = a.kl_coef;
  r.ids_i64 = a.ids_i64;
  const SplitPlan plan(a.T, a.V, a.f32);
  if (plan.split && a.kind != LogitsArgs::LOGP) {
    const auto launch = [&](auto f32, auto bf16, const char* tag) { return (a.f32 ? f32 : bf16)(r, plan, a.ws, a.stats, tag, stream); };
    return a.kind == LogitsArgs::TOKEN ? launch(launch_split<LogitsArgs::TOKEN, float>, launch_split<LogitsArgs::TOKEN, uint16_t>, "token_loss")
                                       : launch(launch_split<LogitsArgs::POLICY, float>, launch_split<LogitsArgs::POLICY, uint16_t>, "policy_loss");
  }
  unsigned groups = 0;
  if (a.T > 0) {
    const hipError_t e = a.kind == LogitsArgs::LOGP    ? launch_rows<LogitsArgs::LOGP>(r, a.f32, "token_logp", &groups, stream)
                         : a.kind == LogitsArgs::TOKEN ? launch_rows<LogitsArgs::TOKEN>(r, a.f32, "token_loss", &groups, stream)
                                                       : launch_rows<LogitsArgs::POLICY>(r, a.f32, "policy_loss", &groups, stream);
    if (e != hipSuccess || a.kind == LogitsArgs::LOGP) return e;
  }
  TimedLaunch tl("loss_sum", stream);
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(1024), 0, stream, (const double*)a.ws, (int)groups, a.kind == LogitsArgs::TOKEN ? 2 : 3,
                     a.stats);
  return hipGetLastError();
}

hipError_t run_token_logp_bwd(const LogitsArgs& a, hipStream_t stream) {
  BwdRows r{};
  r.logits = a.logits; r.ids = a.ids; r.dlogits = a.dlogits; r.dlogp = a.dlogp; r.dlse = a.dlse; r.lse = a.lse_in; r.T = a.T; r.ld = a.ld;
  r.ld_out = a.ld_out; r.V = (int32_t)a.V; r.scale = a.scale; r.ids_i64 = a.ids_i64;
  // (a wave where it takes a row at once, else two, so that few lanes idle: 60000 x 1000 bf16 43 us, 71 by workgroups of 4;
  // 100000 x 5000 359, 431 by 4; 65536 x 32000 1407 and 1428)
  const int64_t pieces = (a.V + (a.f32 ? 3 : 7)) / (a.f32 ? 4 : 8);
  const int threads = pieces <= kChunk * 64 ? 64 : 128;
  r.chunks = (int32_t)((pieces + kChunk * threads - 1) / (kChunk * threads));
  TimedLaunch tl("token_logp_bwd", stream);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(a.T * r.chunks, 1 << 20)), dim3((unsigned)threads), 0, stream, r);
  };
  if (threads == 64)
    a.f32 ? launch(logp_bwd_kernel<float, 64>) : launch(logp_bwd_kernel<uint16_t, 64>);
  else
    a.f32 ? launch(logp_bwd_kernel<float, 128>) : launch(logp_bwd_kernel<uint16_t, 128>);
  return hipGetLastError();
}

}  // namespace elas
