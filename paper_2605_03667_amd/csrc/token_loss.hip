// Log-probabilities of tokens from logits and the losses on them, with their gradients
// (the formulas are in include/elas_loss.h).
//
// A workgroup takes a row at a time: one pass for the running maximum and the sum of
// exp2((x - max) scale log2(e)), then the token's own terms, then, where a gradient is wanted, a second
// pass that writes it.  The maximum is of the logits themselves, so that a row of nothing
// but a type's lowest value is a uniform distribution at any scale.  Statistics are 64-bit
// sums per workgroup over its rows, added up by a second launch.
#include <math.h>

#include <algorithm>

#include "../../include/elas_loss.h"
#include "internal.h"
#include "spans.h"

namespace elas {

namespace {

constexpr int kGroups = 2048;            // most workgroups that take rows
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
  return expm1f(q) - q;
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
    float loss = -(held ? bounded * adv : ratio * adv), g = held ? 0.f : -ratio * adv, k = 0.f;
    if (a.ref_logp) {
      const float q = (float)((double)a.ref_logp[t] - logp);
      k = exp_minus_line(q);
      loss = fmaf(a.kl_coef, k, loss);
      g = fmaf(-a.kl_coef, expm1f(q), g);
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

template <int KIND, class E, int WAVES, bool GRAD>
__global__ __launch_bounds__(WAVES * 64) void rows_kernel(const Rows a) {
  using S = Span<E>;
  constexpr int N = S::N, TH = WAVES * 64;
  __shared__ float red[2][2 * WAVES + 1];
  const int tid = threadIdx.x;
  const float c = a.scale * kLog2E;
  const int full = a.V / N, rest = a.V - full * N;       // whole pieces, and values behind them
  double sum[kSums] = {0.0, 0.0, 0.0};
  int turn = 0;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const int64_t id = id_of(a.ids, a.ids_i64, t);
    const float w = KIND != LogitsArgs::LOGP && a.weight ? a.weight[t] : 1.f;
    const E* x = (const E*)a.logits + t * a.ld;
    E* d = GRAD ? (E*)a.dlogits + t * a.ld_out : nullptr;
    if (id < 0 || id >= a.V || w == 0.f) {
      if (GRAD) {
        const float zero[N] = {};
        for (int i = tid; i < full; i += TH) S::template store<false>(d + i * N, zero);
        if (tid < rest) set_span_value(d + full * N + tid, 0.f);
      }
      if (tid == 0) {
        if (a.logp) a.logp[t] = 0.f;
        if (a.lse) a.lse[t] = 0.f;
      }
      continue;
    }
    MaxSum r;
    for (int i = tid; i < full; i += TH) {
      S p;
      p.template load<false>(x + i * N);
      float m = r.m;
#pragma unroll
      for (int k = 0; k < N; ++k) m = fmaxf(m, p.get(k));
      r.rescale(m, c);
#pragma unroll
      for (int k = 0; k < N; ++k) r.s += __builtin_amdgcn_exp2f((p.get(k) - m) * c);
    }
    if (tid < rest) {
      const float v = span_value(x[full * N + tid]);
      r.rescale(fmaxf(r.m, v), c);
      r.s += __builtin_amdgcn_exp2f((v - r.m) * c);
    }
    r.rescale(wave_max(r.m), c);
    r.s = wave_sum(r.s);
    float label;
    if (WAVES > 1) {
      // (two buffers in turn: one barrier a row)
      float* lds = red[turn];
      turn ^= 1;
      if ((tid & 63) == 0) lds[tid >> 6] = r.m, lds[WAVES + (tid >> 6)] = r.s;
      if (tid == 0) lds[2 * WAVES] = span_value(x[id]);   // before any wave writes the row in place
      __syncthreads();
      label = lds[2 * WAVES];
      float m = lds[0];
#pragma unroll
      for (int k = 1; k < WAVES; ++k) m = fmaxf(m, lds[k]);
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < WAVES; ++k) s += lds[WAVES + k] * __builtin_amdgcn_exp2f((lds[k] - m) * c);
      r.m = m, r.s = s;
    } else {
      label = span_value(x[id]);
    }
    float logp, lse;
    const Terms o = row_terms<KIND>(a, t, w, label, r, &logp, &lse);
    if (tid == 0) {
      if (a.logp) a.logp[t] = logp;
      if (a.lse) a.lse[t] = lse;
#pragma unroll
      for (int k = 0; k < kSums; ++k) sum[k] += o.sum[k];
    }
    if (!GRAD) continue;
    const int at = (int)id;
    for (int i = tid; i < full; i += TH) {
      S p;
      p.template load<false>(x + i * N);
      float v[N];
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = __builtin_amdgcn_exp2f((p.get(k) - r.m) * c) * o.all;
      if ((unsigned)(at - i * N) < (unsigned)N) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += at - i * N == k ? o.label : 0.f;
      }
      S::template store<false>(d + i * N, v);
    }
    if (tid < rest) {
      const int i = full * N + tid;
      const float v = __builtin_amdgcn_exp2f((span_value(x[i]) - r.m) * c) * o.all;
      set_span_value(d + i, at == i ? v + o.label : v);
    }
  }
  if (KIND != LogitsArgs::LOGP && tid == 0) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) a.part[(int64_t)blockIdx.x * kSums + k] = sum[k];
  }
}

__global__ __launch_bounds__(256) void loss_sum_kernel(const double* part, int groups, int count, float* stats) {
  __shared__ double red[4];
  double s[kSums] = {0.0, 0.0, 0.0};
  for (int g = threadIdx.x; g < groups; g += 256) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) s[k] += part[(int64_t)g * kSums + k];
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    const double v = block_sum<4>(s[k], red);
    if (threadIdx.x == 0 && k < count) stats[k] = (float)v;
    __syncthreads();
  }
}

// Gradient from those of logp and lse: every value by itself, kChunk pieces of a row to a thread at a time.
constexpr int kChunk = 4;

struct BwdRows {
  const void *logits, *ids;
  void* dlogits;
  const float *dlogp, *dlse, *lse;
  int64_t T, ld, ld_out;
  int32_t V, chunks;
  float scale;
  bool ids_i64;
};

template <class E>
__global__ __launch_bounds__(256) void logp_bwd_kernel(const BwdRows a) {
  using S = Span<E>;
  constexpr int N = S::N;
  const int tid = threadIdx.x;
  const int full = a.V / N, rest = a.V - full * N;
  const int64_t items = a.T * a.chunks;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t t = item / a.chunks;
    const int chunk = (int)(item - t * a.chunks);
    const int64_t id = id_of(a.ids, a.ids_i64, t);
    const bool keep = id >= 0 && id < a.V;
    const E* x = (const E*)a.logits + t * a.ld;
    E* d = (E*)a.dlogits + t * a.ld_out;
    const int first = chunk * kChunk * 256 + tid;
    const bool tail = chunk == a.chunks - 1 && tid < rest;
    if (!keep) {
      const float zero[N] = {};
#pragma unroll
      for (int q = 0; q < kChunk; ++q)
        if (first + q * 256 < full) S::template store<false>(d + (first + q * 256) * N, zero);
      if (tail) set_span_value(d + full * N + tid, 0.f);
      continue;
    }
    const float g = a.dlogp[t], e = a.dlse ? a.dlse[t] : 0.f, lse = a.lse[t];
    const float at_label = a.scale * g, all = a.scale * (e - g);
    const int at = (int)id;
    S p[kChunk];
#pragma unroll
    for (int q = 0; q < kChunk; ++q)
      if (first + q * 256 < full) p[q].template load<false>(x + (first + q * 256) * N);
#pragma unroll
    for (int q = 0; q < kChunk; ++q) {
      const int i = first + q * 256;
      if (i >= full) break;
      float v[N];
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = __builtin_amdgcn_exp2f((p[q].get(k) * a.scale - lse) * kLog2E) * all;
      if ((unsigned)(at - i * N) < (unsigned)N) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += at - i * N == k ? at_label : 0.f;
      }
      S::template store<false>(d + i * N, v);
    }
    if (tail) {
      const int i = full * N + tid;
      const float v = __builtin_amdgcn_exp2f((span_value(x[i]) * a.scale - lse) * kLog2E) * all;
      set_span_value(d + i, at == i ? v + at_label : v);
    }
  }
}

// ---- host -----------------------------------------------------------------------------

int groups_of(int64_t T) { return (int)std::min<int64_t>(T, kGroups); }

template <int KIND, class E, int WAVES>
void launch_rows(const Rows& r, hipStream_t stream) {
  const dim3 grid((unsigned)groups_of(r.T)), block(WAVES * 64);
  if (r.dlogits)
    hipLaunchKernelGGL((rows_kernel<KIND, E, WAVES, true>), grid, block, 0, stream, r);
  else
    hipLaunchKernelGGL((rows_kernel<KIND, E, WAVES, false>), grid, block, 0, stream, r);
}
template <int KIND, class E>
void launch_rows(const Rows& r, hipStream_t stream) {
  if (r.V <= 2048 / (int)sizeof(E))
    launch_rows<KIND, E, 1>(r, stream);
  else
    launch_rows<KIND, E, 4>(r, stream);
}
template <int KIND>
hipError_t launch_rows(const Rows& r, bool f32, const char* tag, hipStream_t stream) {
  TimedLaunch tl(tag, stream);
  f32 ? launch_rows<KIND, float>(r, stream) : launch_rows<KIND, uint16_t>(r, stream);
  return hipGetLastError();
}

}  // namespace

size_t token_loss_workspace_bytes(int64_t T, int64_t V, bool f32) {
  (void)V, (void)f32;
  return (size_t)groups_of(T) * kSums * sizeof(double);
}

hipError_t run_token_loss(const LogitsArgs& a, hipStream_t stream) {
  Rows r{};
  r.logits = a.logits; r.ids = a.ids; r.dlogits = a.dlogits; r.weight = a.weight; r.advantage = a.advantage; r.old_logp = a.old_logp;
  r.ref_logp = a.ref_logp; r.logp = a.logp; r.lse = a.lse; r.part = (double*)a.ws; r.T = a.T; r.ld = a.ld; r.ld_out = a.ld_out;
  r.V = (int32_t)a.V; r.scale = a.scale; r.reduce = a.reduce; r.z_coef = a.z_coef; r.low = a.low; r.high = a.high; r.kl_coef = a.kl_coef;
  r.ids_i64 = a.ids_i64;
  if (a.T > 0) {
    const hipError_t e = a.kind == LogitsArgs::LOGP    ? launch_rows<LogitsArgs::LOGP>(r, a.f32, "token_logp", stream)
                         : a.kind == LogitsArgs::TOKEN ? launch_rows<LogitsArgs::TOKEN>(r, a.f32, "token_loss", stream)
                                                       : launch_rows<LogitsArgs::POLICY>(r, a.f32, "policy_loss", stream);
    if (e != hipSuccess || a.kind == LogitsArgs::LOGP) return e;
  }
  TimedLaunch tl("loss_sum", stream);
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(256), 0, stream, (const double*)a.ws, groups_of(a.T), a.kind == LogitsArgs::TOKEN ? 2 : 3,
                     a.stats);
  return hipGetLastError();
}

hipError_t run_token_logp_bwd(const LogitsArgs& a, hipStream_t stream) {
  BwdRows r{};
  r.logits = a.logits; r.ids = a.ids; r.dlogits = a.dlogits; r.dlogp = a.dlogp; r.dlse = a.dlse; r.lse = a.lse_in; r.T = a.T; r.ld = a.ld;
  r.ld_out = a.ld_out; r.V = (int32_t)a.V; r.scale = a.scale; r.ids_i64 = a.ids_i64;
  const int64_t per = (int64_t)kChunk * 256 * (a.f32 ? 4 : 8);
  r.chunks = (int32_t)((a.V + per - 1) / per);
  const unsigned grid = (unsigned)std::min<int64_t>(a.T * r.chunks, 1 << 16);
  TimedLaunch tl("token_logp_bwd", stream);
  if (a.f32)
    hipLaunchKernelGGL(logp_bwd_kernel<float>, dim3(grid), dim3(256), 0, stream, r);
  else
    hipLaunchKernelGGL(logp_bwd_kernel<uint16_t>, dim3(grid), dim3(256), 0, stream, r);
  return hipGetLastError();
}

}  // namespace elas
