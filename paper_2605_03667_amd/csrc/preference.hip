// The loss of paired answers by their log-ratios, with its gradient (the formulas are in
// include/elas_loss.h).
//
// A workgroup takes a pair at a time: the sums of both answers in 64 bits, z and the loss, then the
// gradient, one value for each answer.  The pairs' losses are added up in a fixed order by a
// second launch.
#include <math.h>

#include <algorithm>

#include "../../include/elas_loss.h"
#include "internal.h"
#include "spans.h"

namespace elas {

namespace {

constexpr int kGroups = 2048;
constexpr int kSums = 3;

__device__ __forceinline__ int64_t offset_of(const PreferenceArgs& a, int64_t s) {
  const int64_t o = a.i64 ? ((const int64_t*)a.offsets)[s] : (int64_t)((const int32_t*)a.offsets)[s];
  return o < 0 ? 0 : o > a.N ? a.N : o;
}

__device__ __forceinline__ double answer_sum(const PreferenceArgs& a, int64_t from, int64_t to) {
  double s = 0.0;
  for (int64_t i = from + threadIdx.x; i < to; i += 256) s += (double)a.logp[i] - (a.ref ? (double)a.ref[i] : 0.0);
  return s;
}

__device__ __forceinline__ void fill(float* p, int64_t from, int64_t to, float v) {
  for (int64_t i = from + threadIdx.x; i < to; i += 256) p[i] = v;
}

__global__ __launch_bounds__(256) void preference_kernel(const PreferenceArgs a) {
  __shared__ double red[2][4];
  double* part = (double*)a.ws;
  double sum[kSums] = {0.0, 0.0, 0.0};
  for (int64_t i = blockIdx.x; i < a.pairs; i += gridDim.x) {
    const int64_t o0 = offset_of(a, 2 * i), o1 = offset_of(a, 2 * i + 1), o2 = offset_of(a, 2 * i + 2);
    const double chosen = block_sum<4>(answer_sum(a, o0, o1), red[0]), rejected = block_sum<4>(answer_sum(a, o1, o2), red[1]);
    const double z = (double)a.beta * (chosen - rejected), q = (double)a.smoothing;
    // ln(1 + exp(-|z|)), and sigmoid(-z), without overflow
    const double e = exp(-fabs(z)), soft = log1p(e);
    const double away = (z > 0.0 ? e : 1.0) / (1.0 + e);
    // a weight of 0 takes no part, infinite as the other side may be
    sum[0] += (q < 1.0 ? (1.0 - q) * (soft + fmax(-z, 0.0)) : 0.0) + (q > 0.0 ? q * (soft + fmax(z, 0.0)) : 0.0);
    sum[1] += z > 0.0 ? 1.0 : 0.0;
    sum[2] += z;
    if (threadIdx.x == 0 && a.margin) a.margin[i] = (float)z;
    if (a.dlogp) {
      const float g = (float)((q - away) * (double)a.beta / (double)a.pairs);
      fill(a.dlogp, o0, o1, z != z ? (float)z : g);
      fill(a.dlogp, o1, o2, z != z ? (float)z : -g);
    }
  }
  // what lies outside the sequences
  if (a.dlogp) {
    const int64_t first = a.pairs ? offset_of(a, 0) : 0, last = a.pairs ? offset_of(a, 2 * a.pairs) : 0;
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < first; i += step) a.dlogp[i] = 0.f;
    for (int64_t i = last + (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.N; i += step) a.dlogp[i] = 0.f;
  }
  if (threadIdx.x == 0) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) part[(int64_t)blockIdx.x * kSums + k] = sum[k];
  }
}

__global__ __launch_bounds__(256) void preference_sum_kernel(const double* part, int groups, double pairs, float* stats) {
  __shared__ double red[4];
  double s[kSums] = {0.0, 0.0, 0.0};
  for (int g = threadIdx.x; g < groups; g += 256) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) s[k] += part[(int64_t)g * kSums + k];
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    const double v = block_sum<4>(s[k], red);
    if (threadIdx.x == 0) stats[k] = pairs > 0.0 ? (float)(v / pairs) : 0.f;
    __syncthreads();
  }
}

int groups_of(int64_t pairs) { return (int)std::max<int64_t>(1, std::min<int64_t>(pairs, kGroups)); }

}  // namespace

size_t preference_workspace_bytes(int64_t pairs) { return (size_t)groups_of(pairs) * kSums * sizeof(double); }

hipError_t run_preference(const PreferenceArgs& a, hipStream_t stream) {
  const int groups = groups_of(a.pairs);
  {
    TimedLaunch tl("preference", stream);
    hipLaunchKernelGGL(preference_kernel, dim3((unsigned)groups), dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  TimedLaunch tl("preference_sum", stream);
  hipLaunchKernelGGL(preference_sum_kernel, dim3(1), dim3(256), 0, stream, (const double*)a.ws, groups, (double)a.pairs, a.stats);
  return hipGetLastError();
}

}  // namespace elas
