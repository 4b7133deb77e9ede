// The loss of paired answers by their log-ratios, with its gradient (the formulas are in
// include/elas_loss.h).
//
// A pair's answers are summed in 64 bits by a team of 1, 2, 4 or 16 waves, then come its margin and loss, then the
// gradient, one value for each answer.  The pairs' losses are added up in a fixed order by a second launch.  2048
// pairs of 1000 tokens an answer: 10 us of kernel (49 MB) and 4 for the sum; 8 pairs of 100: 4.3 us, one launch; bound by
// latency below about a thousand pairs.
#include <math.h>

#include <algorithm>

#include "../../include/elas_loss.h"
#include "internal.h"
#include "spans.h"

namespace elas {

namespace {

constexpr int kGroups = 2048;
constexpr int kSums = 3;
// Up to so many pairs and values one workgroup does everything, a pair to a wave (in a graph, 20 pairs of 20 tokens: 5.4 us,
// 7.0 in two launches; 64 pairs of 100: 9.8 and 7.3).
constexpr int64_t kFewPairs = 32, kFewValues = 1 << 14;
// Values of a pair up to which a wave takes it, 2 waves, 4 waves (300 pairs of 600 values: 7.4 us either way; 2048 of 2000: 15.6 by
// one wave, 14.7 by 2, 16.8 by 4; 20000 of 100: 16 by one, 42 by 2; one pair of 40000: 9.8 by 16, 13.8 by 4).
constexpr int64_t kWavePair = 512, kTwoWavePair = 4096, kFourWavePair = 16384;

__device__ __forceinline__ int64_t offset_of(const PreferenceArgs& a, int64_t s) {
  const int64_t o = a.i64 ? ((const int64_t*)a.offsets)[s] : (int64_t)((const int32_t*)a.offsets)[s];
  return o < 0 ? 0 : o > a.N ? a.N : o;
}

// A thread's share of an answer's log-ratios: TH threads, 4 values to each at a time.
template <int TH, bool REF>
__device__ __forceinline__ double answer_sum(const PreferenceArgs& a, int64_t from, int64_t to, int tid) {
  double s = 0.0;
  int64_t i = from + 4 * tid;
#pragma unroll 1
  for (; i + 4 <= to; i += 4 * TH) {
    Four<float> x, y;
    x.template load<false>(a.logp + i);
    if (REF) y.template load<false>(a.ref + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) s += (double)x.get(k) - (REF ? (double)y.get(k) : 0.0);
  }
  if (i < to)
    for (int k = 0; k < 3; ++k)
      if (i + k < to) s += (double)a.logp[i + k] - (REF ? (double)a.ref[i + k] : 0.0);
  return s;
}

template <int TH>
__device__ __forceinline__ void fill(float* p, int64_t from, int64_t to, float v, int tid) {
  const float four[4] = {v, v, v, v};
  int64_t i = from + 4 * tid;
  for (; i + 4 <= to; i += 4 * TH) Four<float>::store<false>(p + i, four);
  if (i < to)
    for (int k = 0; k < 3; ++k)
      if (i + k < to) p[i + k] = v;
}

// Coefficients of the two series below, from the highest: read from memory into scalar registers each time,
// because as literals the compiler keeps all of them in vector registers through the loop over pairs (40, which
// halves the waves).
__constant__ const double kExpSeries[10] = {1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
__constant__ const double kAtanhSeries[10] = {1.0 / 19.0, 1.0 / 17.0, 1.0 / 15.0, 1.0 / 13.0, 1.0 / 11.0, 1.0 / 9.0, 1.0 / 7.0, 1.0 / 5.0, 1.0 / 3.0, 1.0};
template <int N>
__device__ __forceinline__ double series(const double (&c)[N], double x) {
  int first = 0;
  asm volatile("" : "+s"(first));
  double p = c[first];
#pragma unroll
  for (int k = 1; k < N; ++k) p = fma(p, x, c[first + k]);
  return p;
}

// exp(-x) for x >= 0 in 64 bits, to 1e-11 of itself: 2^-n times the series of the rest, which is under 0.347.
// (The library's are right to all 64 bits, with 4 times the instructions.)
__device__ __forceinline__ double exp_of_minus(double x) {
  const double y = fmin(x, 700.0), n = rint(y * 0x1.71547652b82fep0);
  return __builtin_amdgcn_ldexp(series(kExpSeries, fma(n, 0x1.62e42fefa39efp-1, -y)), -(int)n);
}
// ln(1 + e) for 0 <= e <= 1 to 1e-10 of itself: twice the inverse hyperbolic tangent of e / (2 + e), at most 1/3.
__device__ __forceinline__ double log_of_one_and(double e) {
  const double s = e / (2.0 + e);
  return 2.0 * s * series(kAtanhSeries, s * s);
}

// A pair's margin and loss from its answers' sums, and what each value of the chosen answer gets.
struct Pair {
  double z, loss;
  float g;
  __device__ __forceinline__ Pair(const PreferenceArgs& a, double chosen, double rejected) {
    z = (double)a.beta * (chosen - rejected);
    const double q = (double)a.smoothing;
    // ln(1 + exp(-|z|)), and sigmoid(z) and sigmoid(-z), without overflow, the smaller one not as 1 less the larger
    const double e = exp_of_minus(fabs(z)), soft = log_of_one_and(e);
    const double large = 1.0 / (1.0 + e), small = e * large, towards = z > 0.0 ? large : small, away = z > 0.0 ? small : large;
    // a weight of 0 takes no part, infinite as the other side may be
    loss = (q < 1.0 ? (1.0 - q) * (soft + fmax(-z, 0.0)) : 0.0) + (q > 0.0 ? q * (soft + fmax(z, 0.0)) : 0.0);
    g = (float)((q * towards - (1.0 - q) * away) * (double)a.beta / (double)a.pairs);
    if (z != z) loss = z, g = (float)z;
  }
};

// A workgroup takes `rounds` pairs to each of its TEAMS teams of WAVES waves at a time: their sums, then the
// margins and losses, a pair to a lane of the first wave (64-bit exponentials and logarithms are the longest part
// of a short answer), then the gradients.  LAST: the only workgroup, which adds up the statistics itself.
template <int WAVES, int TEAMS, bool LAST, bool REF>
__global__ __launch_bounds__(WAVES * TEAMS * 64) void preference_kernel(const PreferenceArgs a, int rounds) {
  constexpr int TH = WAVES * 64;
  static_assert(WAVES == 1 || TEAMS == 1, "a team is a wave or the workgroup");
  __shared__ double sums[2][64], red[2][WAVES];
  __shared__ int64_t offsets[129];
  __shared__ float gs[64];
  const int team = WAVES == 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0, tid = threadIdx.x % TH, lane = threadIdx.x & 63;
  const int at_once = rounds * TEAMS;      // 64 at most
  double loss = 0.0, won = 0.0, margin = 0.0;
  for (int64_t first = (int64_t)blockIdx.x * at_once; first < a.pairs; first += (int64_t)gridDim.x * at_once) {
    const int here = (int)(a.pairs - first < at_once ? a.pairs - first : at_once);
    for (int k = threadIdx.x; k <= 2 * here; k += TH * TEAMS) offsets[k] = offset_of(a, 2 * first + k);
    __syncthreads();
    for (int k = team; k < here; k += TEAMS) {
      const int64_t o0 = offsets[2 * k], o1 = offsets[2 * k + 1], o2 = offsets[2 * k + 2];
      double c = wave_sum(answer_sum<TH, REF>(a, o0, o1, tid)), d = wave_sum(answer_sum<TH, REF>(a, o1, o2, tid));
      if constexpr (WAVES > 1) {
        if (lane == 0) red[0][tid >> 6] = c, red[1][tid >> 6] = d;
        __syncthreads();
        c = red[0][0], d = red[1][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) c += red[0][w], d += red[1][w];
      }
      if (tid == 0) sums[0][k] = c, sums[1][k] = d;
    }
    __syncthreads();
    if (threadIdx.x < here) {
      const Pair p(a, sums[0][lane], sums[1][lane]);
      loss += p.loss;
      won += p.z > 0.0 ? 1.0 : 0.0;
      margin += p.z;
      gs[lane] = p.g;
      if (a.margin) a.margin[first + lane] = (float)p.z;
    }
    __syncthreads();
    if (a.dlogp)
      for (int k = team; k < here; k += TEAMS) {
        const float g = gs[k];
        fill<TH>(a.dlogp, offsets[2 * k], offsets[2 * k + 1], g, tid);
        fill<TH>(a.dlogp, offsets[2 * k + 1], offsets[2 * k + 2], -g, tid);
      }
    __syncthreads();
  }
  // what lies outside the sequences
  if (a.dlogp) {
    const int64_t first = a.pairs ? offset_of(a, 0) : 0, last = a.pairs ? offset_of(a, 2 * a.pairs) : 0;
    const int64_t at = (int64_t)blockIdx.x * (TH * TEAMS) + threadIdx.x, step = (int64_t)gridDim.x * (TH * TEAMS);
    for (int64_t i = at; i < first; i += step) a.dlogp[i] = 0.f;
    for (int64_t i = last + at; i < a.N; i += step) a.dlogp[i] = 0.f;
  }
  if (threadIdx.x < 64) {
    loss = wave_sum(loss), won = wave_sum(won), margin = wave_sum(margin);
    if (lane < kSums) {
      const double v = lane == 0 ? loss : lane == 1 ? won : margin;
      if (LAST)
        a.stats[lane] = a.pairs > 0 ? (float)(v / (double)a.pairs) : 0.f;
      else
        ((double*)a.ws)[(int64_t)blockIdx.x * kSums + lane] = v;
    }
  }
}

__global__ __launch_bounds__(1024) void preference_sum_kernel(const double* part, int groups, double pairs, float* stats) {
  __shared__ double red[16][kSums];
  double s[kSums] = {0.0, 0.0, 0.0};
  for (int g = threadIdx.x; g < groups; g += 1024) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) s[k] += part[(int64_t)g * kSums + k];
  }
  const double v = block_sums<16>(s, red);
  if (threadIdx.x < kSums) stats[threadIdx.x] = pairs > 0.0 ? (float)(v / pairs) : 0.f;
}

bool few(int64_t N, int64_t pairs) { return pairs <= kFewPairs && N <= kFewValues; }

}  // namespace

size_t preference_workspace_bytes(int64_t N, int64_t pairs) {
  return few(N, pairs) ? 0 : (size_t)std::max<int64_t>(1, std::min<int64_t>(pairs, kGroups)) * kSums * sizeof(double);
}

hipError_t run_preference(const PreferenceArgs& a, hipStream_t stream) {
  unsigned groups = 1;
  const auto launch = [&](auto with_ref, auto without, int threads, int64_t at_once, int teams) {
    TimedLaunch tl("preference", stream);
    groups = (unsigned)std::max<int64_t>(1, std::min<int64_t>((a.pairs + at_once - 1) / at_once, kGroups));
    hipLaunchKernelGGL(a.ref ? with_ref : without, dim3(groups), dim3((unsigned)threads), 0, stream, a, (int)(at_once / teams));
    return hipGetLastError();
  };
  // few short pairs: one workgroup, and no second launch
  if (few(a.N, a.pairs))
    return launch(preference_kernel<1, 16, true, true>, preference_kernel<1, 16, true, false>, 1024, kFewPairs, 16);
  const int64_t length = a.pairs ? a.N / a.pairs : 0;       // both answers
  const hipError_t e =
      length <= kWavePair
          // a pair to a wave, up to 16 a workgroup where that leaves enough workgroups
          ? launch(preference_kernel<1, 4, false, true>, preference_kernel<1, 4, false, false>, 256,
                   4 * std::max<int64_t>(1, std::min<int64_t>(a.pairs / 4096, 4)), 4)
      : length <= kTwoWavePair
          ? launch(preference_kernel<2, 1, false, true>, preference_kernel<2, 1, false, false>, 128, 1, 1)
      : length <= kFourWavePair || a.pairs > 512
          ? launch(preference_kernel<4, 1, false, true>, preference_kernel<4, 1, false, false>, 256, 1, 1)
          : launch(preference_kernel<16, 1, false, true>, preference_kernel<16, 1, false, false>, 1024, 1, 1);
  if (e != hipSuccess) return e;
  TimedLaunch tl("preference_sum", stream);
  hipLaunchKernelGGL(preference_sum_kernel, dim3(1), dim3(1024), 0, stream, (const double*)a.ws, (int)groups, (double)a.pairs, a.stats);
  return hipGetLastError();
}

}  // namespace elas
