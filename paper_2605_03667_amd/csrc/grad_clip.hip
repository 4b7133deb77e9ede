// Global norm of the gradients over many tensors, and their clipping (the formulas
// are in include/elas_train.h).
//
// Two launches for up to kTensors tensors: the squares, as one 64-bit partial sum
// per workgroup, and the scaling, in which every workgroup adds up the partial sums
// for itself (16 KB from L2) instead of waiting for a launch that does it once.
// Tensors are cut into pieces of kPiece values; the pieces of all tensors of a
// launch are numbered through and dealt out to the workgroups in turn, so that one
// long tensor and a hundred short ones load the card alike.  Bound by HBM: one read for
// the norm, one read and one write for the scaling.  The scaling takes the pieces in
// the opposite order, so that it begins with what the caches still hold (985 MB: 570 us,
// in the same order 578: measured before the last part was kept, below).  985 MB in 193
// tensors: 490 us, 6.0 TB/s over the three; 15.5 MB in 49 tensors: 5.7 + 9.1 us of kernels, 24 us
// a call (the tensors' addresses, lengths, types and layouts are read in every one); the norm
// alone of 985 MB 156 us (6.3 TB/s).
#include <math.h>

#include <algorithm>

#include "../../include/elas_train.h"
#include "internal.h"
#include "rows.h"

namespace elas {

namespace {

constexpr int kTensors = 128;     // per launch, at most
constexpr int kPiece = 8192;      // values
constexpr int kGroups = 2048;     // most workgroups, and partial sums, per launch
// The squares are read past the caches, except, where there is more than the last-level
// cache holds, for the last part, which the scaling takes first (1B: all kept 516 us, none
// 512, 64 MB 502, 128 MB 491, 192 MB 498; 152 MB in all: kept 86, not 77).
constexpr int64_t kCache = int64_t(256) << 20, kKeep = int64_t(128) << 20;

// The tensors of a launch, as a kernel argument of room for CAP: what a launch costs the
// host grows by 0.7 us for each KB of it.
template <int CAP>
struct Tensors {
  const void* in[CAP];
  uint32_t first[CAP + 1];   // number of each tensor's first piece; [count] = pieces in all
  uint32_t bf16[CAP / 32];   // bit k: tensor k is bf16
  uint16_t last[CAP];        // values of its last piece
  int count;
  __device__ __forceinline__ bool is_bf16(int k) const { return bf16[k >> 5] >> (k & 31) & 1u; }
  // values of piece c, which is tensor k's
  __device__ __forceinline__ int values(uint32_t c, int k) const { return c + 1 < first[k + 1] ? kPiece : (int)last[k]; }
};
template <int CAP>
struct Outputs {
  void* out[CAP];
};

// Tensors need their element's alignment only: 16-byte accesses at any such address.  (As a
// template argument these types would lose their alignment, so every access names its type.)
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

__device__ __forceinline__ float value_of(float e) { return e; }
__device__ __forceinline__ float value_of(uint16_t e) { return as_float((uint32_t)e << 16); }
__device__ __forceinline__ void set_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void set_value(uint16_t* p, float v) { *p = (uint16_t)bf16x2_rne(v, 0.f); }

// A thread's values of a piece: PARTS parts of 16 bytes, part k of all threads contiguous.
template <class E>
struct Part {
  static constexpr int N = 16 / sizeof(E), PARTS = kPiece / 256 / N;
  static __device__ __forceinline__ int first(int k) { return (k * 256 + (int)threadIdx.x) * N; }
  template <bool STREAM>
  static __device__ __forceinline__ void load(const E* p, float (&v)[N]) {
    if constexpr (N == 4) {
      const f32x4 q = STREAM ? __builtin_nontemporal_load((const f32x4_any*)p) : *(const f32x4_any*)p;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = q[i];
    } else {
      const u32x4 q = STREAM ? __builtin_nontemporal_load((const u32x4_any*)p) : *(const u32x4_any*)p;
      unpack8(make_uint4(q[0], q[1], q[2], q[3]), v);
    }
  }
  static __device__ __forceinline__ void store(E* p, const float (&v)[N]) {
    if constexpr (N == 4)
      __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, (f32x4_any*)p);
    else
      __builtin_nontemporal_store(u32x4{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3]), bf16x2_rne(v[4], v[5]), bf16x2_rne(v[6], v[7])},
                                  (u32x4_any*)p);
  }
};

// Squares are taken in 64 bits: exact for every float, and no sum of them overflows.
// (A piece that the tensor's end cuts: the part that it cuts is taken value by value.)
template <bool STREAM, class E>
__device__ __forceinline__ void square_piece(const E* g, int n, double (&s)[2]) {
  using P = Part<E>;
  auto add = [&](const float (&v)[P::N]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < P::N; ++i) s[i & 1] = fma((double)v[i], (double)v[i], s[i & 1]);
  };
  if (n == kPiece) {
    float v[P::PARTS][P::N];
#pragma unroll
    for (int k = 0; k < P::PARTS; ++k) P::template load<STREAM>(g + P::first(k), v[k]);
#pragma unroll
    for (int k = 0; k < P::PARTS; ++k) add(v[k]);
    return;
  }
#pragma unroll 4
  for (int at = P::first(0); at + P::N <= n; at += 256 * P::N) {
    float v[P::N];
    P::template load<STREAM>(g + at, v);
    add(v);
  }
  const int i = n / P::N * P::N + (int)threadIdx.x;
  if (i < n) {
    const double x = value_of(g[i]);
    s[0] = fma(x, x, s[0]);
  }
}

// A factor as the product of a normal float32 and a power of two, 1 where it is normal itself:
// below 2^-126 a float32 has fewer bits, and none at all for a norm of values near 2^128.
struct Factor {
  float f, power;
  __device__ __forceinline__ explicit Factor(double v) {
    power = v < 0x1p-126 ? 0x1p-126f : 1.f;
    f = (float)(v / (double)power);
  }
  __device__ __forceinline__ float operator()(float v) const { return v * f * power; }
};

template <class E>
__device__ __forceinline__ void scale_piece(const E* g, E* out, int n, const Factor& f) {
  using P = Part<E>;
  auto scaled = [&](int at, float (&v)[P::N]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < P::N; ++i) v[i] = f(v[i]);
    P::store(out + at, v);
  };
  if (n == kPiece) {
    float v[P::PARTS][P::N];
#pragma unroll
    for (int k = 0; k < P::PARTS; ++k) P::template load<true>(g + P::first(k), v[k]);
#pragma unroll
    for (int k = 0; k < P::PARTS; ++k) scaled(P::first(k), v[k]);
    return;
  }
  for (int at = P::first(0); at + P::N <= n; at += 256 * P::N) {
    float v[P::N];
    P::template load<true>(g + at, v);
    scaled(at, v);
  }
  const int i = n / P::N * P::N + (int)threadIdx.x;
  if (i < n) set_value(out + i, f(value_of(g[i])));
}

// Which tensor a piece belongs to: the last one whose first piece is not behind it.
// Lane l holds the first pieces of the tensors l and l + 64.
template <int CAP>
struct Finder {
  uint32_t f0, f1 = ~0u;
  __device__ __forceinline__ explicit Finder(const Tensors<CAP>& g) {
    const int lane = threadIdx.x & 63;
    f0 = lane < g.count ? g.first[lane] : ~0u;
    if (CAP > 64) f1 = lane + 64 < g.count ? g.first[lane + 64] : ~0u;
  }
  __device__ __forceinline__ int operator()(uint32_t piece) const {
    return __popcll(__ballot(f0 <= piece)) + (CAP > 64 ? __popcll(__ballot(f1 <= piece)) : 0) - 1;
  }
};

template <int CAP>
__global__ __launch_bounds__(256) void grad_square_kernel(const Tensors<CAP> g, uint32_t keep, double* part) {
  __shared__ double red[4];
  const Finder<CAP> find(g);
  const uint32_t pieces = g.first[g.count];
  double s[2] = {0.0, 0.0};
  for (uint32_t c = blockIdx.x; c < pieces; c += gridDim.x) {
    const int k = find(c);
    const int64_t at = (int64_t)(c - g.first[k]) * kPiece;
    const int n = g.values(c, k);
    // the last `keep` pieces are left in the caches
    if (g.is_bf16(k)) {
      const uint16_t* p = (const uint16_t*)g.in[k] + at;
      c + keep < pieces ? square_piece<true>(p, n, s) : square_piece<false>(p, n, s);
    } else {
      const float* p = (const float*)g.in[k] + at;
      c + keep < pieces ? square_piece<true>(p, n, s) : square_piece<false>(p, n, s);
    }
  }
  const double sum = block_sum<4>(s[0] + s[1], red);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// Norm from the partial sums, in the same order in every workgroup; 8 loads of a thread
// on their way at once.
__device__ __forceinline__ double norm_of(const double* part, int64_t parts, double* red) {
  double s = 0.0;
  for (int64_t i0 = threadIdx.x; i0 < parts; i0 += kGroups) {
    double v[kGroups / 256];
#pragma unroll
    for (int k = 0; k < kGroups / 256; ++k) v[k] = i0 + k * 256 < parts ? part[i0 + k * 256] : 0.0;
#pragma unroll
    for (int k = 0; k < kGroups / 256; ++k) s += v[k];
  }
  return sqrt(block_sum<4>(s, red));
}

__global__ __launch_bounds__(256) void grad_norm_kernel(const double* part, int64_t parts, float* norm) {
  __shared__ double red[4];
  const double v = norm_of(part, parts, red);
  if (threadIdx.x == 0) norm[0] = (float)v;
}

// stats NULL: another launch writes them.
template <int CAP>
__global__ __launch_bounds__(256) void grad_scale_kernel(const Tensors<CAP> g, const Outputs<CAP> o, const double* part, int64_t parts, float max_norm, float* stats) {
  __shared__ double red[4];
  const Finder<CAP> find(g);
  const double norm = norm_of(part, parts, red);
  const bool finite = norm < (double)INFINITY, clips = finite && norm > (double)max_norm;
  const double factor = clips ? (double)max_norm / norm : 1.0;
  const Factor scale(factor);
  if (stats && blockIdx.x == 0 && threadIdx.x == 0) {
    stats[0] = (float)norm;
    stats[1] = finite ? (float)factor : 0.f;
  }
  const uint32_t pieces = g.first[g.count];
  for (uint32_t i = blockIdx.x; i < pieces; i += gridDim.x) {
    const uint32_t c = pieces - 1 - i;
    const int k = find(c);
    if (!clips && g.in[k] == o.out[k]) continue;
    const int64_t at = (int64_t)(c - g.first[k]) * kPiece;
    const int n = g.values(c, k);
    if (g.is_bf16(k))
      scale_piece((const uint16_t*)g.in[k] + at, (uint16_t*)o.out[k] + at, n, scale);
    else
      scale_piece((const float*)g.in[k] + at, (float*)o.out[k] + at, n, scale);
  }
}

// ---- host -----------------------------------------------------------------------------

struct GradCall {
  const void* const* in;
  void* const* out;
  const int64_t* numel;
  const int32_t* dtype;
  int64_t n;
  float max_norm;
  float* stats;
  double* part;
  hipStream_t stream;
};

// The tensors k0 .. of one launch (empty ones take no piece).
template <int CAP>
void fill(Tensors<CAP>& g, const GradCall& c, int64_t k0, int count) {
  g.count = count;
  uint32_t pieces = 0;
  for (int k = 0; k < CAP / 32; ++k) g.bf16[k] = 0;
  for (int k = 0; k < count; ++k) {
    const int64_t n = c.numel[k0 + k], of = (n + kPiece - 1) / kPiece;
    g.in[k] = c.in[k0 + k];
    g.first[k] = pieces;
    g.last[k] = (uint16_t)(n - (of - 1) * kPiece);
    pieces += (uint32_t)of;
    if (c.dtype[k0 + k] == ELAS_GRAD_BF16) g.bf16[k >> 5] |= 1u << (k & 31);
  }
  g.first[count] = pieces;
}

// Pieces at the end of the launch that make up the last `bytes` of it.
template <int CAP>
uint32_t last_pieces(const Tensors<CAP>& g, int64_t bytes) {
  uint32_t pieces = 0;
  for (int k = g.count - 1; k >= 0 && bytes > 0; --k) {
    const int64_t piece = kPiece * ((g.bf16[k >> 5] >> (k & 31) & 1u) ? 2 : 4), all = g.first[k + 1] - g.first[k];
    const int64_t some = std::min(all, bytes / piece);
    pieces += (uint32_t)some;
    bytes = some < all ? 0 : bytes - some * piece;
  }
  return pieces;
}

// One launch over the tensors k0 .. k0 + count; adds its partial sums to `parts`.
template <int CAP>
hipError_t launch_square(const GradCall& c, int64_t k0, int count, int64_t keep, int64_t& parts) {
  Tensors<CAP> g;
  fill(g, c, k0, count);
  const unsigned groups = std::min<uint32_t>(g.first[count], kGroups);
  if (groups == 0) return hipSuccess;
  TimedLaunch tl("grad_square", c.stream);
  hipLaunchKernelGGL(grad_square_kernel<CAP>, dim3(groups), dim3(256), 0, c.stream, g, last_pieces(g, keep), c.part + parts);
  parts += groups;
  return hipGetLastError();
}
template <int CAP>
hipError_t launch_scale(const GradCall& c, int64_t k0, int count, int64_t parts) {
  Tensors<CAP> g;
  fill(g, c, k0, count);
  Outputs<CAP> o;
  for (int k = 0; k < count; ++k) o.out[k] = c.out[k0 + k];
  TimedLaunch tl("grad_scale", c.stream);
  hipLaunchKernelGGL(grad_scale_kernel<CAP>, dim3(std::max(1u, std::min<uint32_t>(g.first[count], kGroups))), dim3(256), 0, c.stream, g, o,
                     (const double*)c.part, parts, c.max_norm, k0 == 0 ? c.stats : nullptr);
  return hipGetLastError();
}

int64_t launches(int64_t n) { return (n + kTensors - 1) / kTensors; }

}  // namespace

size_t grad_workspace_bytes(int64_t n) { return (size_t)launches(n) * kGroups * sizeof(double); }

hipError_t run_grad_norm(const void* const* grads, void* const* out, const int64_t* numel, const int32_t* dtype, int64_t n, bool clip,
                         float max_norm, float* stats, void* ws, hipStream_t stream) {
  const GradCall c{grads, out, numel, dtype, n, max_norm, stats, (double*)ws, stream};
  int64_t parts = 0, total = 0;
  for (int64_t k = 0; k < n; ++k) total += numel[k] * (dtype[k] == ELAS_GRAD_BF16 ? 2 : 4);
  for (int64_t k = 0; k < n; k += kTensors) {
    const int count = (int)std::min<int64_t>(kTensors, n - k);
    // (a launch other than the last one leaves nothing in the caches)
    const int64_t keep = clip && total > kCache && k + kTensors >= n ? kKeep : 0;
    const hipError_t e = count <= 32   ? launch_square<32>(c, k, count, keep, parts)
                         : count <= 64 ? launch_square<64>(c, k, count, keep, parts)
                                       : launch_square<kTensors>(c, k, count, keep, parts);
    if (e != hipSuccess) return e;
  }
  if (!clip) {
    TimedLaunch tl("grad_norm", stream);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, stream, (const double*)c.part, parts, stats);
    return hipGetLastError();
  }
  // (one launch at least, which writes the statistics where there are no values)
  for (int64_t l = std::max<int64_t>(launches(n), 1) - 1; l >= 0; --l) {
    const int64_t k = l * kTensors;
    const int count = (int)std::min<int64_t>(kTensors, n - k);
    const hipError_t e = count <= 32   ? launch_scale<32>(c, k, count, parts)
                         : count <= 64 ? launch_scale<64>(c, k, count, parts)
                                       : launch_scale<kTensors>(c, k, count, parts);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace elas
