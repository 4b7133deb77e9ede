// Norms before and after a block, fused with its gate and residual scale
// (forward and backward; the formulas are in include/elas_train.h).
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace elas {

namespace {

// ---- rows of up to 512 W NV features, W waves to a row -----------------------------
// The row stays in registers, NV times 8 features to a lane: every operand is read once
// and every output written once, the row's means need no second pass, and what bounds
// the kernels is HBM.  Forward: two sums over the row (of b^2, then of h'^2) and one
// pass.  Backward: the three sums that need no other (of h'^2, q h' and b^2) together,
// then that of p bh; the statistics are computed anew rather than kept by the forward,
// as the row is at hand and its gradient is then that of the formula at the stored h'.
// The sums over the tokens stay in registers over all rows of a workgroup; a second,
// small launch adds up the workgroups' rows of them in a fixed order.
//
// W waves to a row rather than more pieces to a lane (NV = 1 up to 4096 features), for the
// registers: the backward has 115 of them with one piece, 165 with two.  (1B backward, 65536
// tokens, bf16: W = 4, NV = 1 285 us; W = 2, NV = 2 with 768 workgroups, of which 512 fit at
// once, 275, with 512 291; other widths and the float32 stream were not measured so.)  For the
// same reason pieces stay packed between their uses (without that 135 and 246 registers, and
// spills at W = 8; 1B 285 us either way) and gains are read once per workgroup.
//
// Measured, bytes that the call cannot do without over the call's time: forward 1B, 65536
// tokens, float32 stream 265 us (6.1 TB/s; a copy of 1 GiB reaches 5.5); 350M, 2000 tokens
// 6.2 us of kernel; 1B, 16 tokens 3.7.  Backward 1B, 65536 tokens 290 us (5.6 TB/s; kernels 281
// + 5); 350M, 16381 tokens, gate per token, float32 stream 67 us (5.5); 60M, 2048 tokens
// 5.0 + 3.4 us of kernels.

// Where a thread's row and pieces lie; loads and stores of piece v.
template <int W, int NV, bool SPLIT>
struct RowLanes {
  static constexpr int WAVES = W < 4 ? 4 : W;   // of a workgroup
  static constexpr int ROWS = WAVES / W;        // rows it works on at a time
  int slot;
  uint32_t c[NV];   // (unsigned: an offset beside a uniform address)
  bool there[NV], there2[NV];
  __device__ __forceinline__ explicit RowLanes(int d) {
    slot = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W));   // (the same in all of a wave)
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      c[v] = (v * W + threadIdx.x / 64 % W) * 512 + threadIdx.x % 64 * (SPLIT ? 4 : 8);
      there[v] = c[v] < (uint32_t)d;
      there2[v] = SPLIT ? c[v] + 256 < (uint32_t)d : there[v];
    }
  }
  template <bool STREAM = false, class T>
  __device__ __forceinline__ void load(Piece<T, SPLIT>& x, const T* row, int v, bool live) const {
    x.template load<STREAM>(row + c[v], live && there[v], live && there2[v]);
  }
  template <bool STREAM = false, class T>
  __device__ __forceinline__ void store(T* row, const float (&x)[8], int v, bool live) const {
    Piece<T, SPLIT>::template store<STREAM>(row + c[v], x, live && there[v], live && there2[v]);
  }
};

// Sums of N values over a row's W waves.  `red` is free again after the next call
// with another `red`.
template <int W, int WAVES, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float (&red)[WAVES][N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
  if constexpr (W > 1) {
    const int wave = threadIdx.x >> 6, w0 = wave / W * W;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) red[wave][i] = s[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[i] = red[w0][i];
#pragma unroll
      for (int w = 1; w < W; ++w) s[i] += red[w0 + w][i];
    }
  }
}

template <class R, int W, int NV, bool STREAM>
__global__ __launch_bounds__(64 * (W < 4 ? 4 : W)) void join_fwd_kernel(const NormJoinArgs a) {
  constexpr bool SPLIT = sizeof(R) == 4;
  using Lanes = RowLanes<W, NV, SPLIT>;
  __shared__ float red[2][Lanes::WAVES][1];
  const Lanes l((int)a.d);
  const float inv_d = 1.f / (float)a.d;
  for (int64_t t0 = (int64_t)blockIdx.x * Lanes::ROWS; t0 < a.T; t0 += (int64_t)gridDim.x * Lanes::ROWS) {
    const int64_t t = t0 + l.slot, at = t * a.d;
    if (W == 1 && t >= a.T) break;
    const bool live = t < a.T;
    Piece<R, SPLIT> h[NV];
    Piece<uint16_t, SPLIT> b[NV], gate[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      l.load(h[v], (const R*)a.h + at, v, live);
      if (a.b) l.load(b[v], a.b + at, v, live);
      if (a.gate) l.load(gate[v], a.gate + (a.gate_token ? at : 0), v, live);
    }
    float x[NV][8];
    if (a.b) {
      float rho = 1.f;
      if (a.w_post) {
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          float u[8];
          b[v].get(u);
#pragma unroll
          for (int i = 0; i < 8; ++i) s[0] = fmaf(u[i], u[i], s[0]);
        }
        row_sums<W>(s, red[0]);
        rho = 1.f / sqrtf(s[0] * inv_d + a.eps);
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float u[8], k[8];
        b[v].get(u);
        if (a.w_post) {
          Piece<uint16_t, SPLIT> w;
          l.load(w, a.w_post, v, true);
          w.get(k);
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = u[i] * rho * k[i];
        }
        if (a.gate) {
          gate[v].get(k);
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] *= k[i];
        }
        h[v].get(x[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[v][i] = fmaf(a.res_scale, x[v][i], a.block_scale * u[i]);
        l.template store<STREAM>((R*)a.h_out + at, x[v], v, live);
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v) h[v].get(x[v]);
    }
    if (a.w_pre) {
      float s[1] = {0.f};
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fmaf(x[v][i], x[v][i], s[0]);
      row_sums<W>(s, red[1]);
      const float sig = 1.f / sqrtf(s[0] * inv_d + a.eps);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float k[8];
        Piece<uint16_t, SPLIT> w;
        l.load(w, a.w_pre, v, true);
        w.get(k);
#pragma unroll
        for (int i = 0; i < 8; ++i) k[i] *= x[v][i] * sig;
        l.template store<STREAM>(a.n + at, k, v, live);
      }
    }
    // (a lone second or first sum would leave `red` in use)
    if (W > 1 && !(a.w_pre && a.w_post)) __syncthreads();
  }
}

// The sums over the tokens: acc[0] of dn xh, acc[1] of G bh (times the token's
// gate where there is one for each), added up in the workgroup at the end and
// written to row blockIdx.x of `part`, [grid][2][d].  Held to the registers that leave
// a SIMD the waves that the grid has for it: 3, or 4 of workgroups of 8 (NV = 1; where it has
// 3, at 128 registers, for 4, no faster), else 2.
template <class R, int W, int NV, bool STREAM>
__global__ __launch_bounds__(64 * (W < 4 ? 4 : W), NV > 1 ? 2 : W == 8 ? 4 : 3) void join_bwd_kernel(const NormJoinArgs a, float* part) {
  constexpr bool SPLIT = sizeof(R) == 4;
  using Lanes = RowLanes<W, NV, SPLIT>;
  __shared__ float red3[Lanes::WAVES][3], red1[Lanes::WAVES][1];
  const Lanes l((int)a.d);
  const float inv_d = 1.f / (float)a.d;
  float acc[2][NV][8] = {};
  Piece<uint16_t, SPLIT> w_pre[NV], w_post[NV], shared[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if (a.w_pre) l.load(w_pre[v], a.w_pre, v, true);
    if (a.w_post) l.load(w_post[v], a.w_post, v, true);
    if (a.gate && !a.gate_token) l.load(shared[v], a.gate, v, true);
  }
  for (int64_t t0 = (int64_t)blockIdx.x * Lanes::ROWS; t0 < a.T; t0 += (int64_t)gridDim.x * Lanes::ROWS) {
    const int64_t t = t0 + l.slot, at = t * a.d;
    if (W == 1 && t >= a.T) break;
    const bool live = t < a.T;   // (rows past the end are zeros, with factors 0: they add nothing)
    Piece<R, SPLIT> h[NV], dho[NV];
    Piece<uint16_t, SPLIT> dn[NV], b[NV], gate[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (a.w_pre) {
        l.template load<STREAM>(h[v], (const R*)a.h + at, v, live);
        l.template load<STREAM>(dn[v], a.dn + at, v, live);
      }
      if (a.b) l.template load<STREAM>(b[v], a.b + at, v, live);
      if (a.dh_out) l.template load<STREAM>(dho[v], (const R*)a.dh_out + at, v, live);
      if (a.gate_token) l.template load<STREAM>(gate[v], a.gate + at, v, live);
    }
    float s[3] = {0.f, 0.f, 0.f};   // |h'|^2, q h', |b|^2
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      w_pre[v].keep_packed(), w_post[v].keep_packed(), shared[v].keep_packed();
      float x[8], q[8], k[8];
      if (a.w_pre) {
        h[v].get(x), dn[v].get(q), w_pre[v].get(k);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[0] = fmaf(x[i], x[i], s[0]);
          s[1] = fmaf(q[i] * k[i], x[i], s[1]);
        }
      }
      if (a.w_post) {
        b[v].get(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[2] = fmaf(x[i], x[i], s[2]);
      }
    }
    if (a.w_pre || a.w_post) row_sums<W>(s, red3);
    const float sig = live ? 1.f / sqrtf(s[0] * inv_d + a.eps) : 0.f;
    const float rho = a.w_post ? (live ? 1.f / sqrtf(s[2] * inv_d + a.eps) : 0.f) : 1.f;
    const float ch = s[1] * sig * inv_d;   // mean of q xh
    float g[NV][8], pb[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      h[v].keep_packed(), dn[v].keep_packed(), b[v].keep_packed();
      w_pre[v].keep_packed();
      float x[8], q[8], k[8];
      if (a.dh_out)
        dho[v].get(g[v]);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) g[v][i] = 0.f;
      if (a.w_pre) {
        h[v].get(x), dn[v].get(q), w_pre[v].get(k);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float xh = x[i] * sig;
          acc[0][v][i] = fmaf(q[i], xh, acc[0][v][i]);
          g[v][i] = fmaf(sig, fmaf(-ch, xh, q[i] * k[i]), g[v][i]);
        }
      }
      if (a.dh) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = a.res_scale * g[v][i];
        l.template store<true>((R*)a.dh + at, q, v, live);
      }
      if (!a.b) continue;
      b[v].get(x);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= rho;
      if (a.w_post) w_post[v].get(k);
      if (a.gate_token) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = a.block_scale * g[v][i] * (a.w_post ? x[i] * k[i] : x[i]);
        l.template store<true>((uint16_t*)a.dgate + at, q, v, live);
        gate[v].get(q);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[v][i] *= q[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[1][v][i] = fmaf(g[v][i], x[i], acc[1][v][i]);
      if (a.gate && !a.gate_token) {
        shared[v].get(q);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[v][i] *= q[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) g[v][i] *= a.block_scale;
      if (a.w_post) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          g[v][i] *= k[i];
          pb[0] = fmaf(g[v][i], x[i], pb[0]);
        }
      }
    }
    if (a.b) {
      if (a.w_post) {
        row_sums<W>(pb, red1);
        const float cb = pb[0] * inv_d;   // mean of p bh
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          float x[8];
          b[v].keep_packed();
          b[v].get(x);
#pragma unroll
          for (int i = 0; i < 8; ++i) g[v][i] = rho * fmaf(-cb, x[i] * rho, g[v][i]);
        }
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) l.template store<true>(a.db + at, g[v], v, live);
    }
    // (without a second sum red3 would still be in use)
    if (W > 1 && !a.w_post) __syncthreads();
  }
  if (!part) return;
  // rows of a workgroup are added in order, in shared memory
  const bool need[2] = {a.dw_pre != nullptr, a.dw_post || (a.dgate && !a.gate_token)};
  extern __shared__ __attribute__((aligned(16))) float sum[];   // [2][d]
#pragma unroll
  for (int r = 0; r < Lanes::ROWS; ++r) {
    if (l.slot == r) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int v = 0; v < NV; ++v)
          if (need[k]) {
            float* out = (r + 1 == Lanes::ROWS ? part + (int64_t)blockIdx.x * 2 * a.d : sum) + k * a.d;
            if (r > 0) {
              Piece<float, SPLIT> before;
              float x[8];
              l.load(before, (const float*)sum + k * a.d, v, true);
              before.get(x);
#pragma unroll
              for (int i = 0; i < 8; ++i) acc[k][v][i] = x[i] + acc[k][v][i];
            }
            l.store(out, acc[k][v], v, true);
          }
    }
    if (r + 1 < Lanes::ROWS) __syncthreads();
  }
}

// The gradients from the sums `part` [rows][2][d] (with A the second one):
// dw_pre = sum dn xh, dgate = block_scale w_post A, dw_post = block_scale gate A.
// A workgroup takes 32 columns: 8 threads of 4 columns times 32 shares of the rows.
// Columns begin at c0 (d where the first sum is not needed).
__global__ __launch_bounds__(256) void join_reduce_kernel(const NormJoinArgs a, const float* part, int rows, int64_t c0, int64_t c1) {
  __shared__ float4 red[32][8];
  const int64_t d = a.d, c = c0 + (int64_t)blockIdx.x * 32 + threadIdx.x % 8 * 4;
  const int share = threadIdx.x / 8, r1 = (int)((int64_t)rows * (share + 1) / 32);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < c1) {
#pragma unroll 8
    for (int r = (int)((int64_t)rows * share / 32); r < r1; ++r) {
      const float4 x = *(const float4*)(part + r * 2 * d + c);
      s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
    }
  }
  red[share][threadIdx.x % 8] = s;
  __syncthreads();
  const int64_t col = c0 + (int64_t)blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x >= 32 || col >= c1) return;
  float v = 0.f;
#pragma unroll
  for (int k = 0; k < 32; ++k) v += ((const float*)red[k])[threadIdx.x];
  if (col < d) {
    a.dw_pre[col] = v;
    return;
  }
  auto factor = [&](const uint16_t* p) { return p ? as_float((uint32_t)p[col - d] << 16) : 1.f; };
  v *= a.block_scale;
  if (a.dgate && !a.gate_token) ((float*)a.dgate)[col - d] = v * factor(a.w_post);
  if (a.dw_post) a.dw_post[col - d] = v * (a.gate_token ? 1.f : factor(a.gate));
}

// ---- wider rows -------------------------------------------------------------------
// One workgroup per row; the row is read again (from L2) where a sum over it is needed
// first (16384 features, 8192 rows, bf16: 304 us forward, 811 backward).

// 8 features of the operands at column c of row t (absent: zeros, or ones for factors).
template <class R>
struct WideRow {
  const NormJoinArgs& a;
  int64_t at;
  __device__ __forceinline__ void factor(const uint16_t* p, int64_t i, float (&v)[8]) const {
    if (p) return load8(p + i, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 1.f;
  }
  // the forward's u before the gate, or h' where there is no block
  __device__ __forceinline__ void joined(int64_t c, float rho, float (&x)[8]) const {
    load8((const R*)a.h + at + c, x);
    if (!a.b) return;
    float u[8], w[8], k[8];
    load8(a.b + at + c, u);
    factor(a.w_post, c, w);
    factor(a.gate, (a.gate_token ? at : 0) + c, k);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(a.res_scale, x[i], a.block_scale * (u[i] * rho * w[i] * k[i]));
  }
  // the backward's G, and xh and dn where there is a norm
  __device__ __forceinline__ void grad(int64_t c, float sig, float ch, float (&g)[8], float (&xh)[8], float (&q)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 0.f;
    if (a.dh_out) load8((const R*)a.dh_out + at + c, g);
    if (!a.w_pre) return;
    float w[8];
    load8((const R*)a.h + at + c, xh);
    load8(a.dn + at + c, q);
    load8(a.w_pre + c, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      xh[i] *= sig;
      g[i] = fmaf(sig, fmaf(-ch, xh[i], q[i] * w[i]), g[i]);
    }
  }
};

template <class R>
__global__ __launch_bounds__(256) void join_fwd_wide_kernel(const NormJoinArgs a) {
  __shared__ float red[4];
  const float inv_d = 1.f / (float)a.d;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const WideRow<R> row{a, t * a.d};
    float rho = 1.f, sig = 1.f, x[8];
    if (a.w_post) {
      float s = 0.f;
      for (int64_t c = threadIdx.x * 8; c < a.d; c += 2048) {
        load8(a.b + row.at + c, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
      }
      rho = 1.f / sqrtf(block_sum<4>(s, red) * inv_d + a.eps);
    }
    if (a.w_pre) {
      float s = 0.f;
      for (int64_t c = threadIdx.x * 8; c < a.d; c += 2048) {
        row.joined(c, rho, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
      }
      sig = 1.f / sqrtf(block_sum<4>(s, red) * inv_d + a.eps);
    }
    for (int64_t c = threadIdx.x * 8; c < a.d; c += 2048) {
      row.joined(c, rho, x);   // (before the stores, which may go to the same place)
      if (a.b) store8((R*)a.h_out + row.at + c, x);
      if (!a.w_pre) continue;
      float w[8];
      load8(a.w_pre + c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] *= x[i] * sig;
      store8(a.n + row.at + c, w);
    }
  }
}

// The sums over a workgroup's tokens are kept in its row of `part` (a thread's
// columns are its own).
template <class R>
__global__ __launch_bounds__(256) void join_bwd_wide_kernel(const NormJoinArgs a, float* part) {
  __shared__ float red[4];
  const int64_t d = a.d;
  const float inv_d = 1.f / (float)d;
  float* sums = part ? part + (int64_t)blockIdx.x * 2 * d : nullptr;
  bool first = true;
  auto add_sums = [&](float* to, const float (&x)[8], const float (&y)[8]) {
    float s[8] = {};
    if (!first) load8(to, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = fmaf(x[i], y[i], s[i]);
    store8(to, s);
  };
  if (sums && blockIdx.x >= a.T)
    for (int64_t c = threadIdx.x; c < 2 * d; c += 256) sums[c] = 0.f;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x, first = false) {
    const WideRow<R> row{a, t * d};
    float hh = 0.f, qh = 0.f, bb = 0.f, x[8], q[8], w[8], g[8];
    for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
      if (a.w_pre) {
        load8((const R*)a.h + row.at + c, x);
        load8(a.dn + row.at + c, q);
        load8(a.w_pre + c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) hh = fmaf(x[i], x[i], hh), qh = fmaf(q[i] * w[i], x[i], qh);
      }
      if (a.w_post) {
        load8(a.b + row.at + c, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) bb = fmaf(x[i], x[i], bb);
      }
    }
    const float sig = 1.f / sqrtf(block_sum<4>(hh, red) * inv_d + a.eps);
    const float ch = block_sum<4>(qh, red) * sig * inv_d;
    const float b2 = block_sum<4>(bb, red);
    const float rho = a.w_post ? 1.f / sqrtf(b2 * inv_d + a.eps) : 1.f;
    float cb = 0.f;
    if (a.w_post) {
      float pb = 0.f;
      for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
        float k[8];
        row.grad(c, sig, ch, g, x, q);
        load8(a.b + row.at + c, x);
        load8(a.w_post + c, w);
        row.factor(a.gate, (a.gate_token ? row.at : 0) + c, k);
#pragma unroll
        for (int i = 0; i < 8; ++i) pb = fmaf(a.block_scale * g[i] * k[i] * w[i], x[i] * rho, pb);
      }
      cb = block_sum<4>(pb, red) * inv_d;
    }
    for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
      float k[8], o[8];
      row.grad(c, sig, ch, g, x, q);
      if (a.w_pre) add_sums(sums + c, q, x);
      if (a.b) load8(a.b + row.at + c, x);
      if (a.dh) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = a.res_scale * g[i];
        store8((R*)a.dh + row.at + c, o);
      }
      if (!a.b) continue;
      row.factor(a.w_post, c, w);
      row.factor(a.gate, (a.gate_token ? row.at : 0) + c, k);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= rho;   // bh
      if (a.gate_token) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = a.block_scale * g[i] * x[i] * w[i], g[i] *= k[i];
        store8((uint16_t*)a.dgate + row.at + c, o);
      }
      if (sums) add_sums(sums + d + c, g, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = a.block_scale * g[i] * (a.gate_token ? 1.f : k[i]) * w[i];
        g[i] = a.w_post ? rho * fmaf(-cb, x[i], p) : p;
      }
      store8(a.db + row.at + c, g);
    }
  }
}

// How rows of d features are worked on: `waves` to a row (0: the kernels for wider
// rows), `pieces` of 8 features to a lane.
struct RowShape {
  int waves, pieces;
};
RowShape row_shape(int64_t d) {
  if (d <= 512) return {1, 1};
  if (d <= 1024) return {2, 1};
  if (d <= 2048) return {4, 1};
  if (d <= 4096) return {8, 1};
  if (d <= 8192) return {8, 2};
  return {0, 0};
}
int64_t row_groups(int64_t T, int64_t d) {   // workgroups, at one row (or set of rows) each
  const int w = row_shape(d).waves, rows = w == 1 ? 4 : w == 2 ? 2 : 1;
  return (T + rows - 1) / rows;
}
// Forward: a workgroup per row or set of rows (1B, 65536 tokens, float32 stream: 269 us;
// 2048 workgroups that go on to further rows 312).  Backward: each workgroup leaves a row
// of partial sums, so no more than the card holds at once; of these, of 4 waves each, 3 waves
// to a SIMD, or 2 where a value of a row has 10 bytes or more to read.  More waves have more
// rows on their way than the memory serves well, and it is whole waves to each SIMD that load
// it evenly: 1B, 65536 tokens, bf16 (8 bytes): 2 waves 324 us, 2.5 305, 3 286, 3.5 332, 4 300;
// 350M, 16381 tokens, float32, gate per token (14 bytes): 1.5 waves 73, 2 66, 3 71, 4 74.
// Workgroups of 8 waves put 2 on every SIMD, so it is whole workgroups to each CU: 2, and 1
// where the pieces' registers leave no room for a second.  Without post-norm and gate, bf16,
// 256 workgroups / 384 / 512: rows of 2056 (32768) 256 / 211 / 166 us; 4096 (32768) 339 / 278 /
// 275; 8192 (16384, two pieces) 308 / 370 / 311; with post-norm, gate per token and float32,
// where 4-wave workgroups gain by having fewer: 396 / 315 / 286, 564 / 582 / 543, 520 / 598 / 530.
int64_t fwd_grid(int64_t T, int64_t d) { return std::min<int64_t>(row_groups(T, d), 1 << 20); }
int64_t bwd_grid(int64_t T, int64_t d, int waves_per_simd) {
  const RowShape s = row_shape(d);
  const int to_a_cu = s.waves != 8 ? waves_per_simd : s.pieces == 1 ? 2 : 1;
  return std::max<int64_t>(1, std::min<int64_t>(row_groups(T, d), 256 * to_a_cu));
}
constexpr int kMostWaves = 3;
// Bytes of a row's value that the backward reads, and that it writes.
int bwd_reads(const NormJoinArgs& a) {
  const int res = a.res_f32 ? 4 : 2;
  return (a.dh_out ? res : 0) + (a.w_pre ? 2 + res : 0) + (a.b ? 2 : 0) + (a.gate_token ? 2 : 0);
}
int bwd_writes(const NormJoinArgs& a) { return (a.dh ? a.res_f32 ? 4 : 2 : 0) + (a.b ? 2 : 0) + (a.gate_token ? 2 : 0); }
int64_t bwd_grid(const NormJoinArgs& a) { return bwd_grid(a.T, a.d, bwd_reads(a) >= 10 ? 2 : kMostWaves); }

// Backward loads go past the caches where the call moves more than the last-level
// cache's 256 MB (1B, 65536 tokens 298 -> 285 us; 350M, 16381 tokens, float32, gate per token 70
// -> 66); in a smaller one they would miss what that cache holds (350M, 8192 tokens 24.8 ->
// 30.3).  Forward loads never gained (1B 280 -> 288).  Stores: kStreamStores in the forward, always in the backward.
constexpr int64_t kStreamLoads = int64_t(1) << 28;   // bytes

template <class R, bool STREAM>
void launch_fwd(const NormJoinArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)fwd_grid(a.T, a.d));
  const RowShape s = row_shape(a.d);
  if (s.waves == 1)
    hipLaunchKernelGGL((join_fwd_kernel<R, 1, 1, STREAM>), grid, dim3(256), 0, stream, a);
  else if (s.waves == 2)
    hipLaunchKernelGGL((join_fwd_kernel<R, 2, 1, STREAM>), grid, dim3(256), 0, stream, a);
  else if (s.waves == 4)
    hipLaunchKernelGGL((join_fwd_kernel<R, 4, 1, STREAM>), grid, dim3(256), 0, stream, a);
  else if (s.waves == 8 && s.pieces == 1)
    hipLaunchKernelGGL((join_fwd_kernel<R, 8, 1, STREAM>), grid, dim3(512), 0, stream, a);
  else if (s.waves == 8)
    hipLaunchKernelGGL((join_fwd_kernel<R, 8, 2, STREAM>), grid, dim3(512), 0, stream, a);
  else
    hipLaunchKernelGGL((join_fwd_wide_kernel<R>), grid, dim3(256), 0, stream, a);
}

template <class R, bool STREAM>
void launch_bwd(const NormJoinArgs& a, float* part, hipStream_t stream) {
  const dim3 grid((unsigned)bwd_grid(a));
  const RowShape s = row_shape(a.d);
  const size_t lds = part ? (size_t)(2 * a.d) * sizeof(float) : 0;   // (where a workgroup takes several rows)
  if (s.waves == 1)
    hipLaunchKernelGGL((join_bwd_kernel<R, 1, 1, STREAM>), grid, dim3(256), lds, stream, a, part);
  else if (s.waves == 2)
    hipLaunchKernelGGL((join_bwd_kernel<R, 2, 1, STREAM>), grid, dim3(256), lds, stream, a, part);
  else if (s.waves == 4)
    hipLaunchKernelGGL((join_bwd_kernel<R, 4, 1, STREAM>), grid, dim3(256), 0, stream, a, part);
  else if (s.waves == 8 && s.pieces == 1)
    hipLaunchKernelGGL((join_bwd_kernel<R, 8, 1, STREAM>), grid, dim3(512), 0, stream, a, part);
  else if (s.waves == 8)
    hipLaunchKernelGGL((join_bwd_kernel<R, 8, 2, STREAM>), grid, dim3(512), 0, stream, a, part);
  else
    hipLaunchKernelGGL((join_bwd_wide_kernel<R>), grid, dim3(256), 0, stream, a, part);
}

}  // namespace

size_t norm_join_bwd_workspace_bytes(int64_t T, int64_t d) { return (size_t)(bwd_grid(T, d, kMostWaves) * 2 * d) * sizeof(float); }

hipError_t run_norm_join_fwd(const NormJoinArgs& a, hipStream_t stream) {
  TimedLaunch tl("norm_join_fwd", stream);
  const bool streams = a.T * a.d >= kStreamStores;
  if (a.res_f32)
    streams ? launch_fwd<float, true>(a, stream) : launch_fwd<float, false>(a, stream);
  else
    streams ? launch_fwd<uint16_t, true>(a, stream) : launch_fwd<uint16_t, false>(a, stream);
  return hipGetLastError();
}

hipError_t run_norm_join_bwd(const NormJoinArgs& a, hipStream_t stream) {
  const bool first = a.dw_pre, second = a.dw_post || (a.dgate && !a.gate_token);
  float* part = first || second ? (float*)a.ws : nullptr;
  {
    TimedLaunch tl("norm_join_bwd", stream);
    const bool streams = a.T * a.d * (bwd_reads(a) + bwd_writes(a)) >= kStreamLoads;
    if (a.res_f32)
      streams ? launch_bwd<float, true>(a, part, stream) : launch_bwd<float, false>(a, part, stream);
    else
      streams ? launch_bwd<uint16_t, true>(a, part, stream) : launch_bwd<uint16_t, false>(a, part, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !part) return e;
  }
  TimedLaunch tl("norm_join_bwd_sums", stream);
  const int64_t c0 = first ? 0 : a.d, c1 = second ? 2 * a.d : a.d;
  hipLaunchKernelGGL(join_reduce_kernel, dim3((unsigned)((c1 - c0 + 31) / 32)), dim3(256), 0, stream, a, (const float*)part,
                     (int)bwd_grid(a), c0, c1);
  return hipGetLastError();
}

}  // namespace elas
