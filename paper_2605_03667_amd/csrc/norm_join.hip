// Norms before and after a block, fused with its gate and residual scale
// (forward and backward; the formulas are in include/elas_train.h).
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace elas {

namespace {

// One workgroup per row; the row is read again where a sum over it is needed first.
template <class R>
__global__ __launch_bounds__(256) void join_fwd_kernel(const NormJoinArgs a) {
  __shared__ float red[4];
  const int64_t d = a.d;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
  const R* h = (const R*)a.h + t * d;
  const uint16_t* b = a.b ? a.b + t * d : nullptr;
  const uint16_t* gate = a.gate ? a.gate + (a.gate_token ? t * d : 0) : nullptr;
  float rho = 1.f;
  if (a.w_post) {
    float s = 0.f;
    for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
      float v[8];
      load8(b + c, v);
      for (int i = 0; i < 8; ++i) s += v[i] * v[i];
    }
    rho = 1.f / sqrtf(block_sum<4>(s, red) / d + a.eps);
  }
  auto joined = [&](int64_t c, float (&v)[8]) {
    load8(h + c, v);
    if (!b) return;
    float u[8], w[8];
    load8(b + c, u);
    if (a.w_post) {
      load8(a.w_post + c, w);
      for (int i = 0; i < 8; ++i) u[i] = u[i] * rho * w[i];
    }
    if (gate) {
      load8(gate + c, w);
      for (int i = 0; i < 8; ++i) u[i] *= w[i];
    }
    for (int i = 0; i < 8; ++i) v[i] = a.res_scale * v[i] + a.block_scale * u[i];
  };
  float s = 0.f;
  if (a.w_pre)
    for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
      float v[8];
      joined(c, v);
      for (int i = 0; i < 8; ++i) s += v[i] * v[i];
    }
  const float sig = 1.f / sqrtf(block_sum<4>(s, red) / d + a.eps);
  for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
    float v[8], w[8];
    joined(c, v);
    if (a.w_pre) load8(a.w_pre + c, w);
    if (b) store8((R*)a.h_out + t * d + c, v);
    if (a.w_pre) {
      for (int i = 0; i < 8; ++i) v[i] = v[i] * sig * w[i];
      store8(a.n + t * d + c, v);
    }
  }
  }
}

// Workgroup g takes the rows g, g + grid, ..; its sums over them of the gains' and
// the shared gate's gradients go to row g of `part`, [grid][3][d].
template <class R>
__global__ __launch_bounds__(256) void join_bwd_kernel(const NormJoinArgs a, float* part) {
  __shared__ float red[4];
  const int64_t d = a.d;
  float* sums = part + (int64_t)blockIdx.x * 3 * d;
  for (int64_t c = threadIdx.x; c < 3 * d; c += 256) sums[c] = 0.f;
  __syncthreads();
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const R* h = (const R*)a.h + t * d;
    const uint16_t* b = a.b ? a.b + t * d : nullptr;
    const uint16_t* gate = a.gate ? a.gate + (a.gate_token ? t * d : 0) : nullptr;
    float hh = 0.f, qh = 0.f, bb = 0.f;
    for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
      float v[8], q[8], w[8];
      if (a.w_pre) {
        load8(h + c, v);
        load8(a.dn + t * d + c, q);
        load8(a.w_pre + c, w);
        for (int i = 0; i < 8; ++i) hh += v[i] * v[i], qh += q[i] * w[i] * v[i];
      }
      if (a.w_post) {
        load8(b + c, v);
        for (int i = 0; i < 8; ++i) bb += v[i] * v[i];
      }
    }
    hh = block_sum<4>(hh, red);
    qh = block_sum<4>(qh, red);
    bb = block_sum<4>(bb, red);
    const float sig = 1.f / sqrtf(hh / d + a.eps), rho = a.w_post ? 1.f / sqrtf(bb / d + a.eps) : 1.f;
    const float ch = qh * sig * sig * sig / d;
    auto grad = [&](int64_t c, float (&g)[8]) {   // G
      for (int i = 0; i < 8; ++i) g[i] = 0.f;
      if (a.dh_out) load8((const R*)a.dh_out + t * d + c, g);
      if (a.w_pre) {
        float v[8], q[8], w[8];
        load8(h + c, v);
        load8(a.dn + t * d + c, q);
        load8(a.w_pre + c, w);
        for (int i = 0; i < 8; ++i) g[i] += sig * (q[i] * w[i]) - v[i] * ch;
      }
    };
    float pb = 0.f;
    if (a.w_post)
      for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
        float g[8], v[8], w[8];
        grad(c, g);
        load8(a.w_post + c, w);
        load8(b + c, v);
        for (int i = 0; i < 8; ++i) pb += g[i] * a.block_scale * w[i] * v[i] * (gate ? __builtin_bit_cast(float, (uint32_t)gate[c + i] << 16) : 1.f);
      }
    pb = block_sum<4>(pb, red);
    const float cb = pb * rho * rho * rho / d;
    for (int64_t c = threadIdx.x * 8; c < d; c += 2048) {
      float g[8], v[8], q[8], w[8], o[8];
      grad(c, g);
      if (a.w_pre) {
        load8(h + c, v);
        load8(a.dn + t * d + c, q);
        for (int i = 0; i < 8; ++i) sums[2 * d + c + i] += q[i] * v[i] * sig;
      }
      if (b) load8(b + c, v);
      if (a.dh) {
        for (int i = 0; i < 8; ++i) o[i] = (b ? a.res_scale : 1.f) * g[i];
        store8((R*)a.dh + t * d + c, o);
      }
      if (!b) continue;
      for (int i = 0; i < 8; ++i) g[i] *= a.block_scale;
      if (a.w_post) load8(a.w_post + c, w);
      if (gate) {
        float k[8];
        load8(gate + c, k);
        for (int i = 0; i < 8; ++i) o[i] = g[i] * (a.w_post ? v[i] * rho * w[i] : v[i]);
        if (a.gate_token)
          store8((uint16_t*)a.dgate + t * d + c, o);
        else
          for (int i = 0; i < 8; ++i) sums[c + i] += o[i];
        for (int i = 0; i < 8; ++i) g[i] *= k[i];
      }
      if (a.w_post) {
        for (int i = 0; i < 8; ++i) {
          sums[d + c + i] += g[i] * v[i] * rho;
          g[i] = rho * (g[i] * w[i]) - v[i] * cb;
        }
      }
      store8(a.db + t * d + c, g);
    }
  }
}

__global__ __launch_bounds__(256) void join_reduce_kernel(const float* part, int64_t rows, int64_t d, float* dgate, float* dw_post,
                                                          float* dw_pre) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= 3 * d) return;
  float s = 0.f;
  for (int64_t r = 0; r < rows; ++r) s += part[r * 3 * d + c];
  float* out = c < d ? dgate : c < 2 * d ? dw_post : dw_pre;
  if (out) out[c % d] = s;
}

int64_t bwd_groups(int64_t T) { return std::max<int64_t>(1, std::min<int64_t>(T, 1024)); }

}  // namespace

size_t norm_join_bwd_workspace_bytes(int64_t T, int64_t d) { return (size_t)(bwd_groups(T) * 3 * d) * sizeof(float); }

hipError_t run_norm_join_fwd(const NormJoinArgs& a, hipStream_t stream) {
  TimedLaunch tl("norm_join_fwd", stream);
  if (a.res_f32)
    hipLaunchKernelGGL(join_fwd_kernel<float>, dim3((unsigned)std::min<int64_t>(a.T, 1 << 20)), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(join_fwd_kernel<uint16_t>, dim3((unsigned)std::min<int64_t>(a.T, 1 << 20)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t run_norm_join_bwd(const NormJoinArgs& a, hipStream_t stream) {
  float* part = (float*)a.ws;
  const unsigned groups = (unsigned)bwd_groups(a.T);
  {
    TimedLaunch tl("norm_join_bwd", stream);
    if (a.res_f32)
      hipLaunchKernelGGL(join_bwd_kernel<float>, dim3(groups), dim3(256), 0, stream, a, part);
    else
      hipLaunchKernelGGL(join_bwd_kernel<uint16_t>, dim3(groups), dim3(256), 0, stream, a, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  TimedLaunch tl("norm_join_bwd_sums", stream);
  hipLaunchKernelGGL(join_reduce_kernel, dim3((unsigned)((3 * a.d + 255) / 256)), dim3(256), 0, stream, part, (int64_t)groups, a.d,
                     a.gate_token ? nullptr : (float*)a.dgate, a.dw_post, a.dw_pre);
  return hipGetLastError();
}

}  // namespace elas
