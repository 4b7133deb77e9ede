// AdamW over many tensors (the formulas and the 8-bit format are in include/elas_adamw.h).
//
// A first launch of one thread finds the step's factors in 64 bits and counts the step; then
// one launch for up to kTensors tensors does everything to every value: read p, g and the
// moments, write p, the moments and the copy.  Tensors are cut into pieces of kPiece
// values, numbered through and dealt out to the workgroups in turn.  A wave takes 256 values
// at a time, 4 to a lane: a block of moments in 8 bits is one wave's, its largest magnitude
// a maximum over the wave.
#include <math.h>

#include <algorithm>

#include "../../include/elas_adamw.h"
#include "internal.h"
#include "spans.h"

namespace elas {

namespace {

constexpr int kTensors = 64;      // per launch, at most (a lane of a wave to each)
constexpr int kBlock = ELAS_ADAMW_BLOCK;
constexpr int kPiece = 2048;      // values: 2 blocks to each of a workgroup's 4 waves
constexpr int kGroups = 4096;     // most workgroups per launch
constexpr float kTopM = 245760.f, kTopV = 507904.f;     // largest codes: 15 2^14, 31 2^14

// What the step's formulas need, found once.
struct Factors {
  float clip, clip_power;   // the gradients' factor and a power of two: below 2^-126 float32 has fewer bits
  float rate, root;         // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  float lr;                 // (decay_k lr is taken off p)
  uint32_t key;             // mix(t)
  uint32_t skip;
};

// 32 bits mixed: a bijection, so no two inputs share an output.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

__global__ void adamw_factors_kernel(int64_t* step, double rate, const float* rate_factor, double beta1, double beta2, const float* norm,
                                     double max_norm, Factors* out) {
  if (threadIdx.x != 0) return;
  Factors f{};
  double clip = 1.0;
  if (norm) {
    const double n = (double)norm[0];
    f.skip = !(fabs(n) < (double)INFINITY);
    if (n > max_norm) clip = max_norm / n;
  }
  f.clip_power = clip < 0x1p-126 ? 0x1p-126f : 1.f;
  f.clip = (float)(clip / (double)f.clip_power);
  const int64_t t = step[0] + 1;
  const double lr = rate_factor ? rate * (double)rate_factor[0] : rate;
  f.lr = (float)lr;
  f.rate = (float)(lr / (1.0 - pow(beta1, (double)t)));
  f.root = (float)sqrt(1.0 / (1.0 - pow(beta2, (double)t)));
  f.key = mix((uint32_t)t);
  if (!f.skip) step[0] = t;
  out[0] = f;
}

// The tensors of a launch, as a kernel argument of room for CAP.
template <int CAP>
struct Tensors {
  void* p[CAP];
  const void* g[CAP];
  uint16_t* copy[CAP];
  int64_t block[CAP];        // first block of its moments
  uint32_t first[CAP + 1];   // number of its first piece; [count] = pieces in all
  float decay[CAP];
  uint16_t last[CAP];        // values of its last piece
  uint32_t p_bf16[CAP / 32], g_bf16[CAP / 32];
  int count, number;         // tensors here; number of the first of them in the call
  __device__ __forceinline__ int values(uint32_t c, int k) const { return c + 1 < first[k + 1] ? kPiece : (int)last[k]; }
};

struct Moments {
  void *m, *v;
  float *m_scale, *v_scale;
};
struct Betas {
  float b1, c1, b2, c2, eps;   // c = 1 - b
};

// A magnitude's code: y in units of the scale, u 16 random bits.  From 2^MANTISSA on codes are the
// upper bits of a float32, below that whole numbers; adding u below the lowest bit kept and
// cutting off rounds up with the probability of the distance to the lower neighbour.
template <int MANTISSA>
__device__ __forceinline__ uint32_t code_of(float y, uint32_t u) {
  constexpr int SHIFT = 23 - MANTISSA;
  const uint32_t high = ((__builtin_bit_cast(uint32_t, y) + (u << (SHIFT - 16))) >> SHIFT) - ((126u + MANTISSA) << MANTISSA);
  const uint32_t low = (uint32_t)(fminf(y, 64.f) + (float)u * 0x1p-16f);   // (held to the range of the conversion)
  const uint32_t code = y >= (float)(1 << MANTISSA) ? high : low;
  constexpr uint32_t TOP = (16u << MANTISSA) - 1;
  return code < TOP ? code : TOP;
}
// What a code's magnitude stands for, in units of its scale.
template <int MANTISSA>
__device__ __forceinline__ float code_value(uint32_t code) {
  const uint32_t e = code >> MANTISSA;
  const float low = (float)code;
  // the code with a bit in front of its mantissa, as the upper bits of a float32
  const float high = as_float((code + ((126u + MANTISSA) << MANTISSA)) << (23 - MANTISSA));
  return e ? high : low;
}

// Scale of a block from its largest magnitude's bits.
__device__ __forceinline__ float scale_of(uint32_t top_bits, float top) { return as_float(top_bits) / top; }

struct Update {
  Factors f;
  Betas b;
  float keep;    // 1 - lr decay
  __device__ __forceinline__ void moments(float g, float& m, float& v) const {
    g = g * f.clip * f.clip_power;
    m = fmaf(b.b1, m, b.c1 * g);
    v = fmaf(b.b2, v, b.c2 * g * g);
  }
  __device__ __forceinline__ float weight(float p, float m, float v) const {
    return fmaf(p, keep, -(f.rate * (m / (sqrtf(v) * f.root + b.eps))));
  }
};

// 256 values of a tensor from value `at` on, n of them the tensor's; `moment`: their first moment's place.
template <class P, class G, bool EIGHT>
__device__ __forceinline__ void update_block(P* p, const G* g, uint16_t* copy, int n, const Moments& s, int64_t moment, const Update& u,
                                             uint32_t key, uint32_t index) {
  const int lane = threadIdx.x & 63, i = 4 * lane;
  const bool whole = i + 4 <= n;
  float pv[4] = {}, gv[4] = {}, m[4], v[4], scale_m = 0.f, scale_v = 0.f;
  if (whole) {
    Four<P> a;
    Four<G> b;
    a.template load<false>(p + i);
    b.template load<false>(g + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) pv[k] = a.get(k), gv[k] = b.get(k);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) pv[k] = span_value(p[i + k]), gv[k] = span_value(g[i + k]);
  }
  if constexpr (EIGHT) {
    const uint32_t mc = *(const uint32_t*)((const uint8_t*)s.m + moment + i), vc = *(const uint32_t*)((const uint8_t*)s.v + moment + i);
    const int64_t block = moment / kBlock;
    scale_m = s.m_scale[block];
    scale_v = s.v_scale[block];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t c = mc >> (8 * k) & 0xFFu;
      const float x = code_value<3>(c & 0x7Fu) * scale_m;
      m[k] = c & 0x80u ? -x : x;
      v[k] = code_value<4>(vc >> (8 * k) & 0xFFu) * scale_v;
    }
  } else {
    const f32x4 a = *(const f32x4*)((const float*)s.m + moment + i), b = *(const f32x4*)((const float*)s.v + moment + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = a[k], v[k] = b[k];
  }
  float out[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    u.moments(gv[k], m[k], v[k]);
    if (i + k >= n) m[k] = v[k] = 0.f;
    out[k] = u.weight(pv[k], m[k], v[k]);
  }
  if (whole) {
    Four<P>::template store<false>(p + i, out);
    if (copy) Four<uint16_t>::template store<false>(copy + i, out);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) {
        set_span_value(p + i + k, out[k]);
        if (copy) set_span_value(copy + i + k, out[k]);
      }
  }
  if constexpr (EIGHT) {
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t a = __builtin_bit_cast(uint32_t, m[k]) & 0x7FFFFFFFu, b = __builtin_bit_cast(uint32_t, v[k]) & 0x7FFFFFFFu;
      top_m = a > top_m ? a : top_m;
      top_v = b > top_v ? b : top_v;
    }
    scale_m = scale_of(wave_max(top_m), kTopM);
    scale_v = scale_of(wave_max(top_v), kTopV);
    // (a block of zeros, or of magnitudes whose scale float32 cannot hold)
    const float div_m = scale_m > 0.f ? scale_m : 1.f, div_v = scale_v > 0.f ? scale_v : 1.f;
    uint32_t mc = 0, vc = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t bits = mix(index + (uint32_t)(i + k) + key);
      uint32_t c = code_of<3>(fabsf(m[k]) / div_m, bits & 0xFFFFu);
      if (m[k] < 0.f) c |= 0x80u;
      mc |= c << (8 * k);
      c = code_of<4>(v[k] / div_v, bits >> 16);
      if (v[k] > 0.f && c == 0) c = 1;
      vc |= c << (8 * k);
    }
    *(uint32_t*)((uint8_t*)s.m + moment + i) = mc;
    *(uint32_t*)((uint8_t*)s.v + moment + i) = vc;
    if (lane == 0) {
      s.m_scale[moment / kBlock] = scale_m;
      s.v_scale[moment / kBlock] = scale_v;
    }
  } else {
    *(f32x4*)((float*)s.m + moment + i) = f32x4{m[0], m[1], m[2], m[3]};
    *(f32x4*)((float*)s.v + moment + i) = f32x4{v[0], v[1], v[2], v[3]};
  }
}

template <class P, class G, bool EIGHT>
__device__ __forceinline__ void update_piece(P* p, const G* g, uint16_t* copy, int n, const Moments& s, int64_t moment, const Update& u,
                                             uint32_t key, uint32_t index) {
  for (int at = (int)(threadIdx.x >> 6) * kBlock; at < n; at += 4 * kBlock)
    update_block<P, G, EIGHT>(p + at, g + at, copy ? copy + at : nullptr, n - at, s, moment + at, u, key, index + at);
}

template <int CAP, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(const Tensors<CAP> a, const Moments s, const Betas b, const Factors* factors) {
  const Factors f = *factors;
  if (f.skip) return;
  const int lane = threadIdx.x & 63;
  const uint32_t firsts = lane < a.count ? a.first[lane] : ~0u;
  const uint32_t pieces = a.first[a.count];
  for (uint32_t c = blockIdx.x; c < pieces; c += gridDim.x) {
    // the last tensor whose first piece is not behind it
    const int k = __popcll(__ballot(firsts <= c)) - 1;
    const int64_t at = (int64_t)(c - a.first[k]) * kPiece;
    const int n = a.values(c, k);
    const Update u{f, b, 1.f - f.lr * a.decay[k]};
    const uint32_t key = mix(mix(f.key + (uint32_t)(a.number + k)));
    const int64_t moment = a.block[k] * kBlock + at;
    uint16_t* copy = a.copy[k] ? a.copy[k] + at : nullptr;
    const bool pb = a.p_bf16[k >> 5] >> (k & 31) & 1u, gb = a.g_bf16[k >> 5] >> (k & 31) & 1u;
    if (pb) {
      uint16_t* p = (uint16_t*)a.p[k] + at;
      gb ? update_piece<uint16_t, uint16_t, EIGHT>(p, (const uint16_t*)a.g[k] + at, copy, n, s, moment, u, key, (uint32_t)at)
         : update_piece<uint16_t, float, EIGHT>(p, (const float*)a.g[k] + at, copy, n, s, moment, u, key, (uint32_t)at);
    } else {
      float* p = (float*)a.p[k] + at;
      gb ? update_piece<float, uint16_t, EIGHT>(p, (const uint16_t*)a.g[k] + at, copy, n, s, moment, u, key, (uint32_t)at)
         : update_piece<float, float, EIGHT>(p, (const float*)a.g[k] + at, copy, n, s, moment, u, key, (uint32_t)at);
    }
  }
}

// Values of codes, 4 to a lane: a wave to a block.
template <bool SECOND, class E>
__global__ __launch_bounds__(256) void adam8_values_kernel(const uint8_t* codes, const float* scale, int64_t blocks, E* out) {
  const int lane = threadIdx.x & 63;
  for (int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); b < blocks; b += (int64_t)gridDim.x * 4) {
    const int64_t i = b * kBlock + 4 * lane;
    const uint32_t q = *(const uint32_t*)(codes + i);
    const float s = scale[b];
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t c = q >> (8 * k) & 0xFFu;
      if (SECOND) {
        v[k] = code_value<4>(c) * s;
      } else {
        const float x = code_value<3>(c & 0x7Fu) * s;
        v[k] = c & 0x80u ? -x : x;
      }
    }
    Four<E>::template store<false>(out + i, v);
  }
}

// ---- host -----------------------------------------------------------------------------

template <bool EIGHT>
hipError_t launch_update(const AdamwArgs& c, int64_t k0, int count, int64_t& block, const Betas& b, hipStream_t stream) {
  Tensors<kTensors> a{};
  a.count = count;
  a.number = (int)k0;
  uint32_t pieces = 0;
  for (int k = 0; k < count; ++k) {
    const int64_t n = c.numel[k0 + k], of = (n + kPiece - 1) / kPiece;
    a.p[k] = c.params[k0 + k];
    a.g[k] = c.grads[k0 + k];
    a.copy[k] = c.copies ? c.copies[k0 + k] : nullptr;
    a.block[k] = block;
    a.first[k] = pieces;
    a.decay[k] = c.decay[k0 + k];
    a.last[k] = (uint16_t)(n - (of - 1) * kPiece);
    pieces += (uint32_t)of;
    block += (n + kBlock - 1) / kBlock;
    if (c.param_dtype[k0 + k] == ELAS_GRAD_BF16) a.p_bf16[k >> 5] |= 1u << (k & 31);
    if (c.grad_dtype[k0 + k] == ELAS_GRAD_BF16) a.g_bf16[k >> 5] |= 1u << (k & 31);
  }
  a.first[count] = pieces;
  if (pieces == 0) return hipSuccess;
  const Moments s{c.m, c.v, c.m_scale, c.v_scale};
  TimedLaunch tl(EIGHT ? "adamw8" : "adamw", stream);
  hipLaunchKernelGGL((adamw_kernel<kTensors, EIGHT>), dim3(std::min<uint32_t>(pieces, kGroups)), dim3(256), 0, stream, a, s, b,
                     (const Factors*)c.ws);
  return hipGetLastError();
}

}  // namespace

size_t adamw_workspace_bytes() { return sizeof(Factors) + 16 - sizeof(Factors) % 16; }

hipError_t run_adamw(const AdamwArgs& a, hipStream_t stream) {
  {
    TimedLaunch tl("adamw_factors", stream);
    hipLaunchKernelGGL(adamw_factors_kernel, dim3(1), dim3(64), 0, stream, a.step, a.rate, a.rate_factor, a.beta1, a.beta2, a.norm, a.max_norm,
                       (Factors*)a.ws);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const Betas b{(float)a.beta1, (float)(1.0 - a.beta1), (float)a.beta2, (float)(1.0 - a.beta2), (float)a.eps};
  int64_t block = 0;
  for (int64_t k = 0; k < a.n; k += kTensors) {
    const int count = (int)std::min<int64_t>(kTensors, a.n - k);
    const hipError_t e = a.eight ? launch_update<true>(a, k, count, block, b, stream) : launch_update<false>(a, k, count, block, b, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t run_adam8_values(const uint8_t* codes, const float* scale, int64_t blocks, bool second, bool f32, void* out, hipStream_t stream) {
  TimedLaunch tl("adam8_values", stream);
  const auto launch = [&](auto kernel, auto* to) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>((blocks + 3) / 4, 1 << 14)), dim3(256), 0, stream, codes, scale, blocks, to);
  };
  if (second)
    f32 ? launch(adam8_values_kernel<true, float>, (float*)out) : launch(adam8_values_kernel<true, uint16_t>, (uint16_t*)out);
  else
    f32 ? launch(adam8_values_kernel<false, float>, (float*)out) : launch(adam8_values_kernel<false, uint16_t>, (uint16_t*)out);
  return hipGetLastError();
}

}  // namespace elas
