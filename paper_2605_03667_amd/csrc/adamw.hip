// AdamW over many tensors (the formulas and the 8-bit format are in include/elas_adamw.h).
//
// A first launch of one thread finds the step's factors in 64 bits and counts the step; then
// one launch for up to kTensors tensors does everything to every value: read p, g and the
// moments, write p, the moments and the copy.  Tensors are cut into pieces, numbered through, one
// to a workgroup (dealt out to 4096 workgroups in turn 1B in 8 bits took 960 us for 822).  A wave takes 256 values
// at a time, 4 to a lane: a block of moments in 8 bits is one wave's, its largest magnitude
// a maximum over the wave.  Bound by HBM where weights are float32 (1B, 246 M values with copies: 1317 us in 32 bits,
// 5.6 TB/s; 748 in 8 bits, 5.9 TB/s), by about 60 instructions a value in 8 bits with bf16 weights and gradients (524 us, 4.7
// TB/s).  60M, 3.9 M values: 20.6 us of kernel, 22.3 a call.
#include <math.h>

#include <algorithm>

#include "../../include/elas_adamw.h"
#include "internal.h"
#include "spans.h"

namespace elas {

namespace {

constexpr int kTensors = 64;      // per launch, at most (a lane of a wave to each)
constexpr int kBlock = ELAS_ADAMW_BLOCK;
// Values of a piece: AT_ONCE blocks to each of a workgroup's 4 waves.  One, but two where moments in 8 bits and
// weights in bf16 leave a block little to load (1B: 581 us with one, 523 with two; float32 weights 744 and 798).
constexpr int piece_of(int at_once) { return 4 * at_once * kBlock; }
constexpr uint32_t kGroups = 1u << 23;   // most workgroups of a launch, of 256 threads: a grid has fewer than 2^32 threads
// Values from which on nothing is kept in the caches (350M, 46 M values: 231 us, 245 kept; 130M in 8 bits, 17 M: 62 and 59).
constexpr int64_t kStreamed = int64_t(1) << 25;
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
  // the powers side by side, by two lanes, the loads in front of them (one lane 2.9 us, so 2.1; 4.8 where the caches hold none of it)
  if (threadIdx.x > 1) return;
  const int64_t t = step[0] + 1;
  const double n = norm ? (double)norm[0] : 0.0, lr = rate_factor ? rate * (double)rate_factor[0] : rate;
  const double left = 1.0 - pow(threadIdx.x == 0 ? beta1 : beta2, (double)t), left2 = __shfl(left, 1);
  if (threadIdx.x != 0) return;
  Factors f{};
  double clip = 1.0;
  if (norm) {
    f.skip = !(fabs(n) < (double)INFINITY);
    if (n > max_norm) clip = max_norm / n;
  }
  f.clip_power = clip < 0x1p-126 ? 0x1p-126f : 1.f;
  f.clip = (float)(clip / (double)f.clip_power);
  f.lr = (float)lr;
  f.rate = (float)(lr / left);
  f.root = (float)sqrt(1.0 / left2);
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
  __device__ __forceinline__ int values(uint32_t c, int k, int piece) const { return c + 1 < first[k + 1] ? piece : (int)last[k]; }
};

struct Moments {
  void *m, *v;
  float *m_scale, *v_scale;
};
struct Betas {
  float b1, c1, b2, c2, eps;   // c = 1 - b
};

// Codes are the upper bits of a float32: a code in the bits of a float32's lowest exponents and highest mantissa
// stands for its value times 2^-(126 + MANTISSA), subnormals (e = 0) included.
template <int MANTISSA>
constexpr float kUnit = MANTISSA == 3 ? 0x1p-129f : 0x1p-130f;
template <int MANTISSA>
constexpr int kShift = 23 - MANTISSA;

// A magnitude's code: y in units of the scale, u 16 random bits.  Adding u below the lowest bit kept and cutting off
// rounds up with the probability of the distance to the lower neighbour.  (y below 2^MANTISSA is a subnormal here, to
// 2^-20 or 2^-19.)
template <int MANTISSA>
__device__ __forceinline__ uint32_t code_of(float y, uint32_t u, uint32_t least) {
  const uint32_t code = (__builtin_bit_cast(uint32_t, y * kUnit<MANTISSA>) + (u << (kShift<MANTISSA> - 16))) >> kShift<MANTISSA>;
  const uint32_t top = (16u << MANTISSA) - 1;
  return __builtin_elementwise_min(__builtin_elementwise_max(code, least), top);
}

// Values of the 4 codes of a word.  One product with the scale over the unit rounds as a product of value and scale does;
// a scale for which that leaves float32's range takes two.
template <int MANTISSA>
struct Decoder {
  float a, b;
  bool two;
  __device__ __forceinline__ explicit Decoder(float scale) {
    two = !(scale < 0x1p-4f);
    a = 0x1p127f;
    b = scale * (1.f / (kUnit<MANTISSA> * 0x1p127f));      // 4 scale, 8 scale
  }
  template <bool ANY = false>     // (ANY: two products, where lanes hold different scales)
  __device__ __forceinline__ void get(uint32_t codes, float (&v)[4]) const {
    constexpr uint32_t MASK = (16u << MANTISSA) - 1;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = as_float((codes >> (8 * k) & MASK) << kShift<MANTISSA>);
    if (ANY || two) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = v[k] * a * b;
    } else {
      const float c = a * b;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] *= c;
    }
    if constexpr (MANTISSA == 3) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = __builtin_copysignf(v[k], as_float(codes << (24 - 8 * k)));
    }
  }
};

// Largest of two magnitudes each over a wave, as bits (NaN above all): the first in lane 0 .. 31, the second in
// 32 .. 63, read into scalar registers.
__device__ __forceinline__ void wave_max2(uint32_t& a, uint32_t& b) {
  const auto s32 = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  uint32_t v = __builtin_elementwise_max(s32[0], s32[1]);
  const auto s16 = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = __builtin_elementwise_max(s16[0], s16[1]);
  const auto step = [&](uint32_t o) { v = __builtin_elementwise_max(v, o); };
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
  a = (uint32_t)__builtin_amdgcn_readlane((int)v, 0);
  b = (uint32_t)__builtin_amdgcn_readlane((int)v, 32);
}

// A block's scale, its largest magnitude (`top`, as bits) over the largest code, and its magnitudes in units of it: products with
// the reciprocal, corrected by their remainders, which came out
// as the division's rounding in all of 1.7e8 quotients of random mantissas (scales whose remainders may leave the range of
// float32 are divided).  Below float32's normal range a scale has few bits and is rounded up: rounded down it would leave the
// largest magnitude beyond the largest code, or be 0 with nothing left of the block.
template <int MANTISSA>
__device__ __forceinline__ float in_units(uint32_t top, const float (&x)[4], float (&y)[4]) {
  constexpr float TOP = MANTISSA == 3 ? kTopM : kTopV;
  float scale = as_float(top) * (1.f / TOP);
  const float s = top ? scale : 1.f;       // (a block of zeros: unit 1)
  if (s >= 0x1p-90f && s <= 0x1p90f) {
    const float r0 = __builtin_amdgcn_rcpf(s), r = fmaf(fmaf(-s, r0, 1.f), r0, r0);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float v = fabsf(x[k]), q = v * r;
      y[k] = fmaf(fmaf(-q, s, v), r, q);
    }
  } else {
    if (scale < 0x1p-126f && scale * TOP < as_float(top)) scale += 0x1p-149f;
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = fabsf(x[k]) / scale;
  }
  return scale;
}

struct Update {
  Factors f;
  Betas b;
  float keep;    // 1 - lr decay
  // Every product and sum is rounded by itself, in the order of the formulas, and so are the scales and
  // quotients of 8-bit moments: float32 arithmetic in elementary steps gives the same moments bit for bit, and with the
  // same random bits the same codes.  (Fused products would be as exact, but a code that falls to the other
  // neighbour is off by an eighth.)
  __device__ __forceinline__ void moments(float (&g)[4], float (&m)[4], float (&v)[4]) const {
#pragma clang fp contract(off)
#pragma unroll
    for (int k = 0; k < 4; ++k) g[k] = g[k] * f.clip;
    if (f.clip_power != 1.f) {
#pragma unroll
      for (int k = 0; k < 4; ++k) g[k] = g[k] * f.clip_power;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = b.b1 * m[k] + b.c1 * g[k];
      v[k] = b.b2 * v[k] + b.c2 * g[k] * g[k];
    }
  }
  // Roots of subnormals, which the instruction takes for 0, matter beside an eps under 1e-10 alone.
  __device__ __forceinline__ void weights(float (&p)[4], const float (&m)[4], const float (&v)[4]) const {
    float r[4];
    if (b.eps < 1e-10f) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool tiny = v[k] < 0x1p-126f;
        r[k] = __builtin_amdgcn_sqrtf(tiny ? v[k] * 0x1p64f : v[k]);
        r[k] = tiny ? r[k] * 0x1p-32f : r[k];
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = __builtin_amdgcn_sqrtf(v[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = fmaf(p[k], keep, -(f.rate * (m[k] * __builtin_amdgcn_rcpf(r[k] * f.root + b.eps))));
  }
};

// A lane's 4 of the 256 values of a block, as they were loaded.
template <class P, class G, bool EIGHT>
struct Block {
  Four<P> p;
  Four<G> g;
  f32x4 m, v;
  uint32_t mc, vc;
  float m_scale, v_scale;

  // `moment`: the block's first moment; `n` values of the tensor from p, g on.
  template <bool STREAM>
  __device__ __forceinline__ void load(const P* pp, const G* gp, const Moments& s, int64_t moment, int n) {
    const int i = 4 * (int)(threadIdx.x & 63);
    if constexpr (EIGHT) {
      mc = load_as<STREAM>((const uint32_t*)((const uint8_t*)s.m + moment) + i / 4);
      vc = load_as<STREAM>((const uint32_t*)((const uint8_t*)s.v + moment) + i / 4);
      m_scale = s.m_scale[moment / kBlock];
      v_scale = s.v_scale[moment / kBlock];
    } else {
      m = load_as<STREAM>((const f32x4*)((const float*)s.m + moment) + i / 4);
      v = load_as<STREAM>((const f32x4*)((const float*)s.v + moment) + i / 4);
    }
    if (i + 4 <= n) {
      p.template load<STREAM>(pp + i);
      g.template load<STREAM>(gp + i);
    } else {
      float x[4] = {}, y[4] = {};
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (i + k < n) x[k] = span_value(pp[i + k]), y[k] = span_value(gp[i + k]);
      p.set(x);
      g.set(y);
    }
  }

  template <bool STREAM>
  __device__ __forceinline__ void step(P* pp, uint16_t* copy, const Moments& s, int64_t moment, int n, const Update& u, uint32_t key, uint32_t index) {
    const int lane = threadIdx.x & 63, i = 4 * lane;
    float mv[4], vv[4], out[4];
    if constexpr (EIGHT) {
      Decoder<3>(m_scale).get(mc, mv);
      Decoder<4>(v_scale).get(vc, vv);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) mv[k] = m[k], vv[k] = v[k];
    }
    float gv[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) gv[k] = g.get(k), out[k] = p.get(k);
    u.moments(gv, mv, vv);
    u.weights(out, mv, vv);
    if (n < kBlock) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k >= n) mv[k] = vv[k] = 0.f;
    }
    if (i + 4 <= n) {
      Four<P>::template store<STREAM>(pp + i, out);
      if (copy) Four<uint16_t>::template store<false>(copy + i, out);     // (read next)
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (i + k < n) {
          set_span_value(pp + i + k, out[k]);
          if (copy) set_span_value(copy + i + k, out[k]);
        }
    }
    if constexpr (EIGHT) {
      uint32_t top_m = 0, top_v = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t a = __builtin_bit_cast(uint32_t, mv[k]) & 0x7FFFFFFFu, b = __builtin_bit_cast(uint32_t, vv[k]) & 0x7FFFFFFFu;
        top_m = a > top_m ? a : top_m;
        top_v = b > top_v ? b : top_v;
      }
      wave_max2(top_m, top_v);
      float ym[4], yv[4];
      const float new_m = in_units<3>(top_m, mv, ym), new_v = in_units<4>(top_v, vv, yv);
      uint32_t to_m = 0, to_v = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t bits = mix(index + (uint32_t)(i + k) + key), sign = __builtin_bit_cast(uint32_t, mv[k]) >> 31;
        to_m |= (code_of<3>(ym[k], bits & 0xFFFFu, 0u) | sign << 7) << (8 * k);
        const uint32_t least = __builtin_elementwise_min(__builtin_bit_cast(uint32_t, vv[k]), 1u);      // (v is not negative)
        to_v |= code_of<4>(yv[k], bits >> 16, least) << (8 * k);
      }
      store_as<STREAM>((uint32_t*)((uint8_t*)s.m + moment) + lane, to_m);
      store_as<STREAM>((uint32_t*)((uint8_t*)s.v + moment) + lane, to_v);
      if (lane == 0) {
        s.m_scale[moment / kBlock] = new_m;
        s.v_scale[moment / kBlock] = new_v;
      }
    } else {
      store_as<STREAM>((f32x4*)((float*)s.m + moment) + lane, f32x4{mv[0], mv[1], mv[2], mv[3]});
      store_as<STREAM>((f32x4*)((float*)s.v + moment) + lane, f32x4{vv[0], vv[1], vv[2], vv[3]});
    }
  }
};

// A piece: each wave takes AT_ONCE blocks, all of them loaded before the first is computed.
template <class P, class G, bool EIGHT, bool STREAM, int AT_ONCE>
__device__ __forceinline__ void update_piece(P* p, const G* g, uint16_t* copy, int n, const Moments& s, int64_t moment, const Update& u,
                                             uint32_t key, uint32_t index) {
  const int first = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * kBlock;
  Block<P, G, EIGHT> b[AT_ONCE];
#pragma unroll
  for (int q = 0; q < AT_ONCE; ++q) {
    const int at = first + q * 4 * kBlock;
    if (at < n) b[q].template load<STREAM>(p + at, g + at, s, moment + at, n - at);
  }
#pragma unroll
  for (int q = 0; q < AT_ONCE; ++q) {
    const int at = first + q * 4 * kBlock;
    if (at < n) b[q].template step<STREAM>(p + at, copy ? copy + at : nullptr, s, moment + at, n - at, u, key, index + at);
  }
}

template <int CAP, bool EIGHT, bool STREAM, int AT_ONCE>
__global__ __launch_bounds__(256) void adamw_kernel(const Tensors<CAP> a, const Moments s, const Betas b, const Factors* factors) {
  const Factors f = *factors;
  if (f.skip) return;
  const int lane = threadIdx.x & 63;
  const uint32_t firsts = lane < a.count ? a.first[lane] : ~0u;
  const uint32_t pieces = a.first[a.count];
  for (uint32_t c = blockIdx.x; c < pieces; c += gridDim.x) {
    // the last tensor whose first piece is not behind it
    const int k = __popcll(__ballot(firsts <= c)) - 1;
    const int64_t at = (int64_t)(c - a.first[k]) * piece_of(AT_ONCE);
    const int n = a.values(c, k, piece_of(AT_ONCE));
    const Update u{f, b, 1.f - f.lr * a.decay[k]};
    const uint32_t key = mix(mix(f.key + (uint32_t)(a.number + k)));
    const int64_t moment = a.block[k] * kBlock + at;
    uint16_t* copy = a.copy[k] ? a.copy[k] + at : nullptr;
    const bool pb = a.p_bf16[k >> 5] >> (k & 31) & 1u, gb = a.g_bf16[k >> 5] >> (k & 31) & 1u;
    if (pb) {
      uint16_t* p = (uint16_t*)a.p[k] + at;
      gb ? update_piece<uint16_t, uint16_t, EIGHT, STREAM, AT_ONCE>(p, (const uint16_t*)a.g[k] + at, copy, n, s, moment, u, key, (uint32_t)at)
         : update_piece<uint16_t, float, EIGHT, STREAM, AT_ONCE>(p, (const float*)a.g[k] + at, copy, n, s, moment, u, key, (uint32_t)at);
    } else {
      float* p = (float*)a.p[k] + at;
      gb ? update_piece<float, uint16_t, EIGHT, STREAM, AT_ONCE>(p, (const uint16_t*)a.g[k] + at, copy, n, s, moment, u, key, (uint32_t)at)
         : update_piece<float, float, EIGHT, STREAM, AT_ONCE>(p, (const float*)a.g[k] + at, copy, n, s, moment, u, key, (uint32_t)at);
    }
  }
}

// Values of codes, 8 to a lane: half a wave to a block.
template <bool SECOND, class E>
__global__ __launch_bounds__(256) void adam8_values_kernel(const uint8_t* codes, const float* scale, int64_t blocks, E* out) {
  const int64_t lanes = blocks * (kBlock / 8);
  for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < lanes; j += (int64_t)gridDim.x * 256) {
    const u32x2 q = __builtin_nontemporal_load((const u32x2*)codes + j);
    const Decoder<SECOND ? 4 : 3> values(scale[j / (kBlock / 8)]);
    float a[4], b[4];
    values.template get<true>(q[0], a);
    values.template get<true>(q[1], b);
    E* to = out + 8 * j;
    if constexpr (sizeof(E) == 2) {
      const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
      Span<E>::template store<true>(to, v);
    } else {
      Span<E>::template store<true>(to, a);
      Span<E>::template store<true>(to + 4, b);
    }
  }
}

// ---- host -----------------------------------------------------------------------------

template <bool EIGHT>
hipError_t launch_update(const AdamwArgs& c, int64_t k0, int count, int64_t& block, const Betas& b, bool stream_data, hipStream_t stream) {
  Tensors<kTensors> a{};
  a.count = count;
  a.number = (int)k0;
  bool small = EIGHT;
  for (int k = 0; k < count; ++k) small = small && c.param_dtype[k0 + k] == ELAS_GRAD_BF16;
  const int64_t piece = piece_of(small ? 2 : 1);
  uint32_t pieces = 0;
  for (int k = 0; k < count; ++k) {
    const int64_t n = c.numel[k0 + k], of = (n + piece - 1) / piece;
    a.p[k] = c.params[k0 + k];
    a.g[k] = c.grads[k0 + k];
    a.copy[k] = c.copies ? c.copies[k0 + k] : nullptr;
    a.block[k] = block;
    a.first[k] = pieces;
    a.decay[k] = c.decay[k0 + k];
    a.last[k] = (uint16_t)(n - (of - 1) * piece);
    pieces += (uint32_t)of;
    block += (n + kBlock - 1) / kBlock;
    if (c.param_dtype[k0 + k] == ELAS_GRAD_BF16) a.p_bf16[k >> 5] |= 1u << (k & 31);
    if (c.grad_dtype[k0 + k] == ELAS_GRAD_BF16) a.g_bf16[k >> 5] |= 1u << (k & 31);
  }
  a.first[count] = pieces;
  if (pieces == 0) return hipSuccess;
  const Moments s{c.m, c.v, c.m_scale, c.v_scale};
  TimedLaunch tl(EIGHT ? "adamw8" : "adamw", stream);
  const dim3 grid(std::min<uint32_t>(pieces, kGroups));
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, s, b, (const Factors*)c.ws); };
  if constexpr (EIGHT) {
    if (small) {
      stream_data ? launch(adamw_kernel<kTensors, true, true, 2>) : launch(adamw_kernel<kTensors, true, false, 2>);
      return hipGetLastError();
    }
  }
  stream_data ? launch(adamw_kernel<kTensors, EIGHT, true, 1>) : launch(adamw_kernel<kTensors, EIGHT, false, 1>);
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
  int64_t block = 0, total = 0;
  for (int64_t k = 0; k < a.n; ++k) total += a.numel[k];
  const bool stream_data = total >= kStreamed;
  for (int64_t k = 0; k < a.n; k += kTensors) {
    const int count = (int)std::min<int64_t>(kTensors, a.n - k);
    const hipError_t e = a.eight ? launch_update<true>(a, k, count, block, b, stream_data, stream)
                                 : launch_update<false>(a, k, count, block, b, stream_data, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t run_adam8_values(const uint8_t* codes, const float* scale, int64_t blocks, bool second, bool f32, void* out, hipStream_t stream) {
  TimedLaunch tl("adam8_values", stream);
  const auto launch = [&](auto kernel, auto* to) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>((blocks * (kBlock / 8) + 255) / 256, kGroups)), dim3(256), 0, stream, codes,
                       scale, blocks, to);
  };
  if (second)
    f32 ? launch(adam8_values_kernel<true, float>, (float*)out) : launch(adam8_values_kernel<true, uint16_t>, (uint16_t*)out);
  else
    f32 ? launch(adam8_values_kernel<false, float>, (float*)out) : launch(adam8_values_kernel<false, uint16_t>, (uint16_t*)out);
  return hipGetLastError();
}

}  // namespace elas
