// Device helpers of the kernels that read and write spans of values at any alignment of
// their elements: N consecutive values, 16 bytes of float32 or bf16 (or 8 of bf16).
#pragma once

#include <math.h>

#include "rows.h"

namespace elas {

// (As a template argument these types would lose their alignment, so every access names its type.)
typedef f32x4 f32x4_span __attribute__((aligned(4)));
typedef u32x4 u32x4_span __attribute__((aligned(2)));
typedef u32x2 u32x2_span __attribute__((aligned(2)));

__device__ __forceinline__ float span_value(float e) { return e; }
__device__ __forceinline__ float span_value(uint16_t e) { return as_float((uint32_t)e << 16); }
__device__ __forceinline__ void set_span_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void set_span_value(uint16_t* p, float v) { *p = (uint16_t)bf16x2_rne(v, 0.f); }

// 4 values of either type as they were loaded.
template <class E>
struct Four;
template <>
struct Four<float> {
  f32x4 q;
  template <bool STREAM>
  __device__ __forceinline__ void load(const float* p) {
    q = STREAM ? __builtin_nontemporal_load((const f32x4_span*)p) : *(const f32x4_span*)p;
  }
  __device__ __forceinline__ void set(const float (&v)[4]) { q = f32x4{v[0], v[1], v[2], v[3]}; }
  __device__ __forceinline__ float get(int i) const { return q[i]; }
  template <bool STREAM>
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
    const f32x4 q = {v[0], v[1], v[2], v[3]};
    if constexpr (STREAM)
      __builtin_nontemporal_store(q, (f32x4_span*)p);
    else
      *(f32x4_span*)p = q;
  }
};
template <>
struct Four<uint16_t> {
  u32x2 q;
  template <bool STREAM>
  __device__ __forceinline__ void load(const uint16_t* p) {
    q = STREAM ? __builtin_nontemporal_load((const u32x2_span*)p) : *(const u32x2_span*)p;
  }
  __device__ __forceinline__ void set(const float (&v)[4]) { q = u32x2{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])}; }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = q[i >> 1];
    return as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
  }
  template <bool STREAM>
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[4]) {
    const u32x2 q = {bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])};
    if constexpr (STREAM)
      __builtin_nontemporal_store(q, (u32x2_span*)p);
    else
      *(u32x2_span*)p = q;
  }
};

// 16 bytes of either type as they were loaded.
template <class E>
struct Span;
template <>
struct Span<float> : Four<float> {
  static constexpr int N = 4;
  using Four<float>::set;
  __device__ __forceinline__ void set(int i, float v) { q[i] = v; }
  __device__ __forceinline__ void keep_packed() {}
  // -inf everywhere
  __device__ __forceinline__ void clear() { q = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY}; }
};
template <>
struct Span<uint16_t> {
  static constexpr int N = 8;
  u32x4 q;
  __device__ __forceinline__ void clear() { q = u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u}; }
  // Keeps the compiler from holding the values as 8 floats instead of 4 words from here on.
  __device__ __forceinline__ void keep_packed() { asm volatile("" : "+v"(q)); }
  template <bool STREAM>
  __device__ __forceinline__ void load(const uint16_t* p) {
    q = STREAM ? __builtin_nontemporal_load((const u32x4_span*)p) : *(const u32x4_span*)p;
  }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = q[i >> 1];
    return as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
  }
  template <bool STREAM>
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[8]) {
    const u32x4 q = {bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3]), bf16x2_rne(v[4], v[5]), bf16x2_rne(v[6], v[7])};
    if constexpr (STREAM)
      __builtin_nontemporal_store(q, (u32x4_span*)p);
    else
      *(u32x4_span*)p = q;
  }
};

// Largest of a wave, the same in every lane.  (NaN counts as nothing.)
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  v = fmaxf(v, dpp<0x141>(v));
  v = fmaxf(v, dpp<0x140>(v));
  const uint32_t w = __builtin_bit_cast(uint32_t, v);
  const auto s16 = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  v = fmaxf(as_float(s16[0]), as_float(s16[1]));
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const auto s32 = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return fmaxf(as_float(s32[0]), as_float(s32[1]));
}
// K sums over a workgroup of WAVES waves at once, with one barrier; thread k gets the k-th.  `lds` holds WAVES rows.
template <int WAVES, int K>
__device__ __forceinline__ double block_sums(const double (&s)[K], double (*lds)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const double v = wave_sum(s[k]);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6][k] = v;
  }
  __syncthreads();
  double v = 0.0;
  if (threadIdx.x < K)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += lds[w][threadIdx.x];
  return v;
}

}  // namespace elas
