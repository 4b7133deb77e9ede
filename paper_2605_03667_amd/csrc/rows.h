// Device helpers of the kernels that work on rows of features: pieces of 8
// consecutive features as floats, and sums over a wave or a workgroup.
#pragma once

#include "device.h"

namespace elas {

// 8 consecutive values, bf16 or float32, 16-byte aligned.
__device__ __forceinline__ void unpack8(const uint4& q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) { unpack8(*(const uint4*)p, v); }
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
  v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  *(uint4*)p = make_uint4(bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3]), bf16x2_rne(v[4], v[5]), bf16x2_rne(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
  *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// (a function: a bit cast of a vector's element itself reads element 0)
__device__ __forceinline__ float as_float(uint32_t w) { return __builtin_bit_cast(float, w); }

// Sum over a wave, the same bits in every lane: 4, then 16 lanes by lane
// permutations inside the rows of 16, then the rows by the swaps of 16 and 32 lanes.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp<0xB1>(v);    // quad_perm [1,0,3,2]
  v += dpp<0x4E>(v);    // quad_perm [2,3,0,1]
  v += dpp<0x141>(v);   // row_half_mirror
  v += dpp<0x140>(v);   // row_mirror
  const uint32_t w = __builtin_bit_cast(uint32_t, v);
  const auto s16 = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  v = as_float(s16[0]) + as_float(s16[1]);
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const auto s32 = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return as_float(s32[0]) + as_float(s32[1]);
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// 8 consecutive values as they were loaded.
template <class R>
struct Piece;
template <>
struct Piece<uint16_t> {
  uint4 q;
  __device__ __forceinline__ void load(const uint16_t* p, bool there) { q = there ? *(const uint4*)p : make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void get(float (&v)[8]) const { unpack8(q, v); }
  // A piece that stays the same over a loop: keeps the compiler from holding it as
  // 8 floats instead of 4 words.
  __device__ __forceinline__ void keep_packed() { asm volatile("" : "+v"(q.x), "+v"(q.y), "+v"(q.z), "+v"(q.w)); }
};
template <>
struct Piece<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p, bool there) {
    a = there ? *(const float4*)p : make_float4(0.f, 0.f, 0.f, 0.f);
    b = there ? *(const float4*)(p + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
  __device__ __forceinline__ void keep_packed() {}
};

// Sum over a workgroup of WAVES waves, the same in every thread; `lds` holds
// WAVES values and is free again when the next call's barrier is passed.
template <int WAVES, class T>
__device__ __forceinline__ T block_sum(T v, T* lds) {
  v = wave_sum(v);
  if (WAVES == 1) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  T s = lds[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) s += lds[w];
  return s;
}

}  // namespace elas
