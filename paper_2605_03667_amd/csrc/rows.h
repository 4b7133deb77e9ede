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
// STREAM: data that no cache is to keep (non-temporal).
template <bool STREAM, class V>
__device__ __forceinline__ void store_as(V* p, V v) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  *(uint4*)p = make_uint4(bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3]), bf16x2_rne(v[4], v[5]), bf16x2_rne(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
  *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
template <bool STREAM, class V>
__device__ __forceinline__ V load_as(const V* p) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load(p);
  else
    return *p;
}

// Non-temporal outputs from this many values on: the outputs of anything larger than a
// decode step go past the caches (norm join forward: 8192 tokens of 1B 29.2 -> 23.2 us,
// 60011 of 350M 109 -> 104; the product that reads them next is as fast or faster), a
// decode step's stay in L2 for the kernel that follows.
constexpr int64_t kStreamStores = int64_t(1) << 20;

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
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  v += dpp<0x140>(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// A lane's 8 of the 512 features that a wave takes of a row, as they were loaded.  The
// 8 are consecutive, or, SPLIT, 4 at 4 lane and 4 at 256 + 4 lane: then every access of a
// wave is contiguous in float32 too, which non-temporal stores need (65536 x 512 float32
// values: 28 us plain, 55 us non-temporal with consecutive 8).
template <class T, bool SPLIT>
struct Piece;

template <>
struct Piece<uint16_t, false> {
  u32x4 q;
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const uint16_t* p, bool there, bool) {
    q = u32x4{0u, 0u, 0u, 0u};
    if (there) q = load_as<STREAM>((const u32x4*)p);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { unpack8(make_uint4(q[0], q[1], q[2], q[3]), v); }
  template <bool STREAM>
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[8], bool there, bool) {
    if (there) store_as<STREAM>((u32x4*)p, u32x4{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3]), bf16x2_rne(v[4], v[5]), bf16x2_rne(v[6], v[7])});
  }
  // Keeps the compiler from holding the piece as 8 floats instead of 4 words from here on.
  __device__ __forceinline__ void keep_packed() { asm volatile("" : "+v"(q)); }
};
template <>
struct Piece<uint16_t, true> {
  u32x2 a, b;
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const uint16_t* p, bool there, bool there2) {
    a = b = u32x2{0u, 0u};
    if (there) a = load_as<STREAM>((const u32x2*)p);
    if (there2) b = load_as<STREAM>((const u32x2*)(p + 256));
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { unpack8(make_uint4(a[0], a[1], b[0], b[1]), v); }
  template <bool STREAM>
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[8], bool there, bool there2) {
    if (there) store_as<STREAM>((u32x2*)p, u32x2{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])});
    if (there2) store_as<STREAM>((u32x2*)(p + 256), u32x2{bf16x2_rne(v[4], v[5]), bf16x2_rne(v[6], v[7])});
  }
  __device__ __forceinline__ void keep_packed() { asm volatile("" : "+v"(a), "+v"(b)); }
};
template <bool SPLIT>
struct Piece<float, SPLIT> {
  static constexpr int SECOND = SPLIT ? 256 : 4;
  f32x4 a, b;
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const float* p, bool there, bool there2) {
    a = b = f32x4{0.f, 0.f, 0.f, 0.f};
    if (there) a = load_as<STREAM>((const f32x4*)p);
    if (there2) b = load_as<STREAM>((const f32x4*)(p + SECOND));
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
  template <bool STREAM>
  static __device__ __forceinline__ void store(float* p, const float (&v)[8], bool there, bool there2) {
    if (there) store_as<STREAM>((f32x4*)p, f32x4{v[0], v[1], v[2], v[3]});
    if (there2) store_as<STREAM>((f32x4*)(p + SECOND), f32x4{v[4], v[5], v[6], v[7]});
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
