// Token embedding with scaling, and its gradient by sorted tokens (the formulas
// are in include/elas_train.h).
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace elas {

namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

__device__ __forceinline__ int64_t id_at(const void* ids, bool i64, int64_t t) {
  return i64 ? ((const int64_t*)ids)[t] : (int64_t)((const int32_t*)ids)[t];
}

template <class R>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const EmbedArgs a) {
  const int64_t pieces = a.d / 8, total = a.T * pieces;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
    const int64_t t = q / pieces, c = (q - t * pieces) * 8;
    const int64_t id = id_at(a.ids, a.ids_i64, t);
    float v[8] = {};
    if (id >= 0 && id < a.V) {
      load8(a.table + id * a.d + c, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= a.scale;
    }
    store8((R*)a.x + t * a.d + c, v);
  }
}

// ---- the gradient ----------------------------------------------------------------
// Tokens are sorted by id with a stable radix sort of 8 bits a pass (ids outside
// the table become V and sort behind all others); workgroup c holds the tokens
// c * kChunk ...  Then one workgroup adds up the tokens of each row of the table.
constexpr int kChunk = 2048;

__global__ __launch_bounds__(256) void embed_keys_kernel(const EmbedArgs a, uint32_t* key, uint32_t* pos) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= a.T) return;
  const int64_t id = id_at(a.ids, a.ids_i64, t);
  key[t] = id >= 0 && id < a.V ? (uint32_t)id : (uint32_t)a.V;
  pos[t] = (uint32_t)t;
}

__global__ __launch_bounds__(256) void embed_hist_kernel(const uint32_t* key, int64_t T, int shift, uint32_t* hist) {
  __shared__ uint32_t n[256];
  n[threadIdx.x] = 0;
  __syncthreads();
  for (int64_t i = threadIdx.x; i < kChunk; i += 256) {
    const int64_t t = (int64_t)blockIdx.x * kChunk + i;
    if (t < T) atomicAdd(&n[(key[t] >> shift) & 255u], 1u);
  }
  __syncthreads();
  hist[(int64_t)blockIdx.x * 256 + threadIdx.x] = n[threadIdx.x];
}

// hist[c][digit] becomes the place of chunk c's first key with that digit.
__global__ __launch_bounds__(256) void embed_scan_kernel(uint32_t* hist, int64_t chunks) {
  __shared__ uint32_t total[256];
  uint32_t n = 0;
  for (int64_t c = 0; c < chunks; ++c) {
    const uint32_t h = hist[c * 256 + threadIdx.x];
    hist[c * 256 + threadIdx.x] = n;
    n += h;
  }
  total[threadIdx.x] = n;
  __syncthreads();
  uint32_t before = 0;
  for (int k = 0; k < (int)threadIdx.x; ++k) before += total[k];
  for (int64_t c = 0; c < chunks; ++c) hist[c * 256 + threadIdx.x] += before;
}

// One wave per chunk, 64 keys at a time in order: a key's place among the equal
// digits of its 64 is the number of lower lanes that hold the same digit.
__global__ __launch_bounds__(64) void embed_scatter_kernel(const uint32_t* key, const uint32_t* pos, int64_t T, int shift,
                                                           const uint32_t* hist, uint32_t* key_out, uint32_t* pos_out) {
  __shared__ uint32_t base[256];
  const int lane = threadIdx.x;
  for (int k = lane; k < 256; k += 64) base[k] = hist[(int64_t)blockIdx.x * 256 + k];
  __syncthreads();
  for (int64_t i = 0; i < kChunk; i += 64) {
    const int64_t t = (int64_t)blockIdx.x * kChunk + i + lane;
    const bool ok = t < T;
    const uint32_t k = ok ? key[t] : 0u, digit = (k >> shift) & 255u;
    uint64_t same = __ballot(ok);
#pragma unroll
    for (int bit = 0; bit < 8; ++bit) {
      const uint64_t m = __ballot((digit >> bit) & 1u);
      same &= (digit >> bit) & 1u ? m : ~m;
    }
    const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
    const uint32_t at = base[digit] + rank;
    __syncthreads();
    if (ok && rank == 0) base[digit] += __popcll(same);
    __syncthreads();
    if (ok) {
      key_out[at] = k;
      pos_out[at] = pos[t];
    }
  }
}

__device__ __forceinline__ int64_t lower_bound(const uint32_t* key, int64_t T, uint32_t v) {
  int64_t lo = 0, hi = T;
  while (lo < hi) {
    const int64_t m = (lo + hi) / 2;
    if (key[m] < v) lo = m + 1; else hi = m;
  }
  return lo;
}

template <class R>
__global__ __launch_bounds__(256) void embed_sum_kernel(const EmbedArgs a, const uint32_t* key, const uint32_t* pos) {
  for (int64_t v = blockIdx.x; v < a.V; v += gridDim.x) {
    const int64_t p0 = lower_bound(key, a.T, (uint32_t)v), p1 = lower_bound(key, a.T, (uint32_t)v + 1);
    if (a.add && p0 == p1) continue;
    for (int64_t c = threadIdx.x * 8; c < a.d; c += 2048) {
      float s[8] = {}, x[8];
      for (int64_t p = p0; p < p1; ++p) {
        load8((const R*)a.dx + (int64_t)pos[p] * a.d + c, x);
        for (int i = 0; i < 8; ++i) s[i] += x[i];
      }
      float* out = a.dtable + v * a.d + c;
      if (a.add) load8(out, x);
      for (int i = 0; i < 8; ++i) s[i] = a.scale * s[i] + (a.add ? x[i] : 0.f);
      store8(out, s);
    }
  }
}

struct BwdPlan {
  uint32_t *key[2], *pos[2], *hist;
  size_t bytes;
};
BwdPlan plan(void* ws, int64_t T) {
  const size_t n = (size_t)cdiv(T, 64) * 64;
  uint32_t* p = (uint32_t*)ws;
  BwdPlan b;
  for (int i = 0; i < 2; ++i) {
    b.key[i] = p + (2 * i) * n;
    b.pos[i] = p + (2 * i + 1) * n;
  }
  b.hist = p + 4 * n;
  b.bytes = (4 * n + (size_t)cdiv(T, kChunk) * 256) * sizeof(uint32_t);
  return b;
}

}  // namespace

size_t embed_bwd_workspace_bytes(int64_t T, int64_t V, int64_t d, bool add) { return plan(nullptr, T).bytes; }

hipError_t run_embed_fwd(const EmbedArgs& a, hipStream_t stream) {
  TimedLaunch tl("embed_fwd", stream);
  const unsigned grid = (unsigned)std::min<int64_t>(cdiv(a.T * (a.d / 8), 256), 1 << 20);
  if (a.res_f32)
    hipLaunchKernelGGL(embed_fwd_kernel<float>, dim3(grid), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(embed_fwd_kernel<uint16_t>, dim3(grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t run_embed_bwd(const EmbedArgs& a, hipStream_t stream) {
  const BwdPlan b = plan(a.ws, a.T);
  const unsigned chunks = (unsigned)cdiv(a.T, kChunk);
  int at = 0;
  if (a.T > 0) {
    TimedLaunch tl("embed_bwd_sort", stream);
    hipLaunchKernelGGL(embed_keys_kernel, dim3((unsigned)cdiv(a.T, 256)), dim3(256), 0, stream, a, b.key[0], b.pos[0]);
    for (int shift = 0; shift < 32 && (a.V >> shift) > 0; shift += 8) {
      hipLaunchKernelGGL(embed_hist_kernel, dim3(chunks), dim3(256), 0, stream, b.key[at], a.T, shift, b.hist);
      hipLaunchKernelGGL(embed_scan_kernel, dim3(1), dim3(256), 0, stream, b.hist, (int64_t)chunks);
      hipLaunchKernelGGL(embed_scatter_kernel, dim3(chunks), dim3(64), 0, stream, b.key[at], b.pos[at], a.T, shift, b.hist,
                         b.key[1 - at], b.pos[1 - at]);
      at = 1 - at;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  TimedLaunch tl("embed_bwd_sum", stream);
  const unsigned grid = (unsigned)std::min<int64_t>(a.V, 1 << 20);
  if (a.res_f32)
    hipLaunchKernelGGL(embed_sum_kernel<float>, dim3(grid), dim3(256), 0, stream, a, b.key[at], b.pos[at]);
  else
    hipLaunchKernelGGL(embed_sum_kernel<uint16_t>, dim3(grid), dim3(256), 0, stream, a, b.key[at], b.pos[at]);
  return hipGetLastError();
}

}  // namespace elas
