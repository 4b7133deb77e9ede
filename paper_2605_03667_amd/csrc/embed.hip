// Token embedding with scaling, and its gradient by sorted tokens (the formulas
// are in include/elas_train.h).
//
// The lookup is a copy bound by HBM and by latency: a wave takes 4 pieces of 512
// features at a time, of one token or of several, so that 4 rows are on their way at
// once (1B, 65536 tokens: 59 us).
//
// The gradient sorts the tokens by id first (stably, so that every row's sum has one
// order) and then walks the sorted tokens and the table's rows together.  The sort
// works on 4 to 8 bytes a token and is bound by latency and launches; the sum reads dx
// and writes the table once and is bound by HBM.  1B, 65536 tokens whose ids fall off
// like words: 134 us, of which the sort 2 (4.7 + 6.3), the sum 109 (4.9 TB/s), the
// joining of cut rows 6; with one id for all tokens 123.  Up to 4096 tokens one launch does
// it all (60M, 2048 tokens, added: 11.0 us), up to 8192 three do.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace elas {

namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

__device__ __forceinline__ int64_t id_at(const EmbedArgs& a, int64_t t) {
  return a.ids_i64 ? ((const int64_t*)a.ids)[t] : (int64_t)((const int32_t*)a.ids)[t];
}
// Sort key of a token: its id, V where that is outside the table.
__device__ __forceinline__ uint32_t key_at(const EmbedArgs& a, int64_t t) {
  const int64_t id = id_at(a, t);
  return id >= 0 && id < a.V ? (uint32_t)id : (uint32_t)a.V;
}

// ---- lookup -----------------------------------------------------------------------

// Parts of 512 features of consecutive tokens, numbered through; a wave takes 4 of
// them, `parts` to a token.
template <class R, bool STREAM>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const EmbedArgs a, uint32_t parts) {
  constexpr bool SPLIT = sizeof(R) == 4;
  const uint32_t lane = threadIdx.x & 63;
  const int64_t waves = (int64_t)gridDim.x * 4, total = a.T * parts;
  for (int64_t q0 = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 4; q0 < total; q0 += waves * 4) {
    int64_t t = q0 / parts;   // (the one division of a wave's turn)
    uint32_t part = (uint32_t)(q0 - t * parts);
    Piece<uint16_t, SPLIT> row[4];
    int64_t at[4];
    bool there[4], there2[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t c = part * 512 + lane * (SPLIT ? 4 : 8);
      there[k] = t < a.T && c < (uint32_t)a.d;
      there2[k] = SPLIT ? t < a.T && c + 256 < (uint32_t)a.d : there[k];
      const uint32_t key = t < a.T ? key_at(a, t) : (uint32_t)a.V;
      const bool inside = key < (uint32_t)a.V;
      row[k].load(a.table + (int64_t)key * a.d + c, there[k] && inside, there2[k] && inside);
      at[k] = t * a.d + c;
      if (++part == parts) part = 0, ++t;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float v[8];
      row[k].get(v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= a.scale;
      Piece<R, SPLIT>::template store<STREAM>((R*)a.x + at[k], v, there[k], there2[k]);
    }
  }
}

// ---- the sort -----------------------------------------------------------------------
// Least significant digit first, at most 9 bits a pass.  A workgroup of 16 waves takes
// 1024 E tokens, wave w the E rounds of 64 from w 64 E on, so that (wave, round, lane)
// is the order of the tokens.  One LDS counter for each wave and digit: of the lanes of
// a round that hold the same digit the lowest adds their number to the counter, and
// what it held before plus the number of lower such lanes is the token's place among
// the wave's tokens of that digit.  LDS operations of a wave are done in order, so the
// rounds need no wait between them.
constexpr int kDigits = 512;

// Places among the wave's own tokens of the same digit.
template <int E>
__device__ __forceinline__ void wave_ranks(const uint32_t (&digit)[E], const bool (&ok)[E], int bits, uint32_t* count, uint32_t (&rank)[E]) {
  const uint32_t lane = threadIdx.x & 63;
  uint32_t before[E], lower[E];
  int leader[E];
#pragma unroll
  for (int r = 0; r < E; ++r) {
    const uint64_t all = __ballot(ok[r]);
    uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);   // lanes with the same digit
#pragma unroll
    for (int b = 0; b < 9; ++b) {
      if (b >= bits) break;
      const uint32_t mine = (uint32_t)((int32_t)(digit[r] << (31 - b)) >> 31);   // the lane's bit b, in all bits
      const uint64_t m = __ballot(mine != 0u);
      lo &= ~((uint32_t)m ^ mine);
      hi &= ~((uint32_t)(m >> 32) ^ mine);
    }
    lower[r] = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0u));
    leader[r] = lo != 0u ? __ffs(lo) - 1 : 31 + __ffs(hi);
    before[r] = 0;
    if (ok[r] && lower[r] == 0) before[r] = atomicAdd(&count[digit[r]], (uint32_t)(__popc(lo) + __popc(hi)));
  }
#pragma unroll
  for (int r = 0; r < E; ++r) rank[r] = __shfl(before[r], ok[r] ? leader[r] : 0) + lower[r];
}

// Exclusive prefix sums over `bins` <= 512 values, one per thread 0 .. bins - 1.
__device__ __forceinline__ uint32_t bin_scan(uint32_t v, int bins, uint32_t* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // inclusive over the wave: inside the rows of 16 lanes, then row 0 into 1 and 2 into 3,
  // then the first half into the second
  uint32_t s = v;
  s += __builtin_amdgcn_update_dpp(0, s, 0x111, 0xF, 0xF, true);    // row_shr:1
  s += __builtin_amdgcn_update_dpp(0, s, 0x112, 0xF, 0xF, true);    // row_shr:2
  s += __builtin_amdgcn_update_dpp(0, s, 0x114, 0xF, 0xF, true);    // row_shr:4
  s += __builtin_amdgcn_update_dpp(0, s, 0x118, 0xF, 0xF, true);    // row_shr:8
  s += __builtin_amdgcn_update_dpp(0, s, 0x142, 0xA, 0xF, false);   // row_bcast:15
  s += __builtin_amdgcn_update_dpp(0, s, 0x143, 0xC, 0xF, false);   // row_bcast:31
  if (lane == 63 && wave * 64 < bins) tmp[wave] = s;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave && w * 64 < bins; ++w) before += tmp[w];
  return before + s - v;
}

// count[w][digit] becomes the number of equal digits in the waves before w; the return
// value is the workgroup's number of tokens with digit threadIdx.x (< bins).
__device__ __forceinline__ uint32_t wave_prefixes(uint32_t* count, int bins) {
  uint32_t n = 0;
  if ((int)threadIdx.x < bins) {
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      const uint32_t c = count[w * kDigits + threadIdx.x];
      count[w * kDigits + threadIdx.x] = n;
      n += c;
    }
  }
  return n;
}

// n <= 1024 E entries (key << tbits | token) of one workgroup, all passes in shared memory.
template <int E>
__device__ __forceinline__ void sort_in_lds(int n, int passes, int bits, int tbits, uint32_t* count, uint32_t* base, uint32_t* tmp,
                                            uint32_t* entries) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bins = 1 << bits;
  uint32_t e[E], digit[E], rank[E];
  bool ok[E];
#pragma unroll
  for (int r = 0; r < E; ++r) ok[r] = (int)((wave * E + r) * 64 + lane) < n;
  for (int p = 0; p < passes; ++p) {
    for (int w = threadIdx.x >> bits; w < 16; w += 1024 >> bits) count[w * kDigits + (threadIdx.x & (bins - 1))] = 0;
#pragma unroll
    for (int r = 0; r < E; ++r) e[r] = entries[(wave * E + r) * 64 + lane];   // (entries past n: not used)
    __syncthreads();
#pragma unroll
    for (int r = 0; r < E; ++r) digit[r] = (e[r] >> (tbits + p * bits)) & (uint32_t)(bins - 1);
    wave_ranks<E>(digit, ok, bits, count + wave * kDigits, rank);
    __syncthreads();
    const uint32_t first = bin_scan(wave_prefixes(count, bins), bins, tmp);
    if ((int)threadIdx.x < bins) base[threadIdx.x] = first;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < E; ++r)
      if (ok[r]) entries[base[digit[r]] + count[wave * kDigits + digit[r]] + rank[r]] = e[r];
    __syncthreads();
  }
}

// The keys and tokens a pass starts from: the ids in their order (NULL), or what the
// pass before left.
struct SortInput {
  const uint32_t *key, *pos;
};
__device__ __forceinline__ uint32_t input_key(const EmbedArgs& a, const SortInput& in, int64_t t) { return in.key ? in.key[t] : key_at(a, t); }

// A workgroup takes a tile of 1024 E tokens, or, MANY, `tiles` consecutive ones: every
// scattering workgroup reads all workgroups' counts, so that there are kSortGroups of them
// at most, two to a CU, whatever the number of tokens (60M's vocabulary, rows of 64: 32 M
// tokens 2.9 ms, a tile to each of 4096 workgroups 4.9; 8 M 0.81 and 0.86; 4 M, of 512 tiles,
// 0.47 with the loop over them and 0.42 without).
constexpr int kSortGroups = 512;

// hist[workgroup][digit]
template <int E, bool MANY>
__global__ __launch_bounds__(1024) void embed_hist_kernel(const EmbedArgs a, SortInput in, int shift, int bits, int tiles, uint32_t* hist) {
  __shared__ uint32_t count[kDigits];
  const int bins = 1 << bits;
  if ((int)threadIdx.x < bins) count[threadIdx.x] = 0;
  __syncthreads();
  for (int tile = 0; tile < (MANY ? tiles : 1); ++tile) {
    const int64_t t0 = ((int64_t)blockIdx.x * (MANY ? tiles : 1) + tile) * (1024 * E);
#pragma unroll
    for (int r = 0; r < E; ++r) {
      const int64_t t = t0 + r * 1024 + threadIdx.x;
      if (t < a.T) atomicAdd(&count[(input_key(a, in, t) >> shift) & (uint32_t)(bins - 1)], 1u);
    }
  }
  __syncthreads();
  if ((int)threadIdx.x < bins) hist[(int64_t)blockIdx.x * bins + threadIdx.x] = count[threadIdx.x];
}

// (Counting the next pass's digits here, with atomics, instead of in a launch of their own
// was measured: 48 us instead of 10 + 5 at 65536 tokens, most of which share few digits.)
template <int E, bool MANY>
__global__ __launch_bounds__(1024, MANY ? 8 : 4) void embed_scatter_kernel(const EmbedArgs a, SortInput in, int shift, int bits, int tiles,
                                                                           const uint32_t* hist, uint32_t* key_out, uint32_t* pos_out) {
  __shared__ uint32_t count[16 * kDigits], base[kDigits], tmp[8];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bins = 1 << bits;
  uint32_t k[E], pos[E], digit[E], rank[E];
  bool ok[E];
  auto load = [&](int tile) __attribute__((always_inline)) {
    const int64_t t0 = ((int64_t)blockIdx.x * (MANY ? tiles : 1) + tile) * (1024 * E);
#pragma unroll
    for (int r = 0; r < E; ++r) {
      const int64_t t = t0 + (wave * E + r) * 64 + lane;
      ok[r] = t < a.T;
      k[r] = ok[r] ? input_key(a, in, t) : 0u;
      pos[r] = ok[r] && in.pos ? in.pos[t] : (uint32_t)t;
    }
  };
  if (!MANY) load(0);   // (in the loop otherwise: both would not leave room for two workgroups)
  for (int i = threadIdx.x; i < 16 * kDigits; i += 1024) count[i] = 0;
  // the digit's tokens in all workgroups and in those before this one
  uint32_t all = 0, before = 0;
  if ((int)threadIdx.x < bins) {
#pragma unroll 16
    for (uint32_t g = 0; g < gridDim.x; ++g) {
      const uint32_t n = hist[(int64_t)g * bins + threadIdx.x];
      all += n;
      before += g < blockIdx.x ? n : 0u;
    }
  }
  const uint32_t first = bin_scan(all, bins, tmp);   // (its barrier: the counters are cleared)
  if ((int)threadIdx.x < bins) base[threadIdx.x] = first + before;
  for (int tile = 0;;) {
    if (MANY) load(tile);
#pragma unroll
    for (int r = 0; r < E; ++r) digit[r] = (k[r] >> shift) & (uint32_t)(bins - 1);
    wave_ranks<E>(digit, ok, bits, count + wave * kDigits, rank);
    __syncthreads();
    const uint32_t n = wave_prefixes(count, bins);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < E; ++r) {
      if (!ok[r]) continue;
      const uint32_t at = base[digit[r]] + count[wave * kDigits + digit[r]] + rank[r];
      key_out[at] = k[r];
      pos_out[at] = pos[r];
    }
    if (!MANY || ++tile == tiles) break;
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * kDigits; i += 1024) count[i] = 0;
    if ((int)threadIdx.x < bins) base[threadIdx.x] += n;   // the next tile's lie behind this one's
    __syncthreads();
  }
}

// Up to kPlaced tokens the sort is one launch instead: a token's place is the number of
// keys below its own and of equal ones before it, counted against all of them.  A
// workgroup takes 32 tokens, and its 32 half waves a share of the keys each, so that the
// comparisons are spread over all the card.  (60M, all launches of the gradient, 8192 tokens
// 27.4 us, radix sort 33.7; 12000 tokens 42.5 and 37.1.  Keys in registers, 64 compared at
// once and the mask's bits counted: 39.5 at 8192, the scalar unit being shared.)
constexpr int kPlaced = 8192;
__global__ __launch_bounds__(1024) void embed_place_kernel(const EmbedArgs a, int share, uint32_t* key_out, uint32_t* pos_out) {
  extern __shared__ __attribute__((aligned(16))) uint32_t keys[];   // [32 share]; past the tokens: above all
  __shared__ uint32_t place[32];
  const int T = (int)a.T, block = (int)blockIdx.x * 32, mine = threadIdx.x & 31;
  if (threadIdx.x < 32) place[threadIdx.x] = 0;
  for (int t = threadIdx.x; t < 32 * share; t += 1024) keys[t] = t < T ? key_at(a, t) : ~0u;
  __syncthreads();
  const uint32_t key = keys[block + mine];
  const int first = (int)(threadIdx.x >> 5) * share;   // (a multiple of 32)
  uint32_t n = 0;
  for (int k = first; k < first + share; k += 32) {
    if (k == block) {
      for (int i = 0; i < 32; ++i) n += keys[k + i] < key || (keys[k + i] == key && i < mine);
      continue;
    }
    const uint32_t limit = key + (k < block);   // equal keys count where they come before
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      const uint4 o = *(const uint4*)(keys + k + i);
      n += (o.x < limit) + (o.y < limit) + (o.z < limit) + (o.w < limit);
    }
  }
  atomicAdd(&place[mine], n);
  __syncthreads();
  if (threadIdx.x >= 32 || block + mine >= T) return;
  key_out[place[mine]] = key;
  pos_out[place[mine]] = (uint32_t)(block + mine);
}

// ---- the sums -------------------------------------------------------------------------
// Overwriting, the sorted tokens and the table's rows form one sequence: token p lies at
// p + kRowWeight key[p], row v, whose end writes it, after its tokens.  It is cut into
// `chunks` of equal length, so that many tokens of one row, many rows of one token and
// long stretches of rows without tokens load the waves alike (a row's 4 bytes per
// feature written weigh as two tokens' 2 bytes read).  Where a cut falls into a row
// of up to 32 tokens, it is moved behind them.  Rows cut all the same
// are joined by embed_join_kernel: each chunk's sum over the row it leaves open goes to
// `carry`, and the chunk that ends the row writes its own part.
// Adding, only the tokens form the sequence.
constexpr int kRowWeight = 2;

// The sorted tokens: in memory, or in a workgroup's shared memory.
struct MemoryTokens {
  const uint32_t *keys, *positions;
  __device__ __forceinline__ uint32_t key(int64_t p) const { return keys[p]; }
  __device__ __forceinline__ uint32_t pos(int64_t p) const { return positions[p]; }
};
struct SharedTokens {
  const uint32_t* entries;
  int tbits;
  __device__ __forceinline__ uint32_t key(int64_t p) const { return entries[(int)p] >> tbits; }
  __device__ __forceinline__ uint32_t pos(int64_t p) const { return entries[(int)p] & ((1u << tbits) - 1); }
};

// The table's row behind a row's number: itself, or one of those of workgroup `group`
// among 2^bits, which has one of every 2^bits consecutive rows (another one each time, so
// that ids at equal distances do not meet in one workgroup).
struct AllRows {
  __device__ __forceinline__ int64_t operator()(uint32_t v) const { return v; }
};
struct GroupRows {
  uint32_t group;
  int bits;
  __device__ __forceinline__ uint32_t mask() const { return (1u << bits) - 1; }
  __device__ __forceinline__ int64_t operator()(uint32_t v) const { return (int64_t)v << bits | ((group ^ v ^ v >> bits) & mask()); }
  __device__ __forceinline__ bool has(uint32_t key) const { return ((key ^ key >> bits ^ key >> 2 * bits) & mask()) == group; }
  __device__ __forceinline__ uint32_t number(int64_t V) const { return (uint32_t)(V >> bits) + ((*this)((uint32_t)(V >> bits)) < V); }
};

struct SumArgs {
  int64_t chunk;               // length of a chunk
  int chunks, slices;          // slices of 512 features (few tokens: of a workgroup)
  float* carry;                // [chunks][d]
  uint32_t* carry_row;         // [chunks]; ~0: none
};

// First p in [0, T) from which on `holds` is true, else T; a wave probes 64 places at once.
template <class F>
__device__ __forceinline__ int64_t first_where(int64_t T, const F& holds) {
  const int lane = threadIdx.x & 63;
  int64_t lo = 0, hi = T;
  while (lo < hi) {
    const int64_t step = (hi - lo + 63) / 64;
    const int64_t p = min(lo + (lane + 1) * step, hi) - 1;   // the last of the lane's share
    const uint64_t m = __ballot(holds(p));
    if (m == 0) return hi;
    const int k = __ffsll((unsigned long long)m) - 1;
    lo += k * step;
    hi = min(lo + step, hi) - 1;
  }
  return lo;
}

struct Cut {
  int64_t p;      // first token
  uint32_t v;     // first row whose end lies behind the cut
  uint32_t mid;   // whether the cut is inside row v, with tokens of it on both sides
};
template <class Tokens>
__device__ __forceinline__ Cut cut_at(const EmbedArgs& a, const Tokens& tokens, int64_t at) {
  const int lane = threadIdx.x & 63;
  const int weight = a.add ? 0 : kRowWeight;
  const uint32_t V = (uint32_t)a.V;
  Cut c{};
  c.p = a.add ? min(at, a.T) : first_where(a.T, [&](int64_t p) { return p + (int64_t)weight * tokens.key(p) >= at; });
  // the keys of the 32 tokens before and the 32 from the cut on (outside: none of a token's)
  const int64_t q = c.p - 32 + lane;
  const uint32_t none = V + 1, k = q >= 0 && q < a.T ? tokens.key(q) : none;
  const uint32_t left = __builtin_amdgcn_readlane(k, 31), right = __builtin_amdgcn_readlane(k, 32);
  if (left == right && right < V) {
    // in the middle of a row.  Of one of 32 tokens or fewer both ends are seen from every
    // cut, so that all its cuts are moved; of a longer one all are, or none is.
    const uint64_t other = __ballot(k != right);
    const uint32_t below = (uint32_t)other, above = (uint32_t)(other >> 32);
    const int rest = __ffs(above) - 1;
    if (below != 0 && above != 0 && __clz(below) + rest <= 32) {
      c.p += rest;
      c.v = right + 1;
    } else {
      c.v = right;
      c.mid = 1;
    }
    return c;
  }
  // between rows: behind the row on the left, and as far into the rows without tokens as the cut lies
  const uint32_t lo = left < V ? left + 1 : left == none ? 0u : V, hi = right < V ? right : V;
  const int64_t in = weight ? (at - c.p + weight - 1) / weight : 0;
  c.v = (uint32_t)max((int64_t)lo, min((int64_t)hi, in));
  return c;
}

// A value that is the same in all lanes, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// A lane's features of a slice.
struct Columns {
  uint32_t c;
  bool there, there2;
  __device__ __forceinline__ Columns(const EmbedArgs& a, int slice) {
    c = (uint32_t)slice * 512 + (threadIdx.x & 63) * 4;
    there = c < (uint32_t)a.d;
    there2 = c + 256 < (uint32_t)a.d;
  }
};

// What a wave is left with behind its range: the sum over the row that the range's end
// cuts, and (HOLD, a range that begins inside a row) that over the rest of the row which
// it begins in.
struct Open {
  float acc[8] = {}, head[8] = {};
  uint32_t row;
  bool open = false;   // whether the row has tokens here
};

// Sums between two cuts, U tokens on their way at once.
template <class R, bool ADD, bool HOLD, int U, class Tokens, class Rows>
__device__ __forceinline__ Open sum_range(const EmbedArgs& a, const Tokens& tokens, const Rows& rows, const Cut& c0, const Cut& c1,
                                          const Columns& col) {
  const int lane = threadIdx.x & 63;
  const uint32_t V = (uint32_t)a.V;
  Open o;
  o.row = c0.v;
  auto store = [&](uint32_t v, const Piece<float, true>& old) __attribute__((always_inline)) {
    if (HOLD && c0.mid && v == c0.v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) o.head[i] = o.acc[i], o.acc[i] = 0.f;
      return;
    }
    float x[8];
    if (ADD) old.get(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = ADD ? fmaf(a.scale, o.acc[i], x[i]) : a.scale * o.acc[i], o.acc[i] = 0.f;
    Piece<float, true>::store<!ADD>((a.dtable + rows(v) * a.d) + col.c, x, col.there, col.there2);
  };
  const Piece<float, true> nothing = {};
  for (int64_t p = c0.p; p < c1.p; p += 64) {
    const int n = (int)min((int64_t)64, c1.p - p);
    const uint32_t k = lane < n ? tokens.key(p + lane) : V, pos = lane < n ? tokens.pos(p + lane) : 0u;
    const uint32_t after = ADD && lane < n && p + lane + 1 < a.T ? tokens.key(p + lane + 1) : V + 1;
    for (int j = 0; j < n; j += U) {
      Piece<R, true> x[U];
      Piece<float, true> old[ADD ? U : 1];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t ku = __builtin_amdgcn_readlane(k, j + u);   // (past n: V)
        const int64_t t = __builtin_amdgcn_readlane(pos, j + u);
        if (ku >= V) continue;
        x[u].load(((const R*)a.dx + t * a.d) + col.c, col.there, col.there2);
        if (ADD && __builtin_amdgcn_readlane(after, j + u) != ku)
          old[ADD ? u : 0].load((a.dtable + rows(ku) * a.d) + col.c, col.there, col.there2);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t ku = __builtin_amdgcn_readlane(k, j + u);
        if (ku >= V) continue;
        if (!ADD)
          for (; o.row < ku; ++o.row, o.open = false) store(o.row, nothing);
        float v[8];
        x[u].get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) o.acc[i] += v[i];
        o.row = ku;
        o.open = true;
        if (ADD && __builtin_amdgcn_readlane(after, j + u) != ku) {
          store(ku, old[ADD ? u : 0]);
          o.open = false;
        }
      }
    }
  }
  if (!ADD)
    for (; o.row < c1.v; ++o.row, o.open = false) store(o.row, nothing);
  return o;
}

__device__ __forceinline__ Cut uniform(const Cut& c) { return {uniform(c.p), (uint32_t)uniform(c.v), (uint32_t)uniform(c.mid)}; }

// One task (a chunk and a slice) to a wave.
template <class R, bool ADD>
__global__ __launch_bounds__(256) void embed_sum_kernel(const EmbedArgs a, const SumArgs s, const MemoryTokens tokens) {
  __shared__ Cut cuts[5];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // the 4 tasks lie in at most 4 chunks: their cuts, one to a wave
  const int64_t task0 = (int64_t)blockIdx.x * 4, chunk0 = task0 / s.slices, last = (task0 + 3) / s.slices + 1;
  for (int i = wave; chunk0 + i <= last; i += 4) {
    const Cut c = cut_at(a, tokens, (chunk0 + i) * s.chunk);
    if (lane == 0) cuts[i] = c;
  }
  __syncthreads();
  const int64_t task = task0 + wave, chunk = task / s.slices;
  if (chunk >= s.chunks) return;
  const int slice = (int)(task - chunk * s.slices), i = (int)(chunk - chunk0);
  const Columns col(a, slice);
  Open o = sum_range<R, ADD, false, ADD ? 4 : sizeof(R) == 2 ? 16 : 8>(a, tokens, AllRows{}, uniform(cuts[i]), uniform(cuts[i + 1]), col);
  if (o.open) {
#pragma unroll
    for (int k = 0; k < 8; ++k) o.acc[k] *= a.scale;
    Piece<float, true>::store<false>((s.carry + chunk * a.d) + col.c, o.acc, col.there, col.there2);
  }
  if (slice == 0 && lane == 0) s.carry_row[chunk] = o.open ? o.row : ~0u;
}

// Few tokens: a workgroup has one of every 2^gbits rows, looks through all ids for theirs,
// sorts those in shared memory, and walks them and its rows with its 16 waves: the slices
// (s.slices of them, 16 at most) of 16 / s.slices equal shares each.  Rows cut between
// shares are joined in shared memory, so that one launch does it all: the wave that ends
// such a row holds its own part, and adds those of the shares before it in their order.
// (60M, 2048 tokens, added: 11.0 us; where every workgroup sorts all tokens for itself
// 16.5, with the sort a launch of its own 23.)
constexpr int kRanked = 512;   // entries, up to which a place is found by comparing with all
template <class R, bool ADD, int E>
__global__ __launch_bounds__(1024) void embed_few_kernel(const EmbedArgs a, const SumArgs s, int gbits, int passes, int bits, int tbits) {
  __shared__ __attribute__((aligned(16))) uint32_t count[16 * kDigits], entries[1024 * E + 4];
  __shared__ uint32_t base[kDigits], tmp[16];
  __shared__ Cut cuts[17];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const GroupRows rows{blockIdx.x, gbits};
  uint32_t e[E];
  uint64_t mine[E];
  int found = 0;
#pragma unroll
  for (int r = 0; r < E; ++r) {
    const int64_t t = (wave * E + r) * 64 + lane;
    const uint32_t key = t < a.T ? key_at(a, t) : (uint32_t)a.V;
    mine[r] = __ballot(key < (uint32_t)a.V && rows.has(key));
    e[r] = key >> gbits << tbits | (uint32_t)t;
    found += __popcll(mine[r]);
  }
  if (lane == 0) tmp[wave] = (uint32_t)found;
  __syncthreads();
  int at = 0, n = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    at += w < wave ? (int)tmp[w] : 0;
    n += (int)tmp[w];
  }
  n = __builtin_amdgcn_readfirstlane(n);
  if (ADD && n == 0) return;
#pragma unroll
  for (int r = 0; r < E; ++r) {
    if (mine[r] >> lane & 1)
      entries[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(mine[r] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mine[r], 0u))] = e[r];
    at += __popcll(mine[r]);
  }
  if (threadIdx.x < 4) entries[n + threadIdx.x] = ~0u;
  __syncthreads();
  if (n <= kRanked) {
    // each entry's place: the number of those below it
    uint32_t own = 0, place = 0;
    if (wave * 64 < n) {
      own = entries[threadIdx.x];
#pragma unroll 4
      for (int k = 0; k < n; k += 4) {
        const uint4 o = *(const uint4*)(entries + k);
        place += (o.x < own) + (o.y < own) + (o.z < own) + (o.w < own);
      }
    }
    __syncthreads();
    if ((int)threadIdx.x < n) entries[place] = own;
    __syncthreads();
  } else {
    sort_in_lds<E>(n, passes, bits, tbits, count, base, tmp, entries);
  }
  EmbedArgs here = a;   // the workgroup's own tokens and rows
  here.T = n;
  here.V = rows.number(a.V);
  const SharedTokens tokens{entries, tbits};
  const int shares = 16 / s.slices, share = wave / s.slices;
  const bool works = share < shares;   // (16 may not be a multiple of the slices)
  if (wave < shares) {
    Cut c{};
    if (wave > 0) c = cut_at(here, tokens, (here.T + (ADD ? 0 : kRowWeight) * here.V) * wave / shares);
    if (lane == 0) cuts[wave] = c;
  }
  if (threadIdx.x == 0) cuts[shares] = {here.T, (uint32_t)here.V, 0};
  __syncthreads();
  const Columns col(a, (int)blockIdx.y * s.slices + wave - share * s.slices);
  Open o;
  Cut c0{}, c1{};
  if (works) {
    c0 = uniform(cuts[share]), c1 = uniform(cuts[share + 1]);
    o = sum_range<R, ADD, true, ADD ? 4 : 8>(here, tokens, rows, c0, c1, col);
  }
  float(*carry)[512] = (float(*)[512])count;   // (the counters are free)
  const int l = lane * 4;
  if (c1.mid) Piece<float, true>::store<false>(carry[wave] + l, o.acc, true, true);
  __syncthreads();
  // on with the wave that ends the row its range began in: c1 is not inside the same row
  if (!c0.mid || (c1.mid && c1.v == c0.v)) return;
  int i = share - 1;   // the first share with a part of the row
  while (cuts[i].mid && cuts[i].v == c0.v) --i;
  float sum[8] = {};
  for (; i < share; ++i) {
    Piece<float, true> x;
    float v[8];
    x.load(carry[wave - (share - i) * s.slices] + l, true, true);
    x.get(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] += v[k];
  }
  float* out = (a.dtable + rows(c0.v) * a.d) + col.c;
  Piece<float, true> old;
  old.load(out, ADD && col.there, ADD && col.there2);
  float x[8];
  old.get(x);
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = fmaf(a.scale, sum[k] + o.head[k], x[k]);
  Piece<float, true>::store<!ADD>(out, x, col.there, col.there2);
}

// Adds the sums of the chunks that left a row open, in their order, to the row.  A
// workgroup looks after the runs of such chunks that begin at one of kJoinChunks, for
// 256 columns; its kJoinShares waves take an equal share of a run each.  Most chunks leave
// no row open, and what counts is how few waves are launched to find that: 1B, 65536 tokens,
// all launches of the gradient 133.0 us, 134.2 with a chunk to a workgroup, 136.4 with 8 (whose
// runs are then joined one after the other), 134.8 with 8 waves; 60M 49.3, 50.1, 49.0, 49.3.
constexpr int kJoinChunks = 4, kJoinShares = 4;
__global__ __launch_bounds__(64 * kJoinShares) void embed_join_kernel(const EmbedArgs a, const SumArgs s) {
  __shared__ float4 red[2][kJoinShares][64];
  const int lane = threadIdx.x & 63, share = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = blockIdx.x * kJoinChunks;
  // rows of the chunk before, of these and of the next
  const int q0 = first - 1 + lane;
  const uint32_t near = q0 >= 0 && q0 < s.chunks ? s.carry_row[q0] : ~0u;
  const uint32_t before = __shfl_up(near, 1);
  uint64_t heads = __ballot(near != ~0u && near != before) & ((1ull << kJoinChunks) - 1) << 1;
  const int64_t c = (int64_t)blockIdx.y * 256 + lane * 4;
  const bool there = c < a.d;
  for (int turn = 0; heads; turn ^= 1, heads &= heads - 1) {
    const int at = __ffsll((unsigned long long)heads) - 1, c0 = first - 1 + at;
    const uint32_t row = __builtin_amdgcn_readlane(near, at);
    uint64_t other = __ballot(near != row) >> at << at;
    int end = first - 1;   // behind the run's last chunk
    while (other == 0) {
      end += 64;
      other = __ballot(!(end + lane < s.chunks && s.carry_row[end + lane] == row));
    }
    end += __ffsll((unsigned long long)other) - 1;
    const int n = end - c0;
    const int b = c0 + (int)((int64_t)n * share / kJoinShares), e = c0 + (int)((int64_t)n * (share + 1) / kJoinShares);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f), *out = (float4*)(a.dtable + (int64_t)row * a.d + c);
    const float4 o = there && share == 0 ? *out : x;
    if (there) {
#pragma unroll 8
      for (int k = b; k < e; ++k) {
        const float4 y = *(const float4*)(s.carry + (int64_t)k * a.d + c);
        x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
      }
    }
    red[turn][share][lane] = x;
    __syncthreads();   // (two buffers: the next turn's writes do not meet this one's reads)
    if (share > 0 || !there) continue;
#pragma unroll
    for (int q = 1; q < kJoinShares; ++q) {
      const float4 y = red[turn][q][lane];
      x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
    }
    *out = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
  }
}

// ---- host -----------------------------------------------------------------------------

int bit_length(int64_t v) {
  int n = 0;
  for (; v > 0; v >>= 1) ++n;
  return n;
}

// Sort and cuts of one call, and its regions of the workspace.
struct Plan {
  int passes, bits, tbits;
  bool few;            // one launch, embed_few_kernel
  int per_thread;      // tokens of a thread in a tile
  int tiles;           // of a workgroup
  int gbits;           // few: 2^gbits workgroups to a slice group
  int groups;
  int slice_groups;    // few: of sum.slices each
  SumArgs sum;
  uint32_t *key[2], *pos[2], *hist;
  size_t bytes;
};
Plan plan(void* ws, int64_t T, int64_t V, int64_t d, bool add) {
  Plan p{};
  const int key_bits = bit_length(V);   // keys 0 .. V
  p.passes = (key_bits + 8) / 9;
  p.bits = (key_bits + p.passes - 1) / p.passes;
  p.tbits = std::max(1, bit_length(T - 1));
  p.sum.slices = (int)cdiv(d, 512);
  // Few tokens, added: a slice to a workgroup, about 16 tokens to each (1B, 2048 tokens: with
  // 64 the same, 17.2 us; 60M 11.0 and 11.9), all of them on the card at once (1B 17 and 29).
  // Written: all slices of a row in one (1B, 4096 tokens: 50 us, one slice 67), and a workgroup
  // for every 32768 values of the table, so that those with the long rows have little else to
  // do and the others go on (1B 50, with twice the rows 53, with 8 times 72; 60M 20.2, with
  // half the rows 25.2, with twice 23.3), or as many as adding has, if those are more (256
  // rows of 64, 4096 tokens: 10.9 us, in one workgroup 82).
  p.slice_groups = add ? p.sum.slices : (int)cdiv(p.sum.slices, 16);
  const int by_tokens = std::max(0, std::min(8 - bit_length(p.slice_groups - 1), bit_length(T / 16)));
  p.gbits = add ? by_tokens : std::min(12, std::max(by_tokens, bit_length(V * d / 32768)));
  const int few_bits = bit_length((V - 1) >> p.gbits);   // of a row's number in its workgroup
  p.few = T <= 4096 && few_bits + p.tbits <= 32;
  if (p.few) {
    p.passes = (few_bits + 8) / 9;
    p.bits = p.passes ? (few_bits + p.passes - 1) / p.passes : 0;
    p.per_thread = T <= 1024 ? 1 : T <= 2048 ? 2 : 4;
    p.sum.slices = (int)cdiv(p.sum.slices, p.slice_groups);
    return p;
  }
  p.per_thread = T <= 131072 ? 1 : T <= (1 << 18) ? 4 : 8;
  const int64_t tiles = cdiv(T, 1024 * p.per_thread);
  p.tiles = (int)cdiv(tiles, kSortGroups);   // (up to 2^18 tokens there are fewer than that)
  p.groups = (int)cdiv(tiles, p.tiles);
  // about 8 waves to a SIMD (1B, 65536 tokens: 133 us, 4 waves 139; 60M 49.3 and 46.6), and
  // not under a few tokens or rows to each
  const int64_t length = add ? T : T + kRowWeight * V;
  p.sum.chunk = std::max<int64_t>(add ? 4 : 16, cdiv(length * p.sum.slices, 8192));
  p.sum.chunks = (int)std::max<int64_t>(1, cdiv(length, p.sum.chunk));
  size_t used = 0;
  auto take = [&](size_t n) {
    uint32_t* r = ws ? (uint32_t*)((char*)ws + used) : nullptr;
    used += (n * sizeof(uint32_t) + 255) / 256 * 256;
    return r;
  };
  for (int i = 0; i < (p.passes == 1 ? 1 : 2); ++i) {
    p.key[i] = take((size_t)T);
    p.pos[i] = take((size_t)T);
  }
  p.hist = take((size_t)p.groups << p.bits);
  p.sum.carry_row = take((size_t)p.sum.chunks);
  p.sum.carry = (float*)take((size_t)(p.sum.chunks * d));
  p.bytes = used;
  return p;
}

template <int E, bool MANY = false>
hipError_t sort_passes(const EmbedArgs& a, const Plan& p, int& at, hipStream_t stream) {
  const dim3 grid((unsigned)p.groups), block(1024);
  for (int k = 0; k < p.passes; ++k) {
    const int to = p.passes == 1 ? 0 : k & 1;
    const SortInput in = k == 0 ? SortInput{nullptr, nullptr} : SortInput{p.key[1 - to], p.pos[1 - to]};
    {
      TimedLaunch tl("embed_bwd_sort", stream);
      hipLaunchKernelGGL((embed_hist_kernel<E, MANY>), grid, block, 0, stream, a, in, k * p.bits, p.bits, p.tiles, p.hist);
    }
    TimedLaunch tl("embed_bwd_sort", stream);
    hipLaunchKernelGGL((embed_scatter_kernel<E, MANY>), grid, block, 0, stream, a, in, k * p.bits, p.bits, p.tiles, (const uint32_t*)p.hist,
                       p.key[to], p.pos[to]);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    at = to;
  }
  return hipSuccess;
}

hipError_t place(const EmbedArgs& a, const Plan& p, hipStream_t stream) {
  TimedLaunch tl("embed_bwd_sort", stream);
  const int share = (int)cdiv(a.T, 1024) * 32;   // of a half wave
  hipLaunchKernelGGL(embed_place_kernel, dim3((unsigned)cdiv(a.T, 32)), dim3(1024), 32 * share * sizeof(uint32_t), stream, a, share, p.key[0],
                     p.pos[0]);
  return hipGetLastError();
}

template <class R, bool STREAM>
void launch_fwd(const EmbedArgs& a, uint32_t parts, unsigned grid, hipStream_t stream) {
  hipLaunchKernelGGL((embed_fwd_kernel<R, STREAM>), dim3(grid), dim3(256), 0, stream, a, parts);
}

template <class R>
void launch_sum(const EmbedArgs& a, const SumArgs& s, const MemoryTokens& tokens, hipStream_t stream) {
  const dim3 grid((unsigned)cdiv((int64_t)s.chunks * s.slices, 4));
  if (a.add)
    hipLaunchKernelGGL((embed_sum_kernel<R, true>), grid, dim3(256), 0, stream, a, s, tokens);
  else
    hipLaunchKernelGGL((embed_sum_kernel<R, false>), grid, dim3(256), 0, stream, a, s, tokens);
}

template <class R, int E>
void launch_few(const EmbedArgs& a, const Plan& p, hipStream_t stream) {
  const dim3 grid(1u << p.gbits, (unsigned)p.slice_groups);
  if (a.add)
    hipLaunchKernelGGL((embed_few_kernel<R, true, E>), grid, dim3(1024), 0, stream, a, p.sum, p.gbits, p.passes, p.bits, p.tbits);
  else
    hipLaunchKernelGGL((embed_few_kernel<R, false, E>), grid, dim3(1024), 0, stream, a, p.sum, p.gbits, p.passes, p.bits, p.tbits);
}

}  // namespace

size_t embed_bwd_workspace_bytes(int64_t T, int64_t V, int64_t d, bool add) { return plan(nullptr, T, V, d, add).bytes; }

hipError_t run_embed_fwd(const EmbedArgs& a, hipStream_t stream) {
  TimedLaunch tl("embed_fwd", stream);
  const uint32_t parts = (uint32_t)cdiv(a.d, 512);
  const unsigned grid = (unsigned)std::min<int64_t>(cdiv(a.T * parts, 16), 1 << 20);
  if (a.T * a.d < kStreamStores)
    a.res_f32 ? launch_fwd<float, false>(a, parts, grid, stream) : launch_fwd<uint16_t, false>(a, parts, grid, stream);
  else
    a.res_f32 ? launch_fwd<float, true>(a, parts, grid, stream) : launch_fwd<uint16_t, true>(a, parts, grid, stream);
  return hipGetLastError();
}

hipError_t run_embed_bwd(const EmbedArgs& a, hipStream_t stream) {
  const Plan p = plan(a.ws, a.T, a.V, a.d, a.add);
  int at = 0;
  if (!p.few) {
    const hipError_t e = a.T <= kPlaced      ? place(a, p, stream)
                         : p.per_thread == 1 ? sort_passes<1>(a, p, at, stream)
                         : p.per_thread == 4 ? sort_passes<4>(a, p, at, stream)
                         : p.tiles == 1      ? sort_passes<8>(a, p, at, stream)
                                             : sort_passes<8, true>(a, p, at, stream);
    if (e != hipSuccess) return e;
  }
  {
    TimedLaunch tl("embed_bwd_sum", stream);
    const MemoryTokens tokens{p.key[at], p.pos[at]};
    if (!p.few)
      a.res_f32 ? launch_sum<float>(a, p.sum, tokens, stream) : launch_sum<uint16_t>(a, p.sum, tokens, stream);
    else if (p.per_thread == 1)
      a.res_f32 ? launch_few<float, 1>(a, p, stream) : launch_few<uint16_t, 1>(a, p, stream);
    else if (p.per_thread == 2)
      a.res_f32 ? launch_few<float, 2>(a, p, stream) : launch_few<uint16_t, 2>(a, p, stream);
    else
      a.res_f32 ? launch_few<float, 4>(a, p, stream) : launch_few<uint16_t, 4>(a, p, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.few) return hipSuccess;
  TimedLaunch tl("embed_bwd_join", stream);
  hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)cdiv(p.sum.chunks, kJoinChunks), (unsigned)cdiv(a.d, 256)), dim3(64 * kJoinShares),
                     0, stream, a, p.sum);
  return hipGetLastError();
}

}  // namespace elas
