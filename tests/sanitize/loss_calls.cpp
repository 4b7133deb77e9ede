// Which calls of include/elas_loss.h and include/elas_adamw.h reach their launch sequences, which are
// replaced here (tests/test_loss_calls.py): those whose results overlap nothing.  No device is used.
#include <stdio.h>

#include <vector>

#include "elas_adamw.h"
#include "elas_loss.h"
#include "../../paper_2605_03667_amd/csrc/internal.h"

namespace elas {

static int g_calls = 0;

void begin_call() {}
int fail(int code, const char*, ...) { return code; }
int check_ptr(const void* p, const char*) { return !p ? ELAS_ERR_NULL : ((uintptr_t)p & 15) ? ELAS_ERR_ALIGN : ELAS_OK; }
int device_status(hipError_t e, const char*) { return e == hipSuccess ? ELAS_OK : ELAS_ERR_DEVICE; }
size_t token_loss_workspace_bytes(int64_t, int64_t, bool) { return 64; }
size_t preference_workspace_bytes(int64_t, int64_t) { return 64; }
size_t adamw_workspace_bytes() { return 48; }
hipError_t run_token_loss(const LogitsArgs&, hipStream_t) { return ++g_calls, hipSuccess; }
hipError_t run_token_logp_bwd(const LogitsArgs&, hipStream_t) { return ++g_calls, hipSuccess; }
hipError_t run_preference(const PreferenceArgs&, hipStream_t) { return ++g_calls, hipSuccess; }
hipError_t run_adamw(const AdamwArgs&, hipStream_t) { return ++g_calls, hipSuccess; }
hipError_t run_adam8_values(const uint8_t*, const float*, int64_t, bool, bool, void*, hipStream_t) { return ++g_calls, hipSuccess; }

}  // namespace elas

static int g_fail = 0;
static void expect(bool ok, int line, const char* what, long a = 0, long b = 0) {
  if (!ok) fprintf(stderr, "FAIL line %d: %s (%ld, %ld)\n", line, what, a, b), ++g_fail;
}
// A call that is taken reaches its launch sequence, one that is refused does not.
template <class F>
static void expect_call(F call, bool taken, int line, const char* what, long a = 0, long b = 0) {
  const int before = elas::g_calls, status = call();
  expect(taken ? status == ELAS_OK && elas::g_calls == before + 1 : status == ELAS_ERR_OVERLAP && elas::g_calls == before, line, what, a, b);
}
#define TAKEN(...) expect_call([&] { return __VA_ARGS__; }, true, __LINE__, #__VA_ARGS__)
#define REFUSED(...) expect_call([&] { return __VA_ARGS__; }, false, __LINE__, #__VA_ARGS__)

// Addresses of a call's buffers, far from one another; never dereferenced.
struct Buffers {
  std::vector<char*> at;
  explicit Buffers(int n) {
    for (int k = 0; k < n; ++k) at.push_back((char*)0x1000000 + 0x100000 * k);
  }
  template <class T>
  T* get(int k) const { return (T*)at[k]; }
};

// Moves every result over every other buffer: onto its first byte, its last ones, and its own last ones onto the other's
// first.  `bytes` of the buffers, the first `results` of them written, steps of `step` bytes; `same`: a buffer that result
// `may` may lie over, byte for byte.
template <class F>
static void every_pair(F call, const std::vector<long>& bytes, int results, long step, int may, int same, int line) {
  const int n = (int)bytes.size();
  auto align = [&](long v) { return v / step * step; };
  Buffers plain(n);
  expect_call([&] { return call(plain); }, true, line, "as it should be");
  for (int i = 0; i < results; ++i)
    for (int k = 0; k < n; ++k) {
      if (i == k) continue;
      for (long off : {0L, align(bytes[k] - 1), -align(bytes[i] - 1)}) {
        if (off == 0 && i == may && k == same) continue;
        Buffers b(n);
        b.at[i] = b.at[k] + off;
        expect_call([&] { return call(b); }, false, line, "over another", i * 100 + k, off);
      }
      for (long off : {(bytes[k] + step - 1) / step * step, -((bytes[i] + step - 1) / step * step)}) {
        Buffers b(n);
        b.at[i] = b.at[k] + off;
        expect_call([&] { return call(b); }, true, line, "beside another", i * 100 + k, off);
      }
    }
}

int main() {
  constexpr int64_t T = 40, V = 24;
  constexpr long X = T * V * 2, R = T * 4;      // bytes of rows without a gap, of a value for each token
  const auto every = [&](auto call, std::vector<long> bytes, int results, long step, int may, int same, int line) {
    every_pair(call, bytes, results, step, may, same, line);
  };
  // (steps of 16 bytes, which suits every buffer)
  every([&](const Buffers& b) {
    return elas_token_logp_fwd(b.get<void>(2), V, b.get<void>(3), T, V, 1.f, 0, b.get<float>(0), b.get<float>(1), nullptr);
  }, {R, R, X, R}, 2, 16, -1, -1, __LINE__);
  every([&](const Buffers& b) {
    return elas_token_logp_bwd(b.get<float>(3), b.get<float>(4), b.get<void>(1), V, b.get<void>(2), b.get<float>(5), T, V, 1.f, ELAS_IDS_I64,
                               b.get<void>(0), V, nullptr);
  }, {X, X, 2 * R, R, R, R}, 1, 16, 0, 1, __LINE__);
  every([&](const Buffers& b) {
    return elas_token_loss(b.get<void>(5), V, b.get<void>(6), b.get<float>(7), T, V, 1.f, 1.f, 0.f, 0, b.get<float>(0), b.get<float>(1),
                           b.get<void>(2), V, b.get<float>(3), b.get<void>(4), 64, nullptr);
  }, {R, R, X, 8, 64, X, R, R}, 5, 16, 2, 5, __LINE__);
  every([&](const Buffers& b) {
    return elas_policy_loss(b.get<void>(4), V, b.get<void>(5), b.get<float>(6), b.get<float>(7), b.get<float>(8), b.get<float>(9), T, V, 1.f, 1.f,
                            .2f, .2f, .1f, ELAS_LOGITS_F32, b.get<float>(0), b.get<void>(1), V, b.get<float>(2), b.get<void>(3), 64, nullptr);
  }, {R, 2 * X, 12, 64, 2 * X, R, R, R, R, R}, 4, 16, 1, 4, __LINE__);
  constexpr int64_t N = 1000, P = 30;
  every([&](const Buffers& b) {
    return elas_preference_loss(b.get<float>(4), b.get<float>(5), b.get<void>(6), N, P, .1f, 0.f, ELAS_IDS_I64, b.get<float>(0), b.get<float>(1),
                                b.get<float>(2), b.get<void>(3), 64, nullptr);
  }, {4 * P, 4 * N, 12, 64, 4 * N, 4 * N, 8 * (2 * P + 1)}, 4, 16, 1, 4, __LINE__);
  every([&](const Buffers& b) { return elas_adam8_values(b.get<uint8_t>(1), b.get<float>(2), 3, 0, b.get<void>(0), nullptr); },
        {3 * 512, 3 * 256, 12}, 1, 16, -1, -1, __LINE__);

  // AdamW: the state, two parameters and a copy are written; two gradients, norm and rate factor are read.  (Tensors among
  // themselves are the caller's to keep apart.)
  for (int bits : {8, 32}) {
    const long moments = 4 * 256 * bits / 8;       // (600 and 200 values: 3 blocks and 1)
    const std::vector<long> bytes = {moments, moments, 16, 16, 8, 48, 2400, 800, 400, 2400, 800, 4, 4};
    const auto call = [&](const Buffers& b) {
      void* p[] = {b.at[6], b.at[7], (void*)1};
      const void* g[] = {b.at[9], b.at[10], (void*)1};
      uint16_t* c[] = {nullptr, b.get<uint16_t>(8), (uint16_t*)1};
      const int64_t n[] = {600, 200, 0};
      const int32_t t[] = {0, 0, 1};
      const float w[] = {0.f, 0.f, 0.f};
      float *ms = bits == 8 ? b.get<float>(2) : nullptr, *vs = bits == 8 ? b.get<float>(3) : nullptr;
      return elas_adamw_step(p, g, c, n, t, t, w, 3, bits, b.at[0], ms, b.at[1], vs, b.get<int64_t>(4), 1e-3, b.get<float>(12), 0.9, 0.99, 1e-8,
                             b.get<float>(11), 1.0, b.at[5], 48, nullptr);
    };
    expect_call([&] { return call(Buffers(13)); }, true, __LINE__, "as it should be");
    const auto scale = [&](int k) { return bits == 32 && (k == 2 || k == 3); };
    const auto tensor = [](int k) { return k >= 6 && k <= 10; };
    const auto read = [](int k) { return k >= 9; };
    for (int i = 0; i < 13; ++i)
      for (int k = 0; k < 13; ++k) {
        if (i == k || scale(i) || scale(k) || (tensor(i) && tensor(k))) continue;
        const bool fine = read(i) && read(k);
        for (long off : {0L, (bytes[k] - 1) / 16 * 16, -((bytes[i] - 1) / 16 * 16)}) {
          Buffers b(13);
          b.at[i] = b.at[k] + off;
          expect_call([&] { return call(b); }, fine, __LINE__, "over another", i * 100 + k, off);
        }
        for (long off : {(bytes[k] + 15) / 16 * 16, -((bytes[i] + 15) / 16 * 16)}) {
          Buffers b(13);
          b.at[i] = b.at[k] + off;
          expect_call([&] { return call(b); }, true, __LINE__, "beside another", i * 100 + k, off);
        }
      }
  }

  // what is not given or empty overlaps nothing
  char *A = (char*)0x1000000, *B = (char*)0x2000000, *C = (char*)0x3000000;
  float* f = (float*)C;
  TAKEN(elas_token_loss(A, V, B, nullptr, T, V, 1.f, 1.f, 0.f, 0, nullptr, nullptr, nullptr, 0, f, C + 64, 64, nullptr));
  TAKEN(elas_token_loss(A, V, A, f, 0, V, 1.f, 1.f, 0.f, 0, f, f, A, V, f, C + 64, 64, nullptr));
  REFUSED(elas_token_loss(A, V, A, f, 0, V, 1.f, 1.f, 0.f, 0, f, f, A, V, f, C, 64, nullptr));
  TAKEN(elas_preference_loss(f, f, f, 0, 0, .1f, 0.f, 0, f, f, f, C + 64, 64, nullptr));
  // results and operands in the gaps of a pitch, and columns beside one another
  TAKEN(elas_token_logp_bwd((float*)(C), nullptr, A, 64, B, (float*)(C + 256), T, V, 1.f, 0, A + 2 * V, 64, nullptr));
  TAKEN(elas_token_logp_bwd((float*)(C), nullptr, A + 2 * V, 64, B, (float*)(C + 256), T, V, 1.f, 0, A, 64, nullptr));
  REFUSED(elas_token_logp_bwd((float*)(C), nullptr, A, 64, B, (float*)(C + 256), T, V, 1.f, 0, A + 2 * V - 2, 64, nullptr));
  REFUSED(elas_token_logp_bwd((float*)(C), nullptr, A, 64, B, (float*)(C + 256), T, V, 1.f, 0, A + 128 - 2, 64, nullptr));
  REFUSED(elas_token_logp_bwd((float*)(C), nullptr, A, 64, B, (float*)(C + 256), T, V, 1.f, 0, A + 2 * V, 48, nullptr));
  for (long gap : {0L, 5L * 512, 39L * 512}) {
    TAKEN(elas_token_logp_fwd(A, 256, B, T, V, 1.f, 0, (float*)(A + gap + 2 * V), nullptr, nullptr));
    TAKEN(elas_token_logp_fwd(A, 256, B, T, V, 1.f, 0, (float*)(A + gap + 512 - 4 * T), nullptr, nullptr));
    REFUSED(elas_token_logp_fwd(A, 256, B, T, V, 1.f, 0, (float*)(A + gap + 2 * V - 4), nullptr, nullptr));
    if (gap < 39 * 512) REFUSED(elas_token_logp_fwd(A, 256, B, T, V, 1.f, 0, (float*)(A + gap + 512 - 4 * T + 4), nullptr, nullptr));
  }
  // the largest rows end beyond the address space
  const int64_t big = int64_t(1) << 31;
  REFUSED(elas_token_logp_fwd(A, big, (void*)(uintptr_t(1) << 62), (1 << 24), V, 1.f, ELAS_LOGITS_F32, (float*)(A + 4), nullptr, nullptr));
  REFUSED(elas_token_logp_fwd(A, big, (void*)(uintptr_t(1) << 50), big - 1, 1 << 30, 1.f, ELAS_LOGITS_F32, (float*)B, nullptr, nullptr));

  printf("loss calls: %d failures\n", g_fail);
  return g_fail != 0;
}
