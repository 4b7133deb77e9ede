// Host-side exercise of include/elas_loss.h and include/elas_adamw.h for AddressSanitizer /
// UndefinedBehaviorSanitizer builds (tests/test_loss_sanitizers.py): argument checks and workspace
// planning.  No call may reach a kernel launch: every launching call here has an invalid argument or
// nothing to do.
#include <math.h>
#include <stdio.h>

#include <vector>

#include "elas_adamw.h"
#include "elas_loss.h"

static int g_fail = 0;
#define EXPECT(cond)                                                                  \
  do {                                                                                \
    if (!(cond)) {                                                                    \
      fprintf(stderr, "FAIL line %d: %s (%s)\n", __LINE__, #cond, elas_last_error()); \
      ++g_fail;                                                                       \
    }                                                                                 \
  } while (0)

int main() {
  void* A = (void*)0x10000;   // aligned, never dereferenced
  float* f = (float*)A;
  const int64_t big = INT64_MAX;

  // logits: sizes and pitches whose products leave the range of integers are refused before they are formed
  for (int64_t bad : {big, INT64_MIN, int64_t(-1), int64_t(1) << 31}) {
    EXPECT(elas_token_logp_fwd(A, 16, A, bad, 10, 1.f, 0, f, f, nullptr) == ELAS_ERR_SHAPE);
    EXPECT(elas_token_logp_fwd(A, 16, A, 4, bad, 1.f, 0, f, f, nullptr) == ELAS_ERR_SHAPE);
    EXPECT(elas_token_logp_bwd(f, f, A, 16, A, f, 4, 10, 1.f, 0, (char*)A + 64, bad == int64_t(1) << 31 ? big : bad, nullptr) == ELAS_ERR_SHAPE);
    EXPECT(elas_token_loss_workspace_bytes(bad, 10, 0) == 0 && elas_token_loss_workspace_bytes(4, bad, 0) == 0);
  }
  EXPECT(elas_token_logp_fwd(A, big, A, 4, 10, 1.f, 0, f, f, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_token_loss(A, 16, A, f, 4, 10, 1.f, 1.f, 0.f, 0, f, f, nullptr, 0, f, A, 0, nullptr) == ELAS_ERR_WORKSPACE);
  EXPECT(elas_token_loss(A, 16, A, f, 4, 10, 1.f, 1.f, 0.f, 0, f, f, A, 17, f, A, 1 << 20, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_policy_loss(A, 16, A, f, f, nullptr, f, 4, 10, 1.f, 1.f, .2f, .2f, .1f, 0, f, nullptr, 0, f, A, 1 << 20, nullptr) == ELAS_ERR_NULL);
  EXPECT(elas_policy_loss(A, 16, A, f, f, f, f, 4, 10, 1.f, 1.f, NAN, .2f, .1f, 0, f, nullptr, 0, f, A, 1 << 20, nullptr) == ELAS_ERR_SHAPE);
  for (int64_t T : {int64_t(1), int64_t(2047), int64_t(2049), (int64_t(1) << 31) - 1})
    for (int64_t V : {int64_t(1), int64_t(32000), int64_t(1) << 30})
      for (uint32_t flags : {0u, ELAS_LOGITS_F32}) {
        const size_t n = elas_token_loss_workspace_bytes(T, V, flags);
        EXPECT(n > 0 && n < (size_t)1 << 24);
      }
  EXPECT(elas_preference_loss(f, f, A, 10, big, .1f, 0.f, 0, f, f, f, A, 1 << 20, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_preference_loss(f, f, A, big, 4, .1f, 0.f, 0, f, f, f, A, 1 << 20, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_preference_loss(f, f, A, 100000, 4, .1f, 0.f, 0, f, f, f, A, 0, nullptr) == ELAS_ERR_WORKSPACE);

  // AdamW
  std::vector<void*> p(5, A);
  std::vector<const void*> g(5, A);
  std::vector<uint16_t*> c(5, (uint16_t*)A);
  std::vector<int64_t> n(5, 100);
  std::vector<int32_t> t(5, ELAS_GRAD_F32), u(5, ELAS_GRAD_BF16);
  std::vector<float> w(5, 0.1f);
  auto step = [&](int bits, size_t bytes) {
    float* s = bits == 8 ? f : nullptr;
    return elas_adamw_step(p.data(), g.data(), c.data(), n.data(), t.data(), u.data(), w.data(), 5, bits, A, s, A, s, (int64_t*)A, 1e-3, f, 0.9, 0.95,
                           1e-8, f, 1.0, A, bytes, nullptr);
  };
  EXPECT(step(8, 0) == ELAS_ERR_WORKSPACE && step(32, 0) == ELAS_ERR_WORKSPACE && step(4, 0) == ELAS_ERR_SHAPE);
  n[4] = big;
  EXPECT(step(8, 1 << 20) == ELAS_ERR_SHAPE);
  n[4] = 0, p[4] = nullptr, g[4] = nullptr, c[4] = nullptr;
  EXPECT(step(8, 0) == ELAS_ERR_WORKSPACE);
  c[3] = (uint16_t*)((char*)A + 1);
  EXPECT(step(8, 1 << 20) == ELAS_ERR_ALIGN);
  c[3] = nullptr, u[3] = 9;
  EXPECT(step(8, 1 << 20) == ELAS_ERR_FLAGS);
  EXPECT(elas_adam8_values((uint8_t*)A, f, big, 0, A, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_adam8_values(nullptr, nullptr, 0, 0, nullptr, nullptr) == ELAS_OK);

  printf("loss driver: %d failures\n", g_fail);
  return g_fail != 0;
}
