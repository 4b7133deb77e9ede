// Host-side exercise of include/elas_train.h for AddressSanitizer / Undefined-
// BehaviorSanitizer builds (tests/test_train_sanitizers.py): every argument check, and
// the workspace planning over many shapes.  No call may reach a kernel launch: every
// launching call here has an invalid argument or nothing to do.
#include <math.h>
#include <stdio.h>

#include <vector>

#include "elas_train.h"

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
  void* U = (void*)0x10008;   // misaligned
  uint16_t* a = (uint16_t*)A;
  float* f = (float*)A;

  // norm join
  EXPECT(elas_norm_join_fwd(A, a, a, a, a, 4, 16, 1.f, 1.f, 1e-6f, 16u, A, a, nullptr) == ELAS_ERR_FLAGS);
  EXPECT(elas_norm_join_fwd(A, a, a, a, a, 4, 65544, 1.f, 1.f, 1e-6f, 0, A, a, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_norm_join_fwd(A, a, a, a, a, INT64_MAX, 16, 1.f, 1.f, 1e-6f, 0, A, a, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_norm_join_fwd(A, a, a, a, a, 4, 16, NAN, 1.f, 1e-6f, 0, A, a, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_norm_join_fwd(A, a, a, a, a, 4, 16, 1.f, 1.f, -1.f, 0, A, a, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_norm_join_fwd(A, a, a, a, a, 4, 16, 1.f, 1.f, 1e-6f, 0, U, a, nullptr) == ELAS_ERR_ALIGN);
  EXPECT(elas_norm_join_fwd(A, nullptr, a, a, a, 4, 16, 1.f, 1.f, 1e-6f, 0, A, a, nullptr) == ELAS_ERR_FLAGS);
  EXPECT(elas_norm_join_fwd(A, a, a, a, nullptr, 4, 16, 1.f, 1.f, 1e-6f, 0, A, a, nullptr) == ELAS_ERR_FLAGS);
  EXPECT(elas_norm_join_fwd(nullptr, nullptr, nullptr, nullptr, nullptr, 0, 16, 1.f, 1.f, 0.f, 0, nullptr, nullptr, nullptr) == ELAS_OK);
  EXPECT(elas_norm_join_bwd(A, a, A, a, a, a, a, 4, 16, 1.f, 1.f, 1e-6f, 0, A, a, A, f, f, A, 0, nullptr) == ELAS_ERR_WORKSPACE);
  EXPECT(elas_norm_join_bwd(A, a, A, a, a, a, a, 4, 16, 1.f, 1.f, 1e-6f, 0, A, a, A, f, f, U, 1 << 30, nullptr) == ELAS_ERR_ALIGN);
  EXPECT(elas_norm_join_bwd(nullptr, nullptr, A, a, a, a, nullptr, 4, 16, 1.f, 1.f, 1e-6f, 0, A, a, A, f, nullptr, A, 1 << 30, nullptr) ==
         ELAS_ERR_NULL);

  // embedding
  EXPECT(elas_embed_fwd(A, a, 4, 0, 16, 1.f, 0, A, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_embed_fwd(A, a, 4, 10, 16, INFINITY, 0, A, nullptr) == ELAS_ERR_SHAPE);
  EXPECT(elas_embed_fwd((char*)A + 4, a, 4, 10, 16, 1.f, ELAS_IDS_I64, A, nullptr) == ELAS_ERR_ALIGN);
  EXPECT(elas_embed_fwd(A, a, 4, 10, 16, 1.f, ELAS_EMBED_ADD, A, nullptr) == ELAS_ERR_FLAGS);
  EXPECT(elas_embed_bwd(A, A, 5000, 10, 16, 1.f, 0, f, A, 0, nullptr) == ELAS_ERR_WORKSPACE);
  EXPECT(elas_embed_bwd_workspace_bytes(4096, 32000, 512, 0) == 0);
  EXPECT(elas_embed_bwd(A, A, 4, 10, 16, 1.f, 0, nullptr, A, 1 << 30, nullptr) == ELAS_ERR_NULL);
  EXPECT(elas_embed_bwd(nullptr, nullptr, 0, 10, 16, 1.f, ELAS_EMBED_ADD, nullptr, nullptr, 0, nullptr) == ELAS_OK);

  // gradients
  std::vector<const void*> g(5, A);
  std::vector<void*> o(5, A);
  std::vector<int64_t> n(5, 100);
  std::vector<int32_t> t(5, ELAS_GRAD_F32);
  auto clip = [&](float max_norm, float* stats) {
    return elas_grad_clip(g.data(), o.data(), n.data(), t.data(), 5, max_norm, stats, A, 0, nullptr);
  };
  EXPECT(clip(1.f, f) == ELAS_ERR_WORKSPACE);
  EXPECT(clip(-1.f, f) == ELAS_ERR_SHAPE);
  EXPECT(clip(1.f, (float*)((char*)A + 2)) == ELAS_ERR_ALIGN);
  n[4] = INT64_MAX;
  EXPECT(clip(1.f, f) == ELAS_ERR_SHAPE);
  n[4] = 0, g[4] = nullptr, o[4] = nullptr;
  EXPECT(clip(1.f, f) == ELAS_ERR_WORKSPACE);
  t[3] = -7;
  EXPECT(clip(1.f, f) == ELAS_ERR_FLAGS);
  EXPECT(elas_grad_norm(nullptr, nullptr, nullptr, 1, f, A, 1 << 30, nullptr) == ELAS_ERR_NULL);

  // workspace sizes: finite, and growing at most with the sizes they are for
  for (int64_t T : {int64_t(0), int64_t(1), int64_t(4096), int64_t(4097), int64_t(131072), int64_t(131073), int64_t(1) << 20, (int64_t(1) << 31) - 1})
    for (int64_t d : {8, 512, 520, 2048, 65536})
      for (uint32_t flags : {0u, ELAS_RES_F32, ELAS_EMBED_ADD}) {
        const size_t join = elas_norm_join_bwd_workspace_bytes(T, d, flags & ELAS_RES_F32);
        EXPECT(join > 0 && join <= (size_t)1024 * 2 * d * 4);
        for (int64_t V : {int64_t(1), int64_t(32000), (int64_t(1) << 31) - 1}) {
          const size_t embed = elas_embed_bwd_workspace_bytes(T, V, d, flags);
          EXPECT(embed <= (size_t)T * 32 + (size_t)(9000 + d) * 512 * 4 + (1 << 20) * (size_t)(1 + T / 1000000));
        }
      }
  EXPECT(elas_grad_workspace_bytes(-1) == 0 && elas_grad_workspace_bytes((1 << 20) - 1) > 0);

  printf("train driver: %d failures\n", g_fail);
  return g_fail != 0;
}
