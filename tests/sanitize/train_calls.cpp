// What the entry points of include/elas_train.h hand on to their launch sequences, which
// are replaced here (tests/test_train_calls.py); no device is used.
#include <stdarg.h>
#include <stdio.h>

#include "elas_train.h"
#include "../../paper_2605_03667_amd/csrc/internal.h"

namespace elas {

static NormJoinArgs g_join;
static int g_calls = 0;

void begin_call() {}
int fail(int code, const char*, ...) { return code; }
int check_ptr(const void* p, const char*) { return !p ? ELAS_ERR_NULL : ((uintptr_t)p & 15) ? ELAS_ERR_ALIGN : ELAS_OK; }
int device_status(hipError_t e, const char*) { return e == hipSuccess ? ELAS_OK : ELAS_ERR_DEVICE; }
size_t norm_join_bwd_workspace_bytes(int64_t, int64_t) { return 64; }
size_t embed_bwd_workspace_bytes(int64_t, int64_t, int64_t, bool) { return 0; }
size_t grad_workspace_bytes(int64_t) { return 0; }
hipError_t run_norm_join_fwd(const NormJoinArgs& a, hipStream_t) { return g_join = a, ++g_calls, hipSuccess; }
hipError_t run_norm_join_bwd(const NormJoinArgs& a, hipStream_t) { return g_join = a, ++g_calls, hipSuccess; }
hipError_t run_embed_fwd(const EmbedArgs&, hipStream_t) { return hipSuccess; }
hipError_t run_embed_bwd(const EmbedArgs&, hipStream_t) { return hipSuccess; }
hipError_t run_grad_norm(const void* const*, void* const*, const int64_t*, const int32_t*, int64_t, bool, float, float*, void*, hipStream_t) {
  return hipSuccess;
}

}  // namespace elas

static int g_fail = 0;
#define EXPECT(cond)                                             \
  do {                                                           \
    if (!(cond)) {                                               \
      fprintf(stderr, "FAIL line %d: %s\n", __LINE__, #cond);    \
      ++g_fail;                                                  \
    }                                                            \
  } while (0)

int main() {
  using elas::g_calls;
  using elas::g_join;
  void* A = (void*)0x10000;
  void* U = (void*)0x10009;   // stale: neither aligned nor anybody's memory
  uint16_t *a = (uint16_t*)A, *u = (uint16_t*)U;
  float *x = (float*)0x20000, *y = (float*)0x30000, *z = (float*)0x40000;

  // backward without tokens: only the weight gradients are handed on
  for (uint32_t flags : {0u, ELAS_RES_F32, ELAS_GATE_TOKEN}) {
    g_calls = 0;
    EXPECT(elas_norm_join_bwd(U, u, U, u, u, u, u, 0, 16, 1.f, 1.f, 1e-6f, flags, U, u, flags & ELAS_GATE_TOKEN ? U : (void*)x, y, z, A, 64,
                              nullptr) == ELAS_OK);
    EXPECT(g_calls == 1 && g_join.T == 0 && g_join.d == 16);
    EXPECT(!g_join.h && !g_join.b && !g_join.gate && !g_join.w_post && !g_join.w_pre);
    EXPECT(!g_join.dh_out && !g_join.dn && !g_join.dh && !g_join.db);
    EXPECT(g_join.dw_post == y && g_join.dw_pre == z && (flags & ELAS_GATE_TOKEN || g_join.dgate == x));
  }
  // with tokens: everything is
  EXPECT(elas_norm_join_bwd(A, a, A, a, a, a, a, 4, 16, 1.f, 1.f, 1e-6f, 0, A, a, x, y, z, A, 64, nullptr) == ELAS_OK);
  EXPECT(g_join.h && g_join.b && g_join.gate && g_join.w_post && g_join.w_pre && g_join.dh_out && g_join.dn && g_join.dh && g_join.db);
  // forward without tokens: nothing is launched
  g_calls = 0;
  EXPECT(elas_norm_join_fwd(U, u, u, u, u, 0, 16, 1.f, 1.f, 1e-6f, 0, U, u, nullptr) == ELAS_OK && g_calls == 0);

  printf("train calls: %d failures\n", g_fail);
  return g_fail != 0;
}
