// C-ABI layer of the operators around the FFN (include/elas_train.h): argument
// checks on the host, before anything is enqueued.
#include <math.h>

#include "../../include/elas_train.h"
#include "internal.h"

using elas::begin_call;
using elas::check_ptr;
using elas::device_status;
using elas::fail;

namespace {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxWidth = 65536;
constexpr int64_t kMaxTensors = (int64_t(1) << 20) - 1;

int check_rows(int64_t T, int64_t d) {
  if (T < 0 || T > kMaxRows) return fail(ELAS_ERR_SHAPE, "T=%lld out of range", (long long)T);
  if (d <= 0 || d % 8 || d > kMaxWidth)
    return fail(ELAS_ERR_SHAPE, "d=%lld must be a positive multiple of 8, at most 65536", (long long)d);
  return ELAS_OK;
}

int check_scale(float v, const char* name) {
  if (!isfinite(v)) return fail(ELAS_ERR_SHAPE, "%s must be finite", name);
  return ELAS_OK;
}

// Alignment of a pointer that only needs its element's; NULL is an error.
int check_elem_ptr(const void* p, size_t size, const char* name) {
  if (p == nullptr) return fail(ELAS_ERR_NULL, "%s is NULL", name);
  if ((uintptr_t)p % size) return fail(ELAS_ERR_ALIGN, "%s is not %zu-byte aligned", name, size);
  return ELAS_OK;
}

int check_absent(const void* p, const char* name, const char* needs) {
  if (p != nullptr) return fail(ELAS_ERR_FLAGS, "%s is given without %s", name, needs);
  return ELAS_OK;
}

int check_workspace(const void* ws, size_t have, size_t need) {
  if (have < need) return fail(ELAS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", have, need);
  return need ? check_ptr(ws, "workspace") : ELAS_OK;
}

// Sizes, flags and which operands belong together, for both directions.
int check_join(const uint16_t* b, const uint16_t* gate, const uint16_t* w_post, int64_t T, int64_t d, float res_scale,
               float block_scale, float eps, uint32_t flags) {
  if (flags & ~(ELAS_RES_F32 | ELAS_GATE_TOKEN))
    return fail(ELAS_ERR_FLAGS, "norm join flags: only ELAS_RES_F32 and ELAS_GATE_TOKEN are allowed");
  ELAS_CHECK(check_rows(T, d));
  ELAS_CHECK(check_scale(res_scale, "res_scale"));
  ELAS_CHECK(check_scale(block_scale, "block_scale"));
  if (!(eps >= 0.f) || !isfinite(eps)) return fail(ELAS_ERR_SHAPE, "eps must be finite and not negative");
  if (T == 0) return ELAS_OK;
  if (b == nullptr) {
    ELAS_CHECK(check_absent(gate, "gate", "b"));
    ELAS_CHECK(check_absent(w_post, "w_post", "b"));
  }
  if ((flags & ELAS_GATE_TOKEN) && gate == nullptr) return fail(ELAS_ERR_NULL, "gate is NULL, with ELAS_GATE_TOKEN");
  return ELAS_OK;
}

int check_embed(int64_t T, int64_t V, int64_t d, float scale, uint32_t flags, uint32_t allowed) {
  if (flags & ~allowed) return fail(ELAS_ERR_FLAGS, "unknown flags 0x%x", flags & ~allowed);
  ELAS_CHECK(check_rows(T, d));
  if (V <= 0 || V > kMaxRows) return fail(ELAS_ERR_SHAPE, "V=%lld out of range", (long long)V);
  return check_scale(scale, "scale");
}

int check_grads(const void* const* grads, void* const* out, const int64_t* numel, const int32_t* dtype, int64_t n) {
  if (n < 0 || n > kMaxTensors) return fail(ELAS_ERR_SHAPE, "n=%lld out of range", (long long)n);
  if (n == 0) return ELAS_OK;
  if (!grads || !numel || !dtype) return fail(ELAS_ERR_NULL, "grads, numel or dtype is NULL");
  int64_t total = 0;
  for (int64_t k = 0; k < n; ++k) {
    if (dtype[k] != ELAS_GRAD_F32 && dtype[k] != ELAS_GRAD_BF16)
      return fail(ELAS_ERR_FLAGS, "dtype[%lld]=%d is unknown", (long long)k, (int)dtype[k]);
    if (numel[k] < 0 || numel[k] >= (int64_t(1) << 44) - total)
      return fail(ELAS_ERR_SHAPE, "numel[%lld]=%lld out of range", (long long)k, (long long)numel[k]);
    total += numel[k];
    if (numel[k] == 0) continue;
    const size_t size = dtype[k] == ELAS_GRAD_F32 ? 4 : 2;
    ELAS_CHECK(check_elem_ptr(grads[k], size, "a gradient"));
    if (out) ELAS_CHECK(check_elem_ptr(out[k], size, "an output"));
  }
  return ELAS_OK;
}

}  // namespace

extern "C" {

int elas_norm_join_fwd(const void* h, const uint16_t* b, const uint16_t* gate, const uint16_t* w_post, const uint16_t* w_pre,
                       int64_t T, int64_t d, float res_scale, float block_scale, float eps, uint32_t flags, void* h_out,
                       uint16_t* n, void* stream) {
  begin_call();
  ELAS_CHECK(check_join(b, gate, w_post, T, d, res_scale, block_scale, eps, flags));
  if (T == 0) return ELAS_OK;
  ELAS_CHECK(check_ptr(h, "h"));
  if (b) {
    ELAS_CHECK(check_ptr(b, "b"));
    ELAS_CHECK(check_ptr(h_out, "h_out"));
    if (gate) ELAS_CHECK(check_ptr(gate, "gate"));
    if (w_post) ELAS_CHECK(check_ptr(w_post, "w_post"));
  } else {
    ELAS_CHECK(check_absent(h_out, "h_out", "b"));
    ELAS_CHECK(check_ptr(w_pre, "w_pre"));
  }
  if (w_pre) {
    ELAS_CHECK(check_ptr(w_pre, "w_pre"));
    ELAS_CHECK(check_ptr(n, "n"));
  } else {
    ELAS_CHECK(check_absent(n, "n", "w_pre"));
  }
  elas::NormJoinArgs a{};
  a.T = T; a.d = d; a.h = h; a.b = b; a.gate = gate; a.w_post = w_post; a.w_pre = w_pre;
  a.res_scale = b ? res_scale : 1.f; a.block_scale = block_scale; a.eps = eps;
  a.res_f32 = (flags & ELAS_RES_F32) != 0; a.gate_token = (flags & ELAS_GATE_TOKEN) != 0;
  a.h_out = h_out; a.n = n;
  return device_status(elas::run_norm_join_fwd(a, (hipStream_t)stream), "norm join launch");
}

size_t elas_norm_join_bwd_workspace_bytes(int64_t T, int64_t d, uint32_t flags) {
  (void)flags;
  if (T < 0 || T > kMaxRows || d <= 0 || d > kMaxWidth) return 0;
  return elas::norm_join_bwd_workspace_bytes(T, d);
}

int elas_norm_join_bwd(const void* dh_out, const uint16_t* dn, const void* h_out, const uint16_t* b, const uint16_t* gate,
                       const uint16_t* w_post, const uint16_t* w_pre, int64_t T, int64_t d, float res_scale, float block_scale,
                       float eps, uint32_t flags, void* dh, uint16_t* db, void* dgate, float* dw_post, float* dw_pre,
                       void* workspace, size_t workspace_bytes, void* stream) {
  begin_call();
  ELAS_CHECK(check_join(b, gate, w_post, T, d, res_scale, block_scale, eps, flags));
  const bool gate_token = (flags & ELAS_GATE_TOKEN) != 0;
  if (T > 0) {
    if (dh_out) ELAS_CHECK(check_ptr(dh_out, "dh_out"));
    if (dh) ELAS_CHECK(check_ptr(dh, "dh"));
    if (w_pre) {
      ELAS_CHECK(check_ptr(w_pre, "w_pre"));
      ELAS_CHECK(check_ptr(dn, "dn"));
      ELAS_CHECK(check_ptr(h_out, "h_out"));
      ELAS_CHECK(check_ptr(dw_pre, "dw_pre"));
    } else {
      ELAS_CHECK(check_absent(dn, "dn", "w_pre"));
      ELAS_CHECK(check_absent(dw_pre, "dw_pre", "w_pre"));
      if (!dh_out) return fail(ELAS_ERR_NULL, "dh_out is NULL, without w_pre");
    }
    if (b) {
      ELAS_CHECK(check_ptr(b, "b"));
      ELAS_CHECK(check_ptr(db, "db"));
    } else {
      ELAS_CHECK(check_absent(db, "db", "b"));
      ELAS_CHECK(check_ptr(w_pre, "w_pre"));
      ELAS_CHECK(check_ptr(dh, "dh"));
    }
    if (gate) {
      ELAS_CHECK(check_ptr(gate, "gate"));
      ELAS_CHECK(check_ptr(dgate, "dgate"));
    } else {
      ELAS_CHECK(check_absent(dgate, "dgate", "gate"));
    }
    if (w_post) {
      ELAS_CHECK(check_ptr(w_post, "w_post"));
      ELAS_CHECK(check_ptr(dw_post, "dw_post"));
    } else {
      ELAS_CHECK(check_absent(dw_post, "dw_post", "w_post"));
    }
  } else {
    if (dgate && !gate_token) ELAS_CHECK(check_ptr(dgate, "dgate"));
    if (dw_post) ELAS_CHECK(check_ptr(dw_post, "dw_post"));
    if (dw_pre) ELAS_CHECK(check_ptr(dw_pre, "dw_pre"));
  }
  ELAS_CHECK(check_workspace(workspace, workspace_bytes, elas::norm_join_bwd_workspace_bytes(T, d)));
  elas::NormJoinArgs a{};
  a.T = T; a.d = d;
  a.res_scale = b ? res_scale : 1.f; a.block_scale = block_scale; a.eps = eps;
  a.res_f32 = (flags & ELAS_RES_F32) != 0; a.gate_token = gate_token;
  if (T > 0) {   // (without tokens no operand is checked, nor read: the sums are zeros whatever a gain holds)
    a.h = h_out; a.b = b; a.gate = gate; a.w_post = w_post; a.w_pre = w_pre;
    a.dh_out = dh_out; a.dn = dn; a.dh = dh; a.db = db;
  }
  a.dgate = dgate; a.dw_post = dw_post; a.dw_pre = dw_pre;
  a.ws = workspace;
  return device_status(elas::run_norm_join_bwd(a, (hipStream_t)stream), "norm join backward launch");
}

int elas_embed_fwd(const void* ids, const uint16_t* table, int64_t T, int64_t V, int64_t d, float scale, uint32_t flags, void* x,
                   void* stream) {
  begin_call();
  ELAS_CHECK(check_embed(T, V, d, scale, flags, ELAS_RES_F32 | ELAS_IDS_I64));
  if (T == 0) return ELAS_OK;
  elas::EmbedArgs a{};
  a.ids_i64 = (flags & ELAS_IDS_I64) != 0;
  ELAS_CHECK(check_elem_ptr(ids, a.ids_i64 ? 8 : 4, "ids"));
  ELAS_CHECK(check_ptr(table, "table"));
  ELAS_CHECK(check_ptr(x, "x"));
  a.T = T; a.V = V; a.d = d; a.ids = ids; a.res_f32 = (flags & ELAS_RES_F32) != 0; a.scale = scale; a.table = table; a.x = x;
  return device_status(elas::run_embed_fwd(a, (hipStream_t)stream), "embedding launch");
}

size_t elas_embed_bwd_workspace_bytes(int64_t T, int64_t V, int64_t d, uint32_t flags) {
  if (T < 0 || T > kMaxRows || V <= 0 || V > kMaxRows || d <= 0 || d > kMaxWidth) return 0;
  return elas::embed_bwd_workspace_bytes(T, V, d, (flags & ELAS_EMBED_ADD) != 0);
}

int elas_embed_bwd(const void* ids, const void* dx, int64_t T, int64_t V, int64_t d, float scale, uint32_t flags, float* dtable,
                   void* workspace, size_t workspace_bytes, void* stream) {
  begin_call();
  ELAS_CHECK(check_embed(T, V, d, scale, flags, ELAS_RES_F32 | ELAS_IDS_I64 | ELAS_EMBED_ADD));
  elas::EmbedArgs a{};
  a.ids_i64 = (flags & ELAS_IDS_I64) != 0;
  a.add = (flags & ELAS_EMBED_ADD) != 0;
  if (T == 0 && a.add) return ELAS_OK;
  if (T > 0) {
    ELAS_CHECK(check_elem_ptr(ids, a.ids_i64 ? 8 : 4, "ids"));
    ELAS_CHECK(check_ptr(dx, "dx"));
  }
  ELAS_CHECK(check_ptr(dtable, "dtable"));
  ELAS_CHECK(check_workspace(workspace, workspace_bytes, elas::embed_bwd_workspace_bytes(T, V, d, a.add)));
  a.T = T; a.V = V; a.d = d; a.ids = ids; a.res_f32 = (flags & ELAS_RES_F32) != 0; a.scale = scale; a.dx = dx; a.dtable = dtable;
  a.ws = workspace;
  return device_status(elas::run_embed_bwd(a, (hipStream_t)stream), "embedding gradient launch");
}

size_t elas_grad_workspace_bytes(int64_t n) { return n < 0 || n > kMaxTensors ? 0 : elas::grad_workspace_bytes(n); }

int elas_grad_norm(const void* const* grads, const int64_t* numel, const int32_t* dtype, int64_t n, float* norm, void* workspace,
                   size_t workspace_bytes, void* stream) {
  begin_call();
  ELAS_CHECK(check_grads(grads, nullptr, numel, dtype, n));
  ELAS_CHECK(check_elem_ptr(norm, 4, "norm"));
  ELAS_CHECK(check_workspace(workspace, workspace_bytes, elas::grad_workspace_bytes(n)));
  return device_status(elas::run_grad_norm(grads, nullptr, numel, dtype, n, false, 0.f, norm, workspace, (hipStream_t)stream),
                       "gradient norm launch");
}

int elas_grad_clip(const void* const* grads, void* const* out, const int64_t* numel, const int32_t* dtype, int64_t n, float max_norm,
                   float* stats, void* workspace, size_t workspace_bytes, void* stream) {
  begin_call();
  ELAS_CHECK(check_grads(grads, out, numel, dtype, n));
  if (!(max_norm >= 0.f)) return fail(ELAS_ERR_SHAPE, "max_norm must not be negative or NaN");
  ELAS_CHECK(check_elem_ptr(stats, 4, "stats"));
  ELAS_CHECK(check_workspace(workspace, workspace_bytes, elas::grad_workspace_bytes(n)));
  return device_status(elas::run_grad_norm(grads, out ? out : (void* const*)grads, numel, dtype, n, true, max_norm, stats, workspace,
                                           (hipStream_t)stream),
                       "gradient clipping launch");
}

}  // extern "C"
