// C-ABI layer of the AdamW step (include/elas_adamw.h): argument checks on the host, before
// anything is enqueued.
#include <algorithm>

#include "../../include/elas_adamw.h"
#include "checks.h"

using elas::begin_call;
using elas::check_apart;
using elas::check_elem_ptr;
using elas::check_optional_ptr;
using elas::check_ptr;
using elas::check_scale;
using elas::check_workspace;
using elas::device_status;
using elas::fail;
using elas::Memory;

namespace {

constexpr int64_t kMaxTensors = (int64_t(1) << 20) - 1;

int check_type(int32_t t, const char* name, int64_t k) {
  if (t != ELAS_GRAD_F32 && t != ELAS_GRAD_BF16) return fail(ELAS_ERR_FLAGS, "%s[%lld]=%d is unknown", name, (long long)k, (int)t);
  return ELAS_OK;
}

int check_beta(double b, const char* name) {
  // (as float32 too, in which the moments are found)
  if (!(b >= 0.0 && (float)b < 1.f)) return fail(ELAS_ERR_SHAPE, "%s must be at least 0 and below 1", name);
  return ELAS_OK;
}

// What lies around some buffers.
struct Range {
  uint64_t from = UINT64_MAX, to = 0;
  Range(const Memory* m, int n) {
    for (int i = 0; i < n; ++i)
      if (m[i].end()) from = std::min(from, m[i].begin()), to = std::max(to, m[i].end());
  }
  bool meets(const void* p, int64_t bytes) const { return (uint64_t)(uintptr_t)p < to && from < (uint64_t)(uintptr_t)p + (uint64_t)bytes; }
};

}  // namespace

extern "C" {

size_t elas_adamw_workspace_bytes(void) { return elas::adamw_workspace_bytes(); }

int elas_adamw_step(void* const* params, const void* const* grads, uint16_t* const* copies, const int64_t* numel, const int32_t* param_dtype,
                    const int32_t* grad_dtype, const float* decay, int64_t n, int bits, void* m, float* m_scale, void* v, float* v_scale,
                    int64_t* step, double rate, const float* rate_factor, double beta1, double beta2, double eps, const float* norm,
                    double max_norm, void* workspace, size_t workspace_bytes, void* stream) {
  begin_call();
  if (n < 0 || n > kMaxTensors) return fail(ELAS_ERR_SHAPE, "n=%lld out of range", (long long)n);
  if (bits != 8 && bits != 32) return fail(ELAS_ERR_SHAPE, "bits=%d must be 8 or 32", bits);
  ELAS_CHECK(check_scale((float)rate, "rate (as float32)"));
  ELAS_CHECK(check_beta(beta1, "beta1"));
  ELAS_CHECK(check_beta(beta2, "beta2"));
  // (a moment of 0 over an eps whose reciprocal float32 cannot hold would be NaN)
  if (!((float)eps >= 0x1p-126f) || !isfinite((float)eps)) return fail(ELAS_ERR_SHAPE, "eps must be at least 2^-126 and finite in float32");
  if (!(max_norm >= 0.0)) return fail(ELAS_ERR_SHAPE, "max_norm must not be negative or NaN");
  if (n > 0 && (!params || !grads || !numel || !param_dtype || !grad_dtype || !decay))
    return fail(ELAS_ERR_NULL, "params, grads, numel, param_dtype, grad_dtype or decay is NULL");
  int64_t total = 0, blocks = 0;
  for (int64_t k = 0; k < n; ++k) {
    ELAS_CHECK(check_type(param_dtype[k], "param_dtype", k));
    ELAS_CHECK(check_type(grad_dtype[k], "grad_dtype", k));
    if (numel[k] < 0 || numel[k] >= (int64_t(1) << 40) - total)
      return fail(ELAS_ERR_SHAPE, "numel[%lld]=%lld out of range", (long long)k, (long long)numel[k]);
    ELAS_CHECK(check_scale(decay[k], "decay"));
    total += numel[k];
    blocks += (numel[k] + ELAS_ADAMW_BLOCK - 1) / ELAS_ADAMW_BLOCK;
    if (numel[k] == 0) continue;
    ELAS_CHECK(check_elem_ptr(params[k], param_dtype[k] == ELAS_GRAD_F32 ? 4 : 2, "a parameter"));
    ELAS_CHECK(check_elem_ptr(grads[k], grad_dtype[k] == ELAS_GRAD_F32 ? 4 : 2, "a gradient"));
    if (copies) ELAS_CHECK(check_optional_ptr(copies[k], 2, "a copy"));
  }
  if (total > 0) {
    ELAS_CHECK(check_ptr(m, "m"));
    ELAS_CHECK(check_ptr(v, "v"));
    if (bits == 8) {
      ELAS_CHECK(check_ptr(m_scale, "m_scale"));
      ELAS_CHECK(check_ptr(v_scale, "v_scale"));
    }
  }
  if (bits == 32) {
    ELAS_CHECK(elas::check_absent(m_scale, "m_scale", "moments in 8 bits"));
    ELAS_CHECK(elas::check_absent(v_scale, "v_scale", "moments in 8 bits"));
  }
  ELAS_CHECK(check_elem_ptr(step, 8, "step"));
  ELAS_CHECK(check_optional_ptr(rate_factor, 4, "rate_factor"));
  ELAS_CHECK(check_optional_ptr(norm, 4, "norm"));
  ELAS_CHECK(check_workspace(workspace, workspace_bytes, elas::adamw_workspace_bytes()));
  const int64_t moments = blocks * ELAS_ADAMW_BLOCK * (bits / 8);
  const Memory state[] = {Memory(m, moments, "m"), Memory(v, moments, "v"), Memory(m_scale, 4 * blocks, "m_scale"),
                          Memory(v_scale, 4 * blocks, "v_scale"), Memory(step, 8, "step"),
                          Memory(workspace, (int64_t)elas::adamw_workspace_bytes(), "workspace"),
                          Memory(norm, 4, "norm"), Memory(rate_factor, 4, "rate_factor")};
  constexpr int WRITTEN = 6, ALL = 8;
  ELAS_CHECK(check_apart(state, WRITTEN));
  // (the moments in one range and the small buffers in another, most tensors in neither: 49 tensors with gradients and copies
  // take the host up to 0.5 us, compared with every buffer 1.4 to 1.9)
  const Range moments_at(state, 4), others_at(state + 4, ALL - 4);
  const auto apart = [&](const void* p, int64_t bytes, int against, const char* name, int64_t k) {
    if (!moments_at.meets(p, bytes) && !others_at.meets(p, bytes)) return ELAS_OK;
    const Memory t(p, bytes, name);
    for (int i = 0; i < against; ++i)
      if (t.overlaps(state[i])) return fail(ELAS_ERR_OVERLAP, "%s (%lld) overlaps %s", name, (long long)k, state[i].name);
    return ELAS_OK;
  };
  for (int64_t k = 0; k < n; ++k) {
    if (numel[k] == 0) continue;
    ELAS_CHECK(apart(params[k], numel[k] * (param_dtype[k] == ELAS_GRAD_F32 ? 4 : 2), ALL, "a parameter", k));
    ELAS_CHECK(apart(grads[k], numel[k] * (grad_dtype[k] == ELAS_GRAD_F32 ? 4 : 2), WRITTEN, "a gradient", k));
    if (copies && copies[k]) ELAS_CHECK(apart(copies[k], numel[k] * 2, ALL, "a copy", k));
  }
  elas::AdamwArgs a{};
  a.params = params; a.grads = grads; a.copies = copies; a.numel = numel; a.param_dtype = param_dtype; a.grad_dtype = grad_dtype;
  a.decay = decay; a.n = n; a.eight = bits == 8; a.m = m; a.v = v; a.m_scale = m_scale; a.v_scale = v_scale; a.step = step; a.rate = rate;
  a.beta1 = beta1; a.beta2 = beta2; a.eps = eps; a.max_norm = max_norm; a.rate_factor = rate_factor; a.norm = norm; a.ws = workspace;
  return device_status(elas::run_adamw(a, (hipStream_t)stream), "AdamW launch");
}

int elas_adam8_values(const uint8_t* codes, const float* scale, int64_t blocks, uint32_t flags, void* out, void* stream) {
  begin_call();
  if (flags & ~(ELAS_RES_F32 | ELAS_ADAM8_SECOND)) return fail(ELAS_ERR_FLAGS, "flags: only ELAS_RES_F32 and ELAS_ADAM8_SECOND are allowed");
  if (blocks < 0 || blocks >= int64_t(1) << 32) return fail(ELAS_ERR_SHAPE, "blocks=%lld out of range", (long long)blocks);
  if (blocks == 0) return ELAS_OK;
  ELAS_CHECK(check_ptr(codes, "codes"));
  ELAS_CHECK(check_ptr(scale, "scale"));
  ELAS_CHECK(check_ptr(out, "out"));
  ELAS_CHECK(check_apart({Memory(out, blocks * ELAS_ADAMW_BLOCK * (flags & ELAS_RES_F32 ? 4 : 2), "out"),
                          Memory(codes, blocks * ELAS_ADAMW_BLOCK, "codes"), Memory(scale, 4 * blocks, "scale")}, 1));
  return device_status(elas::run_adam8_values(codes, scale, blocks, (flags & ELAS_ADAM8_SECOND) != 0, (flags & ELAS_RES_F32) != 0, out,
                                              (hipStream_t)stream),
                       "moments' values launch");
}

}  // extern "C"
