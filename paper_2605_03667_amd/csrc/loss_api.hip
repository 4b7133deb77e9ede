// C-ABI layer of the losses (include/elas_loss.h): argument checks on the host, before
// anything is enqueued.
#include "../../include/elas_loss.h"
#include "checks.h"

using elas::begin_call;
using elas::check_apart;
using elas::check_elem_ptr;
using elas::check_optional_ptr;
using elas::check_scale;
using elas::check_workspace;
using elas::device_status;
using elas::fail;
using elas::LogitsArgs;
using elas::Memory;

namespace {

constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxVocab = int64_t(1) << 30;
constexpr int64_t kMaxValues = int64_t(1) << 40;
constexpr int64_t kMaxPitch = int64_t(1) << 31;

// What the calls on logits share; nothing is inspected behind the sizes where there are no tokens.
int check_logits(LogitsArgs& a, const void* logits, int64_t ld, const void* ids, int64_t T, int64_t V, float scale, uint32_t flags,
                 void* dlogits, int64_t ld_out) {
  if (flags & ~(ELAS_LOGITS_F32 | ELAS_IDS_I64)) return fail(ELAS_ERR_FLAGS, "flags: only ELAS_LOGITS_F32 and ELAS_IDS_I64 are allowed");
  if (T < 0 || T > kMaxTokens) return fail(ELAS_ERR_SHAPE, "T=%lld out of range", (long long)T);
  if (V <= 0 || V > kMaxVocab) return fail(ELAS_ERR_SHAPE, "V=%lld out of range", (long long)V);
  if (!(scale > 0.f && scale <= 0x1p100f)) return fail(ELAS_ERR_SHAPE, "scale must be positive and at most 2^100");
  if (ld < V || ld > kMaxPitch) return fail(ELAS_ERR_SHAPE, "ld=%lld must be at least V=%lld and at most 2^31", (long long)ld, (long long)V);
  if (dlogits && (ld_out < V || ld_out > kMaxPitch))
    return fail(ELAS_ERR_SHAPE, "ld_out=%lld must be at least V=%lld and at most 2^31", (long long)ld_out, (long long)V);
  if (dlogits && dlogits == logits && ld_out != ld) return fail(ELAS_ERR_SHAPE, "dlogits is logits, with another pitch");
  a.f32 = (flags & ELAS_LOGITS_F32) != 0;
  a.ids_i64 = (flags & ELAS_IDS_I64) != 0;
  a.T = T; a.V = V; a.ld = ld; a.ld_out = ld_out; a.scale = scale;
  a.logits = logits; a.ids = ids; a.dlogits = dlogits;
  if (T == 0) return ELAS_OK;
  const size_t size = a.f32 ? 4 : 2;
  ELAS_CHECK(check_elem_ptr(logits, size, "logits"));
  ELAS_CHECK(check_elem_ptr(ids, a.ids_i64 ? 8 : 4, "ids"));
  ELAS_CHECK(check_optional_ptr(dlogits, size, "dlogits"));
  return ELAS_OK;
}

// What a call on logits reads and writes.  (A gradient in its logits' place: the rows once, as a result.)
Memory gradient(const LogitsArgs& a) {
  const int64_t size = a.f32 ? 4 : 2;
  return Memory(a.dlogits, a.T, a.V * size, a.ld_out * size, "dlogits");
}
Memory logits(const LogitsArgs& a) {
  const int64_t size = a.f32 ? 4 : 2;
  return Memory(a.logits == a.dlogits ? nullptr : a.logits, a.T, a.V * size, a.ld * size, "logits");
}
Memory ids(const LogitsArgs& a) { return Memory(a.ids, a.T * (a.ids_i64 ? 8 : 4), "ids"); }
Memory tokens(const LogitsArgs& a, const float* p, const char* name) { return Memory(p, a.T * 4, name); }

size_t workspace_of(const LogitsArgs& a) { return elas::token_loss_workspace_bytes(a.T, a.V, a.f32); }

}  // namespace

extern "C" {

size_t elas_token_loss_workspace_bytes(int64_t T, int64_t V, uint32_t flags) {
  if (T < 0 || T > kMaxTokens || V <= 0 || V > kMaxVocab) return 0;
  return elas::token_loss_workspace_bytes(T, V, (flags & ELAS_LOGITS_F32) != 0);
}

int elas_token_logp_fwd(const void* logits, int64_t ld, const void* ids, int64_t T, int64_t V, float scale, uint32_t flags, float* logp,
                        float* lse, void* stream) {
  begin_call();
  LogitsArgs a{};
  a.kind = LogitsArgs::LOGP;
  ELAS_CHECK(check_logits(a, logits, ld, ids, T, V, scale, flags, nullptr, 0));
  if (T == 0) return ELAS_OK;
  ELAS_CHECK(check_elem_ptr(logp, 4, "logp"));
  ELAS_CHECK(check_optional_ptr(lse, 4, "lse"));
  ELAS_CHECK(check_apart({tokens(a, logp, "logp"), tokens(a, lse, "lse"), ::logits(a), ::ids(a)}, 2));
  a.logp = logp; a.lse = lse;
  return device_status(elas::run_token_loss(a, (hipStream_t)stream), "log-probability launch");
}

int elas_token_logp_bwd(const float* dlogp, const float* dlse, const void* logits, int64_t ld, const void* ids, const float* lse, int64_t T,
                        int64_t V, float scale, uint32_t flags, void* dlogits, int64_t ld_out, void* stream) {
  begin_call();
  if (!dlogits && T > 0) return fail(ELAS_ERR_NULL, "dlogits is NULL");
  LogitsArgs a{};
  ELAS_CHECK(check_logits(a, logits, ld, ids, T, V, scale, flags, dlogits, ld_out));
  if (T == 0) return ELAS_OK;
  ELAS_CHECK(check_elem_ptr(dlogp, 4, "dlogp"));
  ELAS_CHECK(check_optional_ptr(dlse, 4, "dlse"));
  ELAS_CHECK(check_elem_ptr(lse, 4, "lse"));
  ELAS_CHECK(check_apart({gradient(a), ::logits(a), ::ids(a), tokens(a, dlogp, "dlogp"), tokens(a, dlse, "dlse"), tokens(a, lse, "lse")}, 1));
  a.dlogp = dlogp; a.dlse = dlse; a.lse_in = lse;
  return device_status(elas::run_token_logp_bwd(a, (hipStream_t)stream), "log-probability backward launch");
}

int elas_token_loss(const void* logits, int64_t ld, const void* ids, const float* weight, int64_t T, int64_t V, float scale, float reduce,
                    float z_coef, uint32_t flags, float* logp, float* lse, void* dlogits, int64_t ld_out, float* stats, void* workspace,
                    size_t workspace_bytes, void* stream) {
  begin_call();
  LogitsArgs a{};
  a.kind = LogitsArgs::TOKEN;
  ELAS_CHECK(check_logits(a, logits, ld, ids, T, V, scale, flags, dlogits, ld_out));
  ELAS_CHECK(check_scale(reduce, "reduce"));
  ELAS_CHECK(check_scale(z_coef, "z_coef"));
  if (T > 0) {
    ELAS_CHECK(check_optional_ptr(weight, 4, "weight"));
    ELAS_CHECK(check_optional_ptr(logp, 4, "logp"));
    ELAS_CHECK(check_optional_ptr(lse, 4, "lse"));
  }
  ELAS_CHECK(check_elem_ptr(stats, 4, "stats"));
  ELAS_CHECK(check_workspace(workspace, workspace_bytes, workspace_of(a)));
  ELAS_CHECK(check_apart({tokens(a, logp, "logp"), tokens(a, lse, "lse"), gradient(a), Memory(stats, 8, "stats"),
                          Memory(workspace, (int64_t)workspace_of(a), "workspace"), ::logits(a), ::ids(a), tokens(a, weight, "weight")}, 5));
  a.weight = weight; a.reduce = reduce; a.z_coef = z_coef; a.logp = logp; a.lse = lse; a.stats = stats; a.ws = workspace;
  return device_status(elas::run_token_loss(a, (hipStream_t)stream), "token loss launch");
}

int elas_policy_loss(const void* logits, int64_t ld, const void* ids, const float* advantage, const float* old_logp, const float* ref_logp,
                     const float* weight, int64_t T, int64_t V, float scale, float reduce, float clip_low, float clip_high, float kl_coef,
                     uint32_t flags, float* logp, void* dlogits, int64_t ld_out, float* stats, void* workspace, size_t workspace_bytes,
                     void* stream) {
  begin_call();
  LogitsArgs a{};
  a.kind = LogitsArgs::POLICY;
  ELAS_CHECK(check_logits(a, logits, ld, ids, T, V, scale, flags, dlogits, ld_out));
  ELAS_CHECK(check_scale(reduce, "reduce"));
  ELAS_CHECK(check_scale(kl_coef, "kl_coef"));
  if (!(clip_low >= 0.f && clip_low <= 1.f)) return fail(ELAS_ERR_SHAPE, "clip_low must be between 0 and 1");
  if (!(clip_high >= 0.f)) return fail(ELAS_ERR_SHAPE, "clip_high must not be negative or NaN");
  if (T > 0) {
    if (kl_coef != 0.f && !ref_logp) return fail(ELAS_ERR_NULL, "ref_logp is NULL, with a kl_coef");
    ELAS_CHECK(check_elem_ptr(advantage, 4, "advantage"));
    ELAS_CHECK(check_optional_ptr(old_logp, 4, "old_logp"));
    ELAS_CHECK(check_optional_ptr(ref_logp, 4, "ref_logp"));
    ELAS_CHECK(check_optional_ptr(weight, 4, "weight"));
    ELAS_CHECK(check_optional_ptr(logp, 4, "logp"));
  }
  ELAS_CHECK(check_elem_ptr(stats, 4, "stats"));
  ELAS_CHECK(check_workspace(workspace, workspace_bytes, workspace_of(a)));
  ELAS_CHECK(check_apart({tokens(a, logp, "logp"), gradient(a), Memory(stats, 12, "stats"),
                          Memory(workspace, (int64_t)workspace_of(a), "workspace"), ::logits(a), ::ids(a), tokens(a, advantage, "advantage"),
                          tokens(a, old_logp, "old_logp"), tokens(a, ref_logp, "ref_logp"), tokens(a, weight, "weight")}, 4));
  a.advantage = advantage; a.old_logp = old_logp; a.ref_logp = ref_logp; a.weight = weight; a.reduce = reduce;
  a.low = 1.f - clip_low; a.high = 1.f + clip_high; a.kl_coef = kl_coef; a.logp = logp; a.stats = stats; a.ws = workspace;
  return device_status(elas::run_token_loss(a, (hipStream_t)stream), "policy loss launch");
}

size_t elas_preference_loss_workspace_bytes(int64_t N, int64_t pairs) {
  return pairs < 0 || pairs >= kMaxVocab || N < 0 || N >= kMaxValues ? 0 : elas::preference_workspace_bytes(N, pairs);
}

int elas_preference_loss(const float* logp, const float* ref_logp, const void* offsets, int64_t N, int64_t pairs, float beta, float smoothing,
                         uint32_t flags, float* margin, float* dlogp, float* stats, void* workspace, size_t workspace_bytes, void* stream) {
  begin_call();
  if (flags & ~ELAS_IDS_I64) return fail(ELAS_ERR_FLAGS, "flags: only ELAS_IDS_I64 is allowed");
  if (pairs < 0 || pairs >= kMaxVocab) return fail(ELAS_ERR_SHAPE, "pairs=%lld out of range", (long long)pairs);
  if (N < 0 || N >= kMaxValues) return fail(ELAS_ERR_SHAPE, "N=%lld out of range", (long long)N);
  ELAS_CHECK(check_scale(beta, "beta"));
  if (!(smoothing >= 0.f && smoothing <= 1.f)) return fail(ELAS_ERR_SHAPE, "smoothing must be between 0 and 1");
  elas::PreferenceArgs a{};
  a.i64 = (flags & ELAS_IDS_I64) != 0;
  if (pairs > 0) {
    ELAS_CHECK(check_elem_ptr(offsets, a.i64 ? 8 : 4, "offsets"));
    ELAS_CHECK(check_optional_ptr(margin, 4, "margin"));
    if (N > 0) {
      ELAS_CHECK(check_elem_ptr(logp, 4, "logp"));
      ELAS_CHECK(check_optional_ptr(ref_logp, 4, "ref_logp"));
    }
  }
  if (N > 0) ELAS_CHECK(check_optional_ptr(dlogp, 4, "dlogp"));
  ELAS_CHECK(check_elem_ptr(stats, 4, "stats"));
  const size_t need = elas::preference_workspace_bytes(N, pairs);
  ELAS_CHECK(check_workspace(workspace, workspace_bytes, need));
  // (a gradient in logp's place: once, as a result)
  ELAS_CHECK(check_apart({Memory(margin, 4 * pairs, "margin"), Memory(dlogp, 4 * N, "dlogp"), Memory(stats, 12, "stats"),
                          Memory(workspace, (int64_t)need, "workspace"), Memory(logp == dlogp ? nullptr : logp, 4 * N, "logp"),
                          Memory(ref_logp, 4 * N, "ref_logp"), Memory(pairs ? offsets : nullptr, (2 * pairs + 1) * (a.i64 ? 8 : 4), "offsets")}, 4));
  a.N = N; a.pairs = pairs; a.logp = logp; a.ref = ref_logp; a.offsets = offsets; a.beta = beta; a.smoothing = smoothing;
  a.margin = margin; a.dlogp = N > 0 ? dlogp : nullptr; a.stats = stats; a.ws = workspace;
  return device_status(elas::run_preference(a, (hipStream_t)stream), "preference loss launch");
}

}  // extern "C"
