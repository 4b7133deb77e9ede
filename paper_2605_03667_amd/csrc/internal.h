// Internal host-side interface between the C-ABI layer (api.hip) and the
// kernel translation units.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace elas {

// Row pitches of the compressed 2:4 layout: rows are padded to a multiple of
// 64 features (32 kept values, 8 metadata bytes per 64 features).
inline int64_t vals_ld(int64_t n) { return 32 * ((n + 63) / 64); }
inline int64_t meta_ld(int64_t n) { return 8 * ((n + 63) / 64); }
inline int64_t pad64(int64_t n) { return 64 * ((n + 63) / 64); }
inline int64_t pad256(int64_t n) { return 256 * ((n + 255) / 256); }

// api.hip: errors of the calling thread.  begin_call starts an entry point, fail
// records a message for elas_last_error and returns its code, check_ptr checks one
// device pointer (NULL, 16-byte alignment), device_status turns a launch sequence's
// result, or (ELAS_DEBUG_SYNC) the first failure seen after one of its kernels, into
// a status.
void begin_call();
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int check_ptr(const void* p, const char* name);
int device_status(hipError_t e, const char* what);
#define ELAS_CHECK(expr)            \
  do {                              \
    int rc_ = (expr);               \
    if (rc_ != ELAS_OK) return rc_; \
  } while (0)

// timing.hip: brackets one launch with events when timing is enabled, and
// synchronises after it in the ELAS_DEBUG_SYNC mode (the first failure of
// the calling thread is kept with its kernel tag until the next reset)
bool timing_enabled();
void debug_sync_reset();
hipError_t debug_sync_error(const char** tag);
class TimedLaunch {
 public:
  TimedLaunch(const char* tag, hipStream_t stream);
  ~TimedLaunch();
  TimedLaunch(const TimedLaunch&) = delete;
  TimedLaunch& operator=(const TimedLaunch&) = delete;

 private:
  const char* tag_;
  hipStream_t stream_;
  hipEvent_t start_ = nullptr, stop_ = nullptr;
};

// sparsify.hip
hipError_t launch_sparsify24(const uint16_t* h, int64_t M, int64_t N, bool raw,
                             uint16_t* vals, uint8_t* meta, hipStream_t stream);

// Arguments of one forward or backward call (sizes already validated).
struct FfnArgs {
  int64_t T, d, F, r;
  const uint16_t *x, *U_up, *V_up, *U_down, *V_down;
  // forward outputs / backward inputs
  uint16_t* y;
  const uint16_t* P_in;
  uint16_t* P;
  uint16_t* s_vals;
  uint8_t* s_meta;
  uint16_t* Z;
  // backward
  const uint16_t* dy;
  uint16_t* dx;
  float *dU_up, *dV_up, *dU_down, *dV_down;
  void* ws;
  bool dense;   // activations dense [T x d_ff] (no 2:4 selection)
  bool ste;     // backward: straight-through estimator through the selection
  bool ab;      // forward: factors given as U_up^T, V_up^T, U_down^T, V_down^T
  bool lean;    // forward: the smallest workspace (no weights in fragment order)
  int fused;    // sparse forward: 1 one fused launch, else (0 default, 2 requested) four kernels
};

// fused.hip: the one-launch sparse forward for compact factor shapes
bool fused_fwd_supported(int64_t d, int64_t r);
hipError_t run_fused_fwd(const uint16_t* x, const uint16_t* U_upT, const uint16_t* V_upT, const uint16_t* U_downT,
                         const uint16_t* V_downT, int64_t T, int64_t d, int64_t F, int64_t r, int64_t F_rows,
                         int64_t ld_ud, uint16_t* y, uint16_t* P, uint16_t* s_vals, uint8_t* s_meta, uint16_t* Z,
                         hipStream_t stream);

// Arguments of one norm join, forward or backward (include/elas_train.h; sizes
// validated, T > 0 in the forward).
struct NormJoinArgs {
  int64_t T, d;
  const void* h;            // forward: h; backward: h_out
  const uint16_t *b, *gate, *w_post, *w_pre;
  float res_scale, block_scale, eps;
  bool res_f32, gate_token;
  void* h_out;              // forward outputs
  uint16_t* n;
  const void* dh_out;       // backward inputs and outputs
  const uint16_t* dn;
  void* dh;
  uint16_t* db;
  void* dgate;
  float *dw_post, *dw_pre;
  void* ws;
};

// norm_join.hip
size_t norm_join_bwd_workspace_bytes(int64_t T, int64_t d);
hipError_t run_norm_join_fwd(const NormJoinArgs& a, hipStream_t stream);
hipError_t run_norm_join_bwd(const NormJoinArgs& a, hipStream_t stream);

// Arguments of the embedding, forward or backward.
struct EmbedArgs {
  int64_t T, V, d;
  const void* ids;
  bool ids_i64, res_f32, add;
  float scale;
  const uint16_t* table;    // forward
  void* x;
  const void* dx;           // backward
  float* dtable;
  void* ws;
};

// embed.hip
size_t embed_bwd_workspace_bytes(int64_t T, int64_t V, int64_t d, bool add);
hipError_t run_embed_fwd(const EmbedArgs& a, hipStream_t stream);
hipError_t run_embed_bwd(const EmbedArgs& a, hipStream_t stream);

// grad_clip.hip: out and factor outputs NULL / clip false: the norm alone
size_t grad_workspace_bytes(int64_t n);
hipError_t run_grad_norm(const void* const* grads, void* const* out, const int64_t* numel, const int32_t* dtype, int64_t n,
                         bool clip, float max_norm, float* stats, void* ws, hipStream_t stream);

// Arguments of the calls on logits (include/elas_loss.h).
struct LogitsArgs {
  enum Kind { LOGP, TOKEN, POLICY };
  Kind kind;
  int64_t T, V, ld, ld_out;
  const void *logits, *ids;
  bool f32, ids_i64;
  float scale, reduce;
  const float *weight, *advantage, *old_logp, *ref_logp;
  float z_coef, low, high, kl_coef;   // low, high: the clamp's bounds
  float *logp, *lse, *stats;
  void* dlogits;
  const float *dlogp, *dlse, *lse_in;   // backward
  void* ws;
};

// token_loss.hip
size_t token_loss_workspace_bytes(int64_t T, int64_t V, bool f32);
hipError_t run_token_loss(const LogitsArgs& a, hipStream_t stream);
hipError_t run_token_logp_bwd(const LogitsArgs& a, hipStream_t stream);

// Arguments of the preference loss.
struct PreferenceArgs {
  int64_t N, pairs;
  const float *logp, *ref;
  const void* offsets;
  bool i64;
  float beta, smoothing;
  float *margin, *dlogp, *stats;
  void* ws;
};

// preference.hip
size_t preference_workspace_bytes(int64_t N, int64_t pairs);
hipError_t run_preference(const PreferenceArgs& a, hipStream_t stream);

// Arguments of a step of AdamW (include/elas_adamw.h); host arrays of n.
struct AdamwArgs {
  void* const* params;
  const void* const* grads;
  uint16_t* const* copies;
  const int64_t* numel;
  const int32_t *param_dtype, *grad_dtype;
  const float* decay;
  int64_t n;
  bool eight;
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t* step;
  double rate, beta1, beta2, eps, max_norm;
  const float *rate_factor, *norm;
  void* ws;
};

// adamw.hip
size_t adamw_workspace_bytes();
hipError_t run_adamw(const AdamwArgs& a, hipStream_t stream);
hipError_t run_adam8_values(const uint8_t* codes, const float* scale, int64_t blocks, bool second, bool f32, void* out, hipStream_t stream);

// ffn.hip
size_t spmm_workspace_bytes(int64_t K, int64_t N, int b_layout);
size_t fwd_workspace_bytes(int64_t T, int64_t d, int64_t F, int64_t r, bool dense, bool ab, bool lean = false);
size_t bwd_workspace_bytes(int64_t T, int64_t d, int64_t F, int64_t r, bool dense, bool ste);
hipError_t run_spmm24(const uint16_t* a_vals, const uint8_t* a_meta, int64_t M, int64_t K,
                      const uint16_t* b, int64_t N, bool b_is_nk, uint16_t* c, void* ws,
                      hipStream_t stream);
hipError_t run_fwd(const FfnArgs& a, hipStream_t stream);
hipError_t run_bwd(const FfnArgs& a, hipStream_t stream);
hipError_t run_fullrank_fwd(const uint16_t* x, const uint16_t* W_up, const uint16_t* W_down, int64_t T,
                            int64_t d, int64_t F, uint16_t* y, uint16_t* S, hipStream_t stream);

}  // namespace elas
