// Host-side declarations shared by the launchers and the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tempo.h"
#include "../../include/tempo_tune.h"

namespace tempo {

// Launch-shape knobs.
enum TuneKey {
  kTuneGeluFwdChunks = 0,       // 8-element chunks per lane (1, 2 or 4)
  kTuneGeluBwdChunks = 1,
  kTuneLnFwdBlocksPerCu = 2,    // cap on workgroups per compute unit
  kTuneLnBwdRowsPerGroup = 3,   // rows each lane group walks (sets the grid and the workspace)
  kTuneAttnFwdBlocksPerCu = 4,  // cap on workgroups per compute unit
  kTuneAttnBwdBlocksPerCu = 5,
  kTuneAttnFwdRows = 6,         // rows a lane group of attn fwd fetches at once (1 or 2)
  kTuneLnFwdRows = 7,           // layernorm_fwd: 1 = one row per lane group at a time, else 2 or 4 by shape
  kTuneAttnFwdMaxPieces = 8,    // attn fwd: pieces per lane above which a row takes 2-4 waves
  kTuneAttnBwdMaxPieces = 9,    // the same for attn bwd
  kTuneLnFwdMaxPieces = 10,     // the same for layernorm_fwd
  kTuneLnBwdMaxPieces = 11,     // and layernorm_bwd
  kTuneLnBwdLoopBlocksPerCu = 12,  // layernorm_bwd: workgroups per CU beyond which they loop
  kTuneGeluFwdSmallGroupsFrom = 13,  // bf16 gelu/silu fwd: Mi elements from which 512-lane groups
  kTuneAttnThreads = 14,        // attn fwd / bwd: lanes per workgroup (64, 128 or 256; at least a row's, two where a forward row takes two waves)
  kTuneGeluF32Threads = 15,     // float32 gelu/silu: lanes per workgroup (64, 128, 256; 1 = per kernel)
  kTuneCount = 16
};
int tune_get(TuneKey k);
int compute_units();

inline tempo_status launch_status() {
  return hipGetLastError() == hipSuccess ? TEMPO_OK : TEMPO_ERR_LAUNCH;
}

// kind: TEMPO_GELU_ERF, TEMPO_GELU_TANH or kActSilu (the activation kernels serve all three).
constexpr int kActSilu = 2;
tempo_status launch_gelu_fwd(const void* x, void* y, uint32_t* mask, int64_t n, tempo_dtype dt,
                             int kind, hipStream_t st);
tempo_status launch_gelu_bwd(const void* dy, const void* y, const uint32_t* mask, void* dx,
                             int64_t n, tempo_dtype dt, int kind, hipStream_t st);
tempo_status launch_layernorm_fwd(const void* x, const float* gamma, const float* beta, void* y,
                                  float* rstd, float* mean, int64_t N, int64_t M, float eps,
                                  tempo_dtype dt, hipStream_t st);
size_t layernorm_bwd_workspace_bytes(int64_t N, int64_t M, tempo_dtype dt);
// TEMPO_ERR_WORKSPACE if workspace_bytes is less than this call's launch plan needs.
tempo_status launch_layernorm_bwd(const void* dy, const void* y, const float* gamma,
                                  const float* beta, const float* rstd, void* dx, float* dgamma,
                                  float* dbeta, float* workspace, size_t workspace_bytes,
                                  int64_t N, int64_t M, tempo_dtype dt, hipStream_t st);

// Device address of the current device's static scratch array (TEMPO_STATIC_SCRATCH_BYTES).
tempo_status static_scratch(void** ptr);
tempo_status launch_attn_fwd(const void* scores, const int32_t* key_len, int causal, void* probs,
                             void* out, uint32_t* keep_bits, int64_t B, int64_t A, int64_t Sq,
                             int64_t Sk, float p, uint64_t seed, uint64_t offset, tempo_dtype dt,
                             hipStream_t st);
tempo_status launch_attn_bwd(const void* dout, const void* probs, const uint32_t* keep_bits,
                             void* dscores, void* out_re, int64_t B, int64_t A, int64_t Sq,
                             int64_t Sk, float p, tempo_dtype dt, hipStream_t st);
tempo_status launch_attn_bwd_bytemask(const void* dout, const void* probs,
                                      const uint8_t* keep_bytes, void* dscores, void* out_re,
                                      int64_t B, int64_t A, int64_t Sq, int64_t Sk, float p,
                                      tempo_dtype dt, hipStream_t st);
tempo_status launch_attn_bwd_regen(const void* dout, const void* probs, void* dscores,
                                   void* out_re, int64_t B, int64_t A, int64_t Sq, int64_t Sk,
                                   float p, uint64_t seed, uint64_t offset, tempo_dtype dt,
                                   hipStream_t st);
// axes: null, or which axis each pair turns by; back: the other way round.
struct RotaryAxes {
  const uint8_t* of_pairs;
  int count;
  int64_t stride;  // of positions
};
tempo_status launch_rotary(const tempo_rotary_heads* q, const tempo_rotary_heads* k, const double* freqs,
                           const tempo_rotary_positions* at, const RotaryAxes* axes, int64_t B, int64_t S, int64_t D, int64_t R,
                           tempo_rotary_layout layout, float scale, bool back, tempo_dtype dt, hipStream_t st);
// What the two entry points of the gated unit take; each looks at its own.
struct GluCall {
  const void *x, *w, *bias;
  void *gu, *h;
  const void* dh;
  void *dgu, *dx, *dw, *dbias;
  void* workspace;
  size_t workspace_bytes;
  int64_t T, H, F;
  tempo_glu_kind kind;
};
bool glu_takes(int64_t T, int64_t H, int64_t F);
size_t glu_workspace_bytes(int64_t T, int64_t H, int64_t F, tempo_dtype dt, bool back);
tempo_status launch_glu_fwd(const GluCall& c, tempo_dtype dt, hipStream_t st);
tempo_status launch_glu_bwd(const GluCall& c, tempo_dtype dt, hipStream_t st);
// What the two entry points of the residual norm take; each looks at its own.
struct ResidualCall {
  const void *x, *f, *y, *dy, *dh;
  void *to_y, *h, *dx, *df;
  const float* gate;
  int64_t groups;
  const tempo_norm *post, *pre;
  float *dgate, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
  float alpha, beta;
  void* workspace;
  size_t workspace_bytes;
  int64_t N, M;
};
bool residual_norm_takes(const ResidualCall& c, tempo_dtype dt);
size_t residual_norm_workspace_bytes(const ResidualCall& c, tempo_dtype dt);
tempo_status launch_residual_norm_fwd(const ResidualCall& c, tempo_dtype dt, hipStream_t st);
tempo_status launch_residual_norm_bwd(const ResidualCall& c, tempo_dtype dt, hipStream_t st);
// What the two entry points of window attention take; each looks at its own.
struct WindowCall {
  const tempo_attn_heads *q, *k, *v, *out, *dout, *dq, *dk, *dv;
  float* lse;
  const int32_t *key_len, *query_start;
  void* workspace;
  size_t workspace_bytes;
  int64_t B, Sq, Sk, heads, kv_heads, D, window, sinks;
  float scale;
};
bool window_attn_takes(const WindowCall& c);
size_t window_attn_workspace_bytes(const WindowCall& c, tempo_dtype dt, bool back);
tempo_status launch_window_attn_fwd(const WindowCall& c, tempo_dtype dt, hipStream_t st);
tempo_status launch_window_attn_bwd(const WindowCall& c, tempo_dtype dt, hipStream_t st);
tempo_status launch_mask_bits_to_bytes(const uint32_t* bits, uint8_t* bytes, int64_t n,
                                       hipStream_t st);
tempo_status launch_mask_bytes_to_bits(const uint8_t* bytes, uint32_t* bits, int64_t n,
                                       hipStream_t st);

}  // namespace tempo
