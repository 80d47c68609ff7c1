// C ABI of libtempo: argument validation, then one launcher per entry point.
#include <atomic>
#include <cmath>

#include "tempo_device.h"
#include "tempo_host.h"

namespace tempo {

static std::atomic<int> g_tune[kTuneCount] = {
    {4},      // gelu fwd: chunks per lane
    {2},      // gelu bwd: chunks per lane
    {3},      // layernorm fwd: workgroups per CU (beyond that they loop with prefetch)
    {4},      // layernorm bwd: rows per lane group
    {65536},  // attention fwd: workgroups per CU (65536 = one row per lane group)
    {65536},  // attention bwd: workgroups per CU
    {2},      // attention fwd: rows per lane group
    {2},      // layernorm fwd: rows per lane group
    {4},      // attention fwd: most pieces per lane of a one-wave row
    {4},      // attention bwd: the same
    {4},      // layernorm fwd: the same
    {3},      // layernorm bwd: the same (3: rows of 4 pieces per lane would keep their parameters in LDS)
    {1},      // layernorm bwd: workgroups per CU beyond which they loop with prefetch
    {24},     // bf16 gelu/silu fwd: Mi elements from which workgroups have 512 lanes
    {128},    // attention fwd / bwd: lanes per workgroup
    {1},      // float32 gelu/silu: lanes per workgroup (1: chosen per kernel)
};

int tune_get(TuneKey k) { return g_tune[k].load(std::memory_order_relaxed); }

int compute_units() {
  static std::atomic<int> cached{0};
  int v = cached.load(std::memory_order_relaxed);
  if (v > 0) return v;
  int dev = 0;
  hipDeviceProp_t prop;
  if (hipGetDevice(&dev) != hipSuccess || hipGetDeviceProperties(&prop, dev) != hipSuccess ||
      prop.multiProcessorCount <= 0) {
    (void)hipGetLastError();
    return 256;
  }
  cached.store(prop.multiProcessorCount, std::memory_order_relaxed);
  return prop.multiProcessorCount;
}

static bool dtype_ok(tempo_dtype dt) { return dt == TEMPO_F32 || dt == TEMPO_BF16; }
static bool kind_ok(tempo_gelu_kind k) { return k == TEMPO_GELU_ERF || k == TEMPO_GELU_TANH; }
static bool aligned_to(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
static bool prob_ok(float p) { return p >= 0.0f && p < 1.0f; }  // false for NaN

// A tensor has at most 2^40 elements (terabytes: far beyond device memory), so that no product
// of sizes and no grid computed from one can overflow.  Sizes are known to be >= 0 here.
constexpr int64_t kMaxElements = int64_t{1} << 40;
static bool count_ok(int64_t a, int64_t b = 1, int64_t c = 1, int64_t d = 1) {
  int64_t n = a;
  for (int64_t f : {b, c, d}) {
    if (f != 0 && n > kMaxElements / f) return false;
    n *= f;
  }
  return n <= kMaxElements;
}

// Workgroups of the yardstick kernels are single waves: measured on 1 GiB tensors, one-wave
// workgroups move 3.5 % (one read, one write) to 6 % (two and two) more than four-wave ones.
constexpr int kCopyThreads = kWave;

// Plain streaming copy, 16 bytes per lane and access: the reference point for what the memory
// system delivers to a kernel that does nothing else, and the known-size kernel against which
// hardware byte counters are calibrated.
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(const u32x4* __restrict__ src,
                                                            u32x4* __restrict__ dst, int64_t n16) {
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kCopyThreads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kCopyThreads + threadIdx.x; i < n16;
       i += stride)
    __builtin_nontemporal_store(__builtin_nontemporal_load(src + i), dst + i);
}

// The same with several streams: reads NR tensors, combines them (XOR, so that no load can be
// dropped) and writes NW tensors, one 16-byte piece per lane and stream, a full grid of
// short-lived workgroups.  What the memory system delivers depends on the mix of read and
// write streams (two reads and two writes reach less than one and one), so each layer kernel
// is held against the plain kernel of its own mix.
template <int NR, int NW>
__global__ __launch_bounds__(kCopyThreads) void copy_streams_kernel(const u32x4* r0, const u32x4* r1,
                                                           const u32x4* r2, u32x4* w0, u32x4* w1,
                                                           int64_t n16) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kCopyThreads + threadIdx.x;
  if (i >= n16) return;
  u32x4 v = __builtin_nontemporal_load(r0 + i);
  if constexpr (NR >= 2) v ^= __builtin_nontemporal_load(r1 + i);
  if constexpr (NR >= 3) v ^= __builtin_nontemporal_load(r2 + i);
  __builtin_nontemporal_store(v, w0 + i);
  if constexpr (NW >= 2) __builtin_nontemporal_store(v + 1u, w1 + i);
}

}  // namespace tempo

using namespace tempo;

extern "C" {

const char* tempo_status_string(tempo_status s) {
  switch (s) {
    case TEMPO_OK: return "ok";
    case TEMPO_ERR_INVALID_ARG: return "invalid argument";
    case TEMPO_ERR_UNSUPPORTED: return "unsupported (pointer not 16-byte aligned)";
    case TEMPO_ERR_WORKSPACE: return "workspace too small";
    case TEMPO_ERR_LAUNCH: return "kernel launch failed";
  }
  return "unknown status";
}

int tempo_version(void) { return 100; }

TEMPO_API int tempo_set_launch_param(int key, int value) {
  if (key < 0 || key >= kTuneCount || value < 1 || value > 65536) return TEMPO_ERR_INVALID_ARG;
  g_tune[key].store(value, std::memory_order_relaxed);
  return TEMPO_OK;
}

TEMPO_API int tempo_get_launch_param(int key) {
  if (key < 0 || key >= kTuneCount) return -1;
  return tune_get(static_cast<TuneKey>(key));
}

tempo_status tempo_copy(const void* src, void* dst, int64_t nbytes, int blocks_per_cu,
                        void* hip_stream) {
  if (nbytes < 0 || (nbytes & 15) != 0 || blocks_per_cu < 1) return TEMPO_ERR_INVALID_ARG;
  if (nbytes == 0) return TEMPO_OK;
  if (!src || !dst) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(src) || !aligned16(dst)) return TEMPO_ERR_UNSUPPORTED;
  const int64_t n16 = nbytes / 16;
  const int64_t want = (n16 + kCopyThreads - 1) / kCopyThreads;
  const int64_t cap = static_cast<int64_t>(compute_units()) * blocks_per_cu;
  hipLaunchKernelGGL(copy_kernel, dim3(static_cast<unsigned>(want < cap ? want : cap)),
                     dim3(kCopyThreads), 0,
                     static_cast<hipStream_t>(hip_stream), static_cast<const u32x4*>(src),
                     static_cast<u32x4*>(dst), n16);
  return launch_status();
}

tempo_status tempo_copy_streams(const void* const* reads, int n_reads, void* const* writes,
                                int n_writes, int64_t nbytes, void* hip_stream) {
  if (nbytes < 0 || (nbytes & 15) != 0 || n_reads < 1 || n_reads > 3 || n_writes < 1 ||
      n_writes > 2 || nbytes / 16 > (int64_t{1} << 31) * kCopyThreads)
    return TEMPO_ERR_INVALID_ARG;
  if (nbytes == 0) return TEMPO_OK;
  if (!reads || !writes) return TEMPO_ERR_INVALID_ARG;
  const u32x4* r[3] = {nullptr, nullptr, nullptr};
  u32x4* w[2] = {nullptr, nullptr};
  for (int i = 0; i < n_reads; ++i) {
    if (!reads[i]) return TEMPO_ERR_INVALID_ARG;
    if (!aligned16(reads[i])) return TEMPO_ERR_UNSUPPORTED;
    r[i] = static_cast<const u32x4*>(reads[i]);
  }
  for (int i = 0; i < n_writes; ++i) {
    if (!writes[i]) return TEMPO_ERR_INVALID_ARG;
    if (!aligned16(writes[i])) return TEMPO_ERR_UNSUPPORTED;
    w[i] = static_cast<u32x4*>(writes[i]);
  }
  const int64_t n16 = nbytes / 16;
  const dim3 grid(static_cast<unsigned>((n16 + kCopyThreads - 1) / kCopyThreads));
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
#define TEMPO_LAUNCH(NR, NW)                                                                 \
  hipLaunchKernelGGL((copy_streams_kernel<NR, NW>), grid, dim3(kCopyThreads), 0, st, r[0], r[1], \
                     r[2], w[0], w[1], n16)
  switch (n_reads * 10 + n_writes) {
    case 11: TEMPO_LAUNCH(1, 1); break;
    case 12: TEMPO_LAUNCH(1, 2); break;
    case 21: TEMPO_LAUNCH(2, 1); break;
    case 22: TEMPO_LAUNCH(2, 2); break;
    case 31: TEMPO_LAUNCH(3, 1); break;
    default: TEMPO_LAUNCH(3, 2); break;
  }
#undef TEMPO_LAUNCH
  return launch_status();
}

tempo_status tempo_gelu_fwd(const void* x, void* y, uint32_t* mask, int64_t n, tempo_dtype dt,
                            tempo_gelu_kind kind, void* hip_stream) {
  if (n < 0 || !count_ok(n) || !dtype_ok(dt) || !kind_ok(kind)) return TEMPO_ERR_INVALID_ARG;
  if (n == 0) return TEMPO_OK;
  if (!x || !y || !mask) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(y) || !aligned16(mask)) return TEMPO_ERR_UNSUPPORTED;
  return launch_gelu_fwd(x, y, mask, n, dt, kind, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_gelu_bwd(const void* dy, const void* y, const uint32_t* mask, void* dx,
                            int64_t n, tempo_dtype dt, tempo_gelu_kind kind, void* hip_stream) {
  if (n < 0 || !count_ok(n) || !dtype_ok(dt) || !kind_ok(kind)) return TEMPO_ERR_INVALID_ARG;
  if (n == 0) return TEMPO_OK;
  if (!dy || !y || !mask || !dx) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(dy) || !aligned16(y) || !aligned16(mask) || !aligned16(dx))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_gelu_bwd(dy, y, mask, dx, n, dt, kind, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_silu_fwd(const void* x, void* y, uint32_t* mask, int64_t n, tempo_dtype dt,
                            void* hip_stream) {
  if (n < 0 || !count_ok(n) || !dtype_ok(dt)) return TEMPO_ERR_INVALID_ARG;
  if (n == 0) return TEMPO_OK;
  if (!x || !y || !mask) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(y) || !aligned16(mask)) return TEMPO_ERR_UNSUPPORTED;
  return launch_gelu_fwd(x, y, mask, n, dt, kActSilu, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_silu_bwd(const void* dy, const void* y, const uint32_t* mask, void* dx,
                            int64_t n, tempo_dtype dt, void* hip_stream) {
  if (n < 0 || !count_ok(n) || !dtype_ok(dt)) return TEMPO_ERR_INVALID_ARG;
  if (n == 0) return TEMPO_OK;
  if (!dy || !y || !mask || !dx) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(dy) || !aligned16(y) || !aligned16(mask) || !aligned16(dx))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_gelu_bwd(dy, y, mask, dx, n, dt, kActSilu, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_layernorm_fwd(const void* x, const float* gamma, const float* beta, void* y,
                                 float* rstd, float* mean, int64_t N, int64_t M, float eps,
                                 tempo_dtype dt, void* hip_stream) {
  if (N < 0 || M < 0 || !dtype_ok(dt) || !(eps >= 0.0f) || M > INT32_MAX || !count_ok(N, M))
    return TEMPO_ERR_INVALID_ARG;
  if (N == 0 || M == 0) return TEMPO_OK;
  if (!x || !gamma || !beta || !y || !rstd) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(gamma) || !aligned16(beta) || !aligned16(y) ||
      !aligned16(rstd) || !aligned16(mean))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_layernorm_fwd(x, gamma, beta, y, rstd, mean, N, M, eps, dt,
                              static_cast<hipStream_t>(hip_stream));
}

size_t tempo_layernorm_bwd_workspace_bytes(int64_t N, int64_t M) {
  if (N <= 0 || M <= 0 || M > INT32_MAX || !count_ok(N, M)) return 0;
  // the larger of the two dtypes' needs, so one query serves both
  const size_t a = layernorm_bwd_workspace_bytes(N, M, TEMPO_F32);
  const size_t b = layernorm_bwd_workspace_bytes(N, M, TEMPO_BF16);
  return a > b ? a : b;
}

tempo_status tempo_layernorm_bwd(const void* dy, const void* y, const float* gamma,
                                 const float* beta, const float* rstd, void* dx, float* dgamma,
                                 float* dbeta, void* workspace, size_t workspace_bytes, int64_t N,
                                 int64_t M, tempo_dtype dt, void* hip_stream) {
  if (N < 0 || M < 0 || !dtype_ok(dt) || M > INT32_MAX || !count_ok(N, M))
    return TEMPO_ERR_INVALID_ARG;
  if (N == 0 || M == 0) return TEMPO_OK;
  if (!dy || !y || !gamma || !beta || !rstd || !dx || !dgamma || !dbeta || !workspace)
    return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(dy) || !aligned16(y) || !aligned16(gamma) || !aligned16(beta) ||
      !aligned16(rstd) || !aligned16(dx) || !aligned16(dgamma) || !aligned16(dbeta) ||
      !aligned16(workspace))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_layernorm_bwd(dy, y, gamma, beta, rstd, dx, dgamma, dbeta,
                              static_cast<float*>(workspace), workspace_bytes, N, M, dt,
                              static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_layernorm_bwd_static(const void* dy, const void* y, const float* gamma,
                                        const float* beta, const float* rstd, void* dx,
                                        float* dgamma, float* dbeta, int64_t N, int64_t M,
                                        tempo_dtype dt, void* hip_stream) {
  if (N < 0 || M < 0 || !dtype_ok(dt) || M > INT32_MAX || !count_ok(N, M))
    return TEMPO_ERR_INVALID_ARG;
  if (N == 0 || M == 0) return TEMPO_OK;
  if (!dy || !y || !gamma || !beta || !rstd || !dx || !dgamma || !dbeta)
    return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(dy) || !aligned16(y) || !aligned16(gamma) || !aligned16(beta) ||
      !aligned16(rstd) || !aligned16(dx) || !aligned16(dgamma) || !aligned16(dbeta))
    return TEMPO_ERR_UNSUPPORTED;
  void* ptr = nullptr;
  const tempo_status got = static_scratch(&ptr);
  if (got != TEMPO_OK) return got;
  // the launcher checks the plan's need against the array's size before it launches anything
  return launch_layernorm_bwd(dy, y, gamma, beta, rstd, dx, dgamma, dbeta,
                              static_cast<float*>(ptr), TEMPO_STATIC_SCRATCH_BYTES, N, M, dt,
                              static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_attn_softmax_dropout_fwd(const void* scores, const int32_t* key_len, int causal,
                                            void* probs, void* out, uint32_t* keep_bits, int64_t B,
                                            int64_t A, int64_t Sq, int64_t Sk, float p,
                                            uint64_t seed, uint64_t offset, tempo_dtype dt,
                                            void* hip_stream) {
  if (B < 0 || A < 0 || Sq < 0 || Sk < 0 || !dtype_ok(dt) || !prob_ok(p) || Sq > INT32_MAX ||
      Sk > INT32_MAX || !count_ok(B, A, Sq, Sk) || B * A > INT32_MAX)
    return TEMPO_ERR_INVALID_ARG;
  if (B == 0 || A == 0 || Sq == 0 || Sk == 0) return TEMPO_OK;
  if (!scores || !probs || !keep_bits) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(scores) || !aligned16(probs) || !aligned16(out) || !aligned16(keep_bits))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_attn_fwd(scores, key_len, causal, probs, out, keep_bits, B, A, Sq, Sk, p, seed,
                         offset, dt, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_attn_softmax_dropout_bwd(const void* dout, const void* probs,
                                            const uint32_t* keep_bits, void* dscores,
                                            void* out_recomputed, int64_t B, int64_t A, int64_t Sq,
                                            int64_t Sk, float p, tempo_dtype dt, void* hip_stream) {
  if (B < 0 || A < 0 || Sq < 0 || Sk < 0 || !dtype_ok(dt) || !prob_ok(p) || Sq > INT32_MAX ||
      Sk > INT32_MAX || !count_ok(B, A, Sq, Sk) || B * A > INT32_MAX)
    return TEMPO_ERR_INVALID_ARG;
  if (B == 0 || A == 0 || Sq == 0 || Sk == 0) return TEMPO_OK;
  if (!dout || !probs || !keep_bits || !dscores) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(dout) || !aligned16(probs) || !aligned16(keep_bits) || !aligned16(dscores) ||
      !aligned16(out_recomputed))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_attn_bwd(dout, probs, keep_bits, dscores, out_recomputed, B, A, Sq, Sk, p, dt,
                         static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_attn_softmax_dropout_bwd_bytemask(const void* dout, const void* probs,
                                                     const uint8_t* keep_bytes, void* dscores,
                                                     void* out_recomputed, int64_t B, int64_t A,
                                                     int64_t Sq, int64_t Sk, float p,
                                                     tempo_dtype dt, void* hip_stream) {
  if (B < 0 || A < 0 || Sq < 0 || Sk < 0 || !dtype_ok(dt) || !prob_ok(p) || Sq > INT32_MAX ||
      Sk > INT32_MAX || !count_ok(B, A, Sq, Sk) || B * A > INT32_MAX)
    return TEMPO_ERR_INVALID_ARG;
  if (B == 0 || A == 0 || Sq == 0 || Sk == 0) return TEMPO_OK;
  if (!dout || !probs || !keep_bytes || !dscores) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(dout) || !aligned16(probs) || !aligned16(keep_bytes) || !aligned16(dscores) ||
      !aligned16(out_recomputed))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_attn_bwd_bytemask(dout, probs, keep_bytes, dscores, out_recomputed, B, A, Sq, Sk,
                                  p, dt, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_attn_softmax_dropout_bwd_regen(const void* dout, const void* probs,
                                                  void* dscores, void* out_recomputed, int64_t B,
                                                  int64_t A, int64_t Sq, int64_t Sk, float p,
                                                  uint64_t seed, uint64_t offset, tempo_dtype dt,
                                                  void* hip_stream) {
  if (B < 0 || A < 0 || Sq < 0 || Sk < 0 || !dtype_ok(dt) || !prob_ok(p) || Sq > INT32_MAX ||
      Sk > INT32_MAX || !count_ok(B, A, Sq, Sk) || B * A > INT32_MAX)
    return TEMPO_ERR_INVALID_ARG;
  if (B == 0 || A == 0 || Sq == 0 || Sk == 0) return TEMPO_OK;
  if (!dout || !probs || !dscores) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(dout) || !aligned16(probs) || !aligned16(dscores) || !aligned16(out_recomputed))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_attn_bwd_regen(dout, probs, dscores, out_recomputed, B, A, Sq, Sk, p, seed,
                               offset, dt, static_cast<hipStream_t>(hip_stream));
}

static bool rotary_side_ok(const tempo_rotary_heads* h, int64_t B, int64_t S, int64_t D) {
  const int64_t sizes[] = {B, S, h->heads};
  const int64_t in[] = {h->x_batch, h->x_token, h->x_head}, out[] = {h->y_batch, h->y_token, h->y_head};
  int64_t last_in = D, last_out = D;
  for (int i = 0; i < 3; ++i) {
    if (in[i] < 0 || out[i] < 0 || !count_ok(sizes[i], in[i]) || !count_ok(sizes[i], out[i])) return false;
    if (sizes[i] > 1 && (out[i] == 0 || (h->x == h->y && in[i] != out[i]))) return false;
    last_in += sizes[i] * in[i];
    last_out += sizes[i] * out[i];
  }
  return last_in <= kMaxElements && last_out <= kMaxElements;
}
static tempo_status rotary(const tempo_rotary_heads* q, const tempo_rotary_heads* k, const double* freqs,
                           const tempo_rotary_positions* at, const RotaryAxes* axes, int64_t B, int64_t S, int64_t D, int64_t R,
                           tempo_rotary_layout layout, float scale, bool back, tempo_dtype dt, void* hip_stream) {
  constexpr int64_t most = int64_t{1} << 24;  // elements of a token
  if (!q || !at || B < 0 || S < 0 || D < 0 || q->heads < 0 || (k && k->heads < 0) || !dtype_ok(dt) ||
      (layout != TEMPO_ROTARY_HALF && layout != TEMPO_ROTARY_INTERLEAVED))
    return TEMPO_ERR_INVALID_ARG;
  if (R < 2 || R % 2 != 0 || R > D || D > most || q->heads > most || (k && k->heads > most) ||
      (q->heads + (k ? k->heads : 0)) * D > most || !count_ok(B, S) || B * S > INT32_MAX)
    return TEMPO_ERR_INVALID_ARG;
  if (!rotary_side_ok(q, B, S, D) || (k && !rotary_side_ok(k, B, S, D))) return TEMPO_ERR_INVALID_ARG;
  if (at->start < -(int64_t{1} << 53) || at->start > int64_t{1} << 53) return TEMPO_ERR_INVALID_ARG;
  if (at->positions && ((at->bits != 32 && at->bits != 64) || at->batch_stride < 0 || at->token_stride < 0 ||
                        !count_ok(B, at->batch_stride) || !count_ok(S, at->token_stride)))
    return TEMPO_ERR_INVALID_ARG;
  if (axes && (axes->count < 1 || axes->count > TEMPO_ROTARY_MOST_AXES || axes->stride < 0 || !count_ok(axes->count, axes->stride)))
    return TEMPO_ERR_INVALID_ARG;
  if (k && k->heads == 0) k = nullptr;
  if (k && q->heads == 0) q = k, k = nullptr;
  if (B == 0 || S == 0 || q->heads == 0) return TEMPO_OK;
  if (!q->x || !q->y || !freqs || (k && (!k->x || !k->y))) return TEMPO_ERR_INVALID_ARG;
  if (axes && (!axes->of_pairs || !at->positions)) return TEMPO_ERR_INVALID_ARG;
  const uintptr_t element = dt == TEMPO_F32 ? 4 : 2;
  if (!aligned_to(q->x, element) || !aligned_to(q->y, element) || (k && (!aligned_to(k->x, element) || !aligned_to(k->y, element))) ||
      !aligned_to(freqs, 8) || (at->positions && !aligned_to(at->positions, at->bits / 8)))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_rotary(q, k, freqs, at, axes, B, S, D, R, layout, scale, back, dt, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_rotary_fwd(const tempo_rotary_heads* q, const tempo_rotary_heads* k, const double* freqs,
                              const tempo_rotary_positions* positions, int64_t B, int64_t S, int64_t D, int64_t R,
                              tempo_rotary_layout layout, float scale, tempo_dtype dt, void* hip_stream) {
  return rotary(q, k, freqs, positions, nullptr, B, S, D, R, layout, scale, false, dt, hip_stream);
}

tempo_status tempo_rotary_bwd(const tempo_rotary_heads* dq, const tempo_rotary_heads* dk, const double* freqs,
                              const tempo_rotary_positions* positions, int64_t B, int64_t S, int64_t D, int64_t R,
                              tempo_rotary_layout layout, float scale, tempo_dtype dt, void* hip_stream) {
  return rotary(dq, dk, freqs, positions, nullptr, B, S, D, R, layout, scale, true, dt, hip_stream);
}

tempo_status tempo_rotary_axes_fwd(const tempo_rotary_heads* q, const tempo_rotary_heads* k, const double* freqs, const uint8_t* axes,
                                   int n_axes, const tempo_rotary_positions* positions, int64_t axis_stride, int64_t B, int64_t S,
                                   int64_t D, int64_t R, tempo_rotary_layout layout, float scale, tempo_dtype dt, void* hip_stream) {
  const RotaryAxes a{axes, n_axes, axis_stride};
  return rotary(q, k, freqs, positions, &a, B, S, D, R, layout, scale, false, dt, hip_stream);
}

tempo_status tempo_rotary_axes_bwd(const tempo_rotary_heads* dq, const tempo_rotary_heads* dk, const double* freqs, const uint8_t* axes,
                                   int n_axes, const tempo_rotary_positions* positions, int64_t axis_stride, int64_t B, int64_t S,
                                   int64_t D, int64_t R, tempo_rotary_layout layout, float scale, tempo_dtype dt, void* hip_stream) {
  const RotaryAxes a{axes, n_axes, axis_stride};
  return rotary(dq, dk, freqs, positions, &a, B, S, D, R, layout, scale, true, dt, hip_stream);
}

static bool glu_ok(int64_t T, int64_t H, int64_t F, tempo_glu_kind kind, tempo_dtype dt) {
  return T >= 0 && H >= 0 && F >= 0 && dtype_ok(dt) && kind >= TEMPO_GLU_SILU && kind <= TEMPO_GLU_GELU_TANH &&
         count_ok(T, F, 2) && count_ok(T, H) && count_ok(F, H, 2);
}

size_t tempo_glu_fwd_workspace_bytes(int64_t T, int64_t H, int64_t F, tempo_dtype dt) {
  return glu_ok(T, H, F, TEMPO_GLU_SILU, dt) && glu_takes(T, H, F) ? glu_workspace_bytes(T, H, F, dt, false) : 0;
}

size_t tempo_glu_bwd_workspace_bytes(int64_t T, int64_t H, int64_t F, tempo_dtype dt) {
  return glu_ok(T, H, F, TEMPO_GLU_SILU, dt) && glu_takes(T, H, F) ? glu_workspace_bytes(T, H, F, dt, true) : 0;
}

tempo_status tempo_glu_fwd(const void* x, const void* w, const void* bias, void* gu, void* h, void* workspace,
                           size_t workspace_bytes, int64_t T, int64_t H, int64_t F, tempo_glu_kind kind, tempo_dtype dt,
                           void* hip_stream) {
  if (!glu_ok(T, H, F, kind, dt)) return TEMPO_ERR_INVALID_ARG;
  if (T == 0 || F == 0) return TEMPO_OK;
  if (!h || (H > 0 && (!x || !w))) return TEMPO_ERR_INVALID_ARG;
  if (!glu_takes(T, H, F) || !aligned16(x) || !aligned16(w) || !aligned16(bias) || !aligned16(gu) || !aligned16(h) ||
      !aligned16(workspace))
    return TEMPO_ERR_UNSUPPORTED;
  GluCall c{};
  c.x = x, c.w = w, c.bias = bias, c.gu = gu, c.h = h;
  c.workspace = workspace, c.workspace_bytes = workspace ? workspace_bytes : 0;
  c.T = T, c.H = H, c.F = F, c.kind = kind;
  return launch_glu_fwd(c, dt, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_glu_bwd(const void* dh, const void* gu, const void* x, const void* w, void* dgu, void* h, void* dx,
                           void* dw, void* dbias, void* workspace, size_t workspace_bytes, int64_t T, int64_t H, int64_t F,
                           tempo_glu_kind kind, tempo_dtype dt, void* hip_stream) {
  if (!glu_ok(T, H, F, kind, dt)) return TEMPO_ERR_INVALID_ARG;
  // Sums of nothing are written too: dw and dbias of no rows, dx of no columns.
  if (T > 0 && F > 0 && (!dh || !gu || !dgu || (dw && H > 0 && !x) || (dx && H > 0 && !w))) return TEMPO_ERR_INVALID_ARG;
  if (!glu_takes(T, H, F) || !aligned16(dh) || !aligned16(gu) || !aligned16(x) || !aligned16(w) || !aligned16(dgu) ||
      !aligned16(h) || !aligned16(dx) || !aligned16(dw) || !aligned16(dbias) || !aligned16(workspace))
    return TEMPO_ERR_UNSUPPORTED;
  GluCall c{};
  c.x = x, c.w = w, c.gu = const_cast<void*>(gu), c.h = h, c.dh = dh, c.dgu = dgu, c.dx = dx, c.dw = dw, c.dbias = dbias;
  c.workspace = workspace, c.workspace_bytes = workspace ? workspace_bytes : 0;
  c.T = T, c.H = H, c.F = F, c.kind = kind;
  return launch_glu_bwd(c, dt, static_cast<hipStream_t>(hip_stream));
}

static bool norm_ok(const tempo_norm* n) {
  return !n || ((n->kind == TEMPO_NORM_RMS || n->kind == TEMPO_NORM_LAYER) && n->eps >= 0.0f);  // false for NaN
}
static bool residual_norm_ok(int64_t N, int64_t M, int64_t groups, tempo_dtype dt) {
  return N >= 0 && M >= 0 && M <= INT32_MAX && groups >= 1 && N % groups == 0 && dtype_ok(dt) && count_ok(N, M) && count_ok(groups, M);
}
static bool norm_aligned(const tempo_norm* n) {
  return !n || (aligned_to(n->weight, 4) && aligned_to(n->bias, 4) && aligned_to(n->stats, 8));
}

size_t tempo_residual_norm_bwd_workspace_bytes(int64_t N, int64_t M, int64_t groups, tempo_dtype dt) {
  if (!residual_norm_ok(N, M, groups, dt) || M == 0) return 0;
  ResidualCall c{};
  const float one = 1.0f;
  c.gate = &one;  // there is one
  c.N = N, c.M = M, c.groups = groups;
  return residual_norm_takes(c, dt) ? residual_norm_workspace_bytes(c, dt) : 0;
}

tempo_status tempo_residual_norm_fwd(const void* x, const void* f, const float* gate, int64_t groups, const tempo_norm* post,
                                     const tempo_norm* pre, void* y, void* h, float alpha, float beta, int64_t N, int64_t M,
                                     tempo_dtype dt, void* hip_stream) {
  if (!residual_norm_ok(N, M, groups, dt) || !norm_ok(post) || !norm_ok(pre)) return TEMPO_ERR_INVALID_ARG;
  if (N == 0 || M == 0) return TEMPO_OK;
  if (!x || !f || !y || (pre && !h)) return TEMPO_ERR_INVALID_ARG;
  ResidualCall c{};
  c.x = x, c.f = f, c.gate = gate, c.groups = gate ? groups : 1, c.post = post, c.pre = pre, c.to_y = y, c.h = h;
  c.alpha = alpha, c.beta = beta, c.N = N, c.M = M;
  if (!aligned16(x) || !aligned16(f) || !aligned16(y) || !aligned16(h) || !aligned_to(gate, 4) || !norm_aligned(post) ||
      !norm_aligned(pre) || !residual_norm_takes(c, dt))
    return TEMPO_ERR_UNSUPPORTED;
  return launch_residual_norm_fwd(c, dt, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_residual_norm_bwd(const void* dy, const void* dh, const void* f, const void* y, const float* gate, int64_t groups,
                                     const tempo_norm* post, const tempo_norm* pre, void* dx, void* df, float* dgate, float* dpost_weight,
                                     float* dpost_bias, float* dpre_weight, float* dpre_bias, float alpha, float beta, void* workspace,
                                     size_t workspace_bytes, int64_t N, int64_t M, tempo_dtype dt, void* hip_stream) {
  if (!residual_norm_ok(N, M, groups, dt) || !norm_ok(post) || !norm_ok(pre)) return TEMPO_ERR_INVALID_ARG;
  if ((dgate && !gate) || ((dpost_weight || dpost_bias) && !post) || ((dpre_weight || dpre_bias) && !pre)) return TEMPO_ERR_INVALID_ARG;
  if (M == 0) return TEMPO_OK;
  // Sums of no rows are written too.
  if (N > 0 && (!f || !dx || !df || (!dy && !pre) || (post && !post->stats) || (pre && (!dh || !y || !pre->stats)))) return TEMPO_ERR_INVALID_ARG;
  ResidualCall c{};
  c.dy = dy, c.dh = dh, c.f = f, c.y = y, c.gate = gate, c.groups = gate ? groups : 1, c.post = post, c.pre = pre, c.dx = dx, c.df = df;
  c.dgate = dgate, c.dpost_weight = dpost_weight, c.dpost_bias = dpost_bias, c.dpre_weight = dpre_weight, c.dpre_bias = dpre_bias;
  c.alpha = alpha, c.beta = beta, c.workspace = workspace, c.workspace_bytes = workspace ? workspace_bytes : 0, c.N = N, c.M = M;
  for (const void* t : {dy, dh, f, y, static_cast<const void*>(dx), static_cast<const void*>(df), static_cast<const void*>(workspace)})
    if (!aligned16(t)) return TEMPO_ERR_UNSUPPORTED;
  for (const float* t : {gate, static_cast<const float*>(dgate), static_cast<const float*>(dpost_weight), static_cast<const float*>(dpost_bias),
                         static_cast<const float*>(dpre_weight), static_cast<const float*>(dpre_bias)})
    if (!aligned_to(t, 4)) return TEMPO_ERR_UNSUPPORTED;
  if (!norm_aligned(post) || !norm_aligned(pre) || !residual_norm_takes(c, dt)) return TEMPO_ERR_UNSUPPORTED;
  return launch_residual_norm_bwd(c, dt, static_cast<hipStream_t>(hip_stream));
}

static bool window_attn_ok(const WindowCall& c) {
  return c.B >= 0 && c.Sq >= 0 && c.Sk >= 0 && c.heads >= 0 && c.kv_heads >= 0 && c.D >= 1 && c.window >= 1 && c.sinks >= 0 &&
         (c.heads == 0 || (c.kv_heads >= 1 && c.heads % c.kv_heads == 0)) && c.Sq <= INT32_MAX && c.Sk <= INT32_MAX &&
         count_ok(c.B, c.Sq, c.heads, c.D) && count_ok(c.B, c.Sk, c.kv_heads, c.D) && count_ok(c.B, c.heads) &&
         c.B * c.heads <= INT32_MAX;
}
// A [batch, tokens, heads, elements] whose elements lie within what a tensor may have, those of an output apart.
static bool attn_heads_ok(const tempo_attn_heads* h, int64_t B, int64_t S, int64_t heads, int64_t D, bool out) {
  if (!h) return false;
  const int64_t sizes[] = {B, S, heads}, strides[] = {h->batch, h->token, h->head};
  int64_t last = D;
  for (int i = 0; i < 3; ++i) {
    if (strides[i] < 0 || !count_ok(sizes[i], strides[i]) || (out && sizes[i] > 1 && strides[i] == 0)) return false;
    last += sizes[i] * strides[i];
  }
  return last <= kMaxElements;
}
static WindowCall window_sizes(int64_t B, int64_t Sq, int64_t Sk, int64_t heads, int64_t kv_heads, int64_t D, int64_t window,
                               int64_t sinks) {
  constexpr int64_t most = int64_t{1} << 33;  // beyond any position
  WindowCall c{};
  c.B = B, c.Sq = Sq, c.Sk = Sk, c.heads = heads, c.kv_heads = kv_heads, c.D = D;
  if (heads == 0 && kv_heads > 0 && Sq >= 0) c.heads = kv_heads, c.Sq = 0;  // key heads that none reads: no queries, whose gradients are zeros
  c.window = window < most ? window : most;
  c.sinks = sinks < most ? sinks : most;
  return c;
}
static size_t window_attn_bytes(const WindowCall& c, tempo_dtype dt, bool back) {
  return window_attn_ok(c) && dtype_ok(dt) && c.B > 0 && c.heads > 0 && window_attn_takes(c) ? window_attn_workspace_bytes(c, dt, back) : 0;
}

size_t tempo_window_attn_fwd_workspace_bytes(int64_t B, int64_t Sq, int64_t Sk, int64_t heads, int64_t kv_heads, int64_t D,
                                             int64_t window, int64_t sinks, tempo_dtype dt) {
  const WindowCall c = window_sizes(B, Sq, Sk, heads, kv_heads, D, window, sinks);
  return window_attn_bytes(c, dt, false);
}

size_t tempo_window_attn_bwd_workspace_bytes(int64_t B, int64_t Sq, int64_t Sk, int64_t heads, int64_t kv_heads, int64_t D,
                                             int64_t window, int64_t sinks, tempo_dtype dt) {
  const WindowCall c = window_sizes(B, Sq, Sk, heads, kv_heads, D, window, sinks);
  return window_attn_bytes(c, dt, true);
}

// Normal, as scale log2(e) is too (false for NaN).
static bool scale_ok(float scale) { return scale >= 1.17549435e-38f && scale <= 1.70141183e+38f; }

tempo_status tempo_window_attn_fwd(const tempo_attn_heads* q, const tempo_attn_heads* k, const tempo_attn_heads* v,
                                   const tempo_attn_heads* out, float* lse, const int32_t* key_len, const int32_t* query_start,
                                   void* workspace, size_t workspace_bytes, int64_t B, int64_t Sq, int64_t Sk, int64_t heads,
                                   int64_t kv_heads, int64_t D, int64_t window, int64_t sinks, float scale, tempo_dtype dt,
                                   void* hip_stream) {
  WindowCall c = window_sizes(B, Sq, Sk, heads, kv_heads, D, window, sinks);
  if (!window_attn_ok(c) || !dtype_ok(dt) || !scale_ok(scale) || !attn_heads_ok(q, B, Sq, heads, D, false) ||
      !attn_heads_ok(k, B, Sk, kv_heads, D, false) || !attn_heads_ok(v, B, Sk, kv_heads, D, false) ||
      !attn_heads_ok(out, B, Sq, heads, D, true))
    return TEMPO_ERR_INVALID_ARG;
  if (B == 0 || Sq == 0 || heads == 0) return TEMPO_OK;
  if (!q->p || !out->p || (Sk > 0 && (!k->p || !v->p))) return TEMPO_ERR_INVALID_ARG;
  const uintptr_t element = dt == TEMPO_F32 ? 4 : 2;
  for (const tempo_attn_heads* h : {q, k, v, out})
    if (!aligned_to(h->p, element)) return TEMPO_ERR_UNSUPPORTED;
  if (!window_attn_takes(c) || !aligned_to(lse, 4) || !aligned_to(key_len, 4) || !aligned_to(query_start, 4) || !aligned16(workspace))
    return TEMPO_ERR_UNSUPPORTED;
  c.q = q, c.k = k, c.v = v, c.out = out, c.lse = lse, c.key_len = key_len, c.query_start = query_start;
  c.workspace = workspace, c.workspace_bytes = workspace ? workspace_bytes : 0;
  c.scale = scale;
  return launch_window_attn_fwd(c, dt, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_window_attn_bwd(const tempo_attn_heads* dout, const tempo_attn_heads* q, const tempo_attn_heads* k,
                                   const tempo_attn_heads* v, const tempo_attn_heads* out, const float* lse, const tempo_attn_heads* dq,
                                   const tempo_attn_heads* dk, const tempo_attn_heads* dv, const int32_t* key_len,
                                   const int32_t* query_start, void* workspace, size_t workspace_bytes, int64_t B, int64_t Sq,
                                   int64_t Sk, int64_t heads, int64_t kv_heads, int64_t D, int64_t window, int64_t sinks, float scale,
                                   tempo_dtype dt, void* hip_stream) {
  WindowCall c = window_sizes(B, Sq, Sk, heads, kv_heads, D, window, sinks);
  if (!window_attn_ok(c) || !dtype_ok(dt) || !scale_ok(scale)) return TEMPO_ERR_INVALID_ARG;
  for (const tempo_attn_heads* h : {q, out, dout})
    if (!attn_heads_ok(h, B, Sq, heads, D, false)) return TEMPO_ERR_INVALID_ARG;
  for (const tempo_attn_heads* h : {k, v})
    if (!attn_heads_ok(h, B, Sk, kv_heads, D, false)) return TEMPO_ERR_INVALID_ARG;
  if (!attn_heads_ok(dq, B, Sq, heads, D, true) || !attn_heads_ok(dk, B, Sk, kv_heads, D, true) ||
      !attn_heads_ok(dv, B, Sk, kv_heads, D, true))
    return TEMPO_ERR_INVALID_ARG;
  if (B == 0 || c.heads == 0 || (c.Sq == 0 && Sk == 0)) return TEMPO_OK;
  // Gradients of no queries are written too: zeros.
  if (c.Sq > 0 && (!q->p || !out->p || !dout->p || !dq->p || !lse)) return TEMPO_ERR_INVALID_ARG;
  if (Sk > 0 && (!k->p || !v->p || !dk->p || !dv->p)) return TEMPO_ERR_INVALID_ARG;
  const uintptr_t element = dt == TEMPO_F32 ? 4 : 2;
  for (const tempo_attn_heads* h : {q, k, v, out, dout, dq, dk, dv})
    if (!aligned_to(h->p, element)) return TEMPO_ERR_UNSUPPORTED;
  if (!window_attn_takes(c) || !aligned_to(lse, 4) || !aligned_to(key_len, 4) || !aligned_to(query_start, 4) || !aligned16(workspace))
    return TEMPO_ERR_UNSUPPORTED;
  c.q = q, c.k = k, c.v = v, c.out = out, c.dout = dout, c.dq = dq, c.dk = dk, c.dv = dv;
  c.lse = const_cast<float*>(lse), c.key_len = key_len, c.query_start = query_start;
  c.workspace = workspace, c.workspace_bytes = workspace ? workspace_bytes : 0;
  c.scale = scale;
  return launch_window_attn_bwd(c, dt, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_mask_bits_to_bytes(const uint32_t* bits, uint8_t* bytes, int64_t n,
                                      void* hip_stream) {
  if (n < 0 || !count_ok(n)) return TEMPO_ERR_INVALID_ARG;
  if (n == 0) return TEMPO_OK;
  if (!bits || !bytes) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(bits) || !aligned16(bytes)) return TEMPO_ERR_UNSUPPORTED;
  return launch_mask_bits_to_bytes(bits, bytes, n, static_cast<hipStream_t>(hip_stream));
}

tempo_status tempo_mask_bytes_to_bits(const uint8_t* bytes, uint32_t* bits, int64_t n,
                                      void* hip_stream) {
  if (n < 0 || !count_ok(n)) return TEMPO_ERR_INVALID_ARG;
  if (n == 0) return TEMPO_OK;
  if (!bits || !bytes) return TEMPO_ERR_INVALID_ARG;
  if (!aligned16(bits) || !aligned16(bytes)) return TEMPO_ERR_UNSUPPORTED;
  return launch_mask_bytes_to_bits(bytes, bits, n, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
