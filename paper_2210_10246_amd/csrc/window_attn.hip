// Window attention, forward.
#include "window_attn.h"

namespace tempo {
namespace {

// A lane's running maximum (of base 2) and its part of the sum of exponentials, of the row that the lane has.
struct Running {
  float top = kMinusInf, sum = 0.0f;
  // Scores of BLOCKS x 32 keys to exponentials; c: scale log2(e).  What they are relative to follows the maximum only where they would pass
  // 2^8: nothing is lost below that.
  template <int BLOCKS, int COLUMNS>
  __device__ __forceinline__ void exponentials(f32x16 (&p)[BLOCKS], float c, f32x16 (&acc)[COLUMNS]) {
    float most = p[0][0];
#pragma unroll
    for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, p[kb][i]);
    most = c * across_rows<32>(most, [](float x, float y) { return fmaxf(x, y); });
    if (__any(most > top + 8.0f)) {
      const float next = fmaxf(top, most);
      rescale(next, __builtin_amdgcn_exp2f(top - finite(next)), acc);
    }
    const float from = finite(top);
#pragma unroll
    for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[kb][i] = __builtin_amdgcn_exp2f(fmaf(p[kb][i], c, -from));
        sum += p[kb][i];
      }
  }
  __device__ static __forceinline__ float finite(float x) { return x == kMinusInf ? 0.0f : x; }
  template <int COLUMNS>
  __device__ __forceinline__ void rescale(float next, float by, f32x16 (&acc)[COLUMNS]) {
    top = next;
    sum *= by;
#pragma unroll
    for (int d = 0; d < COLUMNS; ++d) acc[d] *= by;
  }
};

// What a row has in the end, to the output or as part `part` of it, of a.splits.
template <typename T, int COLUMNS>
__device__ __forceinline__ void finish(const Attn& a, const Running& run, const f32x16 (&acc)[COLUMNS], int b, int kv, const WaveRows& w, int part,
                                       int64_t all_rows) {
  const float sum = across_rows<32>(run.sum, [](float x, float y) { return x + y; });
  const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
  const float lse = sum == 0.0f ? kMinusInf : run.top + __builtin_amdgcn_logf(sum);
  const bool first_half = threadIdx.x % kWave < 32;
  if (a.splits > 1) {
    const int64_t at_row = part * all_rows + (static_cast<int64_t>(b) * a.kv_heads + kv) * a.rows + w.row;
    if (first_half) a.partial_lse[at_row] = lse;
#pragma unroll
    for (int d = 0; d < COLUMNS; ++d) store_sums(a.partial + at_row * a.pitch, a.pitch, d, acc[d], by);
  } else {
    const int head = kv * a.group + w.g;
    if (a.lse && first_half) a.lse[(static_cast<int64_t>(b) * a.heads + head) * a.Sq + w.i] = lse * kLn2;
    T* const to = const_cast<T*>(at<T>(a.out, b, w.i, head));
#pragma unroll
    for (int d = 0; d < COLUMNS; ++d) store_sums(to, a.D, d, acc[d], by);
  }
}

// Waves on a SIMD: two where their registers allow it, one at its matrix instructions while the other is at its exponentials.  The forward of
// rows of up to 128 bfloat16 with tiles of 32 keys allows three: 8192 tokens of 32 / 8 heads of 128, window 1024 164 us, 178 with tiles of 64
// and two, 172 with tiles of 32 and two; 16384 with a window of 4096 994, 1000 and 1050 us (968 TFLOP/s).  Two groups of waves held
// apart by barriers, one at the exponentials while the other is at its products, take 204 and 1148 us.
template <typename T, int DP, bool DIRECT>
constexpr int kForward = DIRECT && sizeof(T) == 2 && DP <= 128 ? 3 : kAtOnce<T, DP, DIRECT>;

template <typename T, int DP, int BK, bool DIRECT>
__global__ __launch_bounds__(kThreads, (kForward<T, DP, DIRECT>)) void forward_kernel(Attn a) {
  using R = Rows<T, DP>;
  using Stream = KeyStream<T, DP, BK, DIRECT>;
  constexpr int kBlocks = BK / 32, kColumns = DP / 32;
  __shared__ __attribute__((aligned(16))) char lds[2][2][Stream::kBytes];
  const int job = in_order(blockIdx.x, gridDim.x), split = job % a.splits, tile = job / a.splits % a.tiles;
  const int bk = job / a.splits / a.tiles, b = bk / a.kv_heads, kv = bk - b * a.kv_heads;
  const Sight s(a, b);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int first_row = tile * kRows, last_row = min(first_row + kRows, a.rows) - 1;
  const KeyTiles keys(s, a.by_group.divide(first_row), a.by_group.divide(last_row), BK);
  const int each = (keys.count + a.splits - 1) / a.splits, n0 = split * each, n1 = min(n0 + each, keys.count);
  Stream stream(a, keys, b, kv, lds, n0, n1);
  const WaveRows w(a, s, first_row + wave * 32);
  u32x4 q[R::kSteps];
  const int half = threadIdx.x % kWave / 32;
  load_half_row<T, DP>(at<T>(a.q, b, w.i, kv * a.group + w.g), half, a.D, q);
  fit_half_row<T, DP>(half, a.D, q);
  f32x16 acc[kColumns];
#pragma unroll
  for (int d = 0; d < kColumns; ++d) acc[d] = zeros();
  Running run;
  stream.each([&](int j0, const char* k_tile, const char* v_tile) {
    if (!w.any || w.none(s, j0, BK)) return;
    f32x16 p[kBlocks];
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
      p[kb] = zeros();
#pragma unroll
      for (int t = 0; t < R::kSteps; ++t) p[kb] = multiply<T>(R::rows(k_tile, kb * 32, t), q[t], p[kb]);
    }
    if (!w.all(s, j0, BK)) w.hide(s, j0, p, kMinusInf);
    run.exponentials(p, a.c, acc);
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
      const Weights<T> weights(p[kb]);
#pragma unroll
      for (int d = 0; d < kColumns; ++d) acc[d] = multiply_columns<T, DP>(v_tile, kb * 32, d, weights, acc[d]);
    }
  });
  if (w.r0 + static_cast<int>(threadIdx.x) % 32 >= a.rows) return;
  finish<T>(a, run, acc, b, kv, w, split, static_cast<int64_t>(gridDim.x / (a.splits * a.tiles)) * a.rows);
}

// Up to 32 rows for a key head, as for a token each of the sequences of a cache: bound by the bytes of k and v.  Each wave takes its own blocks of 32
// keys, without barriers, by way of registers, which the next block is on its way to while one is worked on, and the wave's own LDS.  Lanes side
// by side load pieces side by side, past the caches: 48 tokens of 32 / 8 heads of 128, window 4096 134 us, 160 through them, 181 with k as a matrix
// instruction takes it, two pieces of each row at a time.  The waves' sums are joined in LDS, those of the workgroups that share a head by join_kernel.
template <typename T, int DP>
constexpr int kFewWaves = sizeof(T) * DP <= 256 ? 8 : 4;
// WHOLE: rows of DP elements.
template <typename T, int DP, bool WHOLE>
__global__ __launch_bounds__((kFewWaves<T, DP> * kWave), (kFewWaves<T, DP> / 4)) void few_kernel(Attn a) {
  const int D = WHOLE ? DP : a.D;
  using R = Rows<T, DP>;
  constexpr int W = kFewWaves<T, DP>, kColumns = DP / 32, kBytes = R::bytes(32);
  constexpr int kRow = DP + 4;  // floats of a row of a wave's sums, 16 bytes further in the banks than the row before
  __shared__ __attribute__((aligned(16))) char lds[W * (2 * kBytes > 32 * kRow * 4 ? 2 * kBytes : 32 * kRow * 4)];
  __shared__ float2 tops[W][32];
  const int job = in_order(blockIdx.x, gridDim.x), split = job % a.splits, bk = job / a.splits, b = bk / a.kv_heads, kv = bk - b * a.kv_heads;
  const Sight s(a, b);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, half = lane / 32;
  const KeyTiles keys(s, 0, a.by_group.divide(a.rows - 1), 32);
  const WaveRows w(a, s, 0);
  char *const own_k = lds + 2 * wave * kBytes, *const own_v = own_k + kBytes;
  const int step = a.splits * W;
  int n = split * W + wave;
  u32x4 k[R::kSteps], v[R::kSteps], q[R::kSteps];
  auto fetch = [&](int j0) {
#pragma unroll
    for (int p = 0; p < R::kSteps; ++p) {
      const int row = (p * kWave + lane) / R::P, piece = (p * kWave + lane) % R::P, key = keys.seen(j0 + row);
      k[p] = load_piece<T, true, WHOLE>(at<T>(a.k, b, key, kv), piece, D);
      v[p] = load_piece<T, true, WHOLE>(at<T>(a.v, b, key, kv), piece, D);
    }
  };
  if (n < keys.count) fetch(keys.key(n, 32));
  load_half_row<T, DP>(at<T>(a.q, b, w.i, kv * a.group + w.g), half, D, q);
  fit_half_row<T, DP>(half, D, q);
  f32x16 acc[kColumns];
#pragma unroll
  for (int d = 0; d < kColumns; ++d) acc[d] = zeros();
  Running run;
  for (; n < keys.count; n += step) {
    const int j0 = keys.key(n, 32);
#pragma unroll
    for (int t = 0; t < R::kSteps; ++t) {
      const int row = (t * kWave + lane) / R::P, piece = (t * kWave + lane) % R::P, to = R::place(row) + ((piece ^ R::swizzle(row)) << 4);
      *reinterpret_cast<u32x4*>(own_k + to) = fitted<T>(k[t], piece, D, DP);
      *reinterpret_cast<u32x4*>(own_v + to) = fitted<T>(v[t], piece, D, DP);
    }
    if (n + step < keys.count) fetch(keys.key(n + step, 32));
    wave_lds_fence();
    f32x16 p[1] = {zeros()};
#pragma unroll
    for (int t = 0; t < R::kSteps; ++t) p[0] = multiply<T>(R::rows(own_k, 0, t), q[t], p[0]);
    if (!w.all(s, j0, 32)) w.hide(s, j0, p, kMinusInf);
    run.exponentials(p, a.c, acc);
    const Weights<T> weights(p[0]);
#pragma unroll
    for (int d = 0; d < kColumns; ++d) acc[d] = multiply_columns<T, DP>(own_v, 0, d, weights, acc[d]);
    wave_lds_fence();
  }
  lds_barrier();
  float* const all_sums = reinterpret_cast<float*>(lds);
  if (lane % 32 < a.rows) {
    const float sum = across_rows<32>(run.sum, [](float x, float y) { return x + y; });
    if (half == 0) tops[wave][lane] = make_float2(run.top, sum);
    float* const to = all_sums + (wave * 32 + lane) * kRow - half * 32 * kRow + 4 * half;
#pragma unroll
    for (int d = 0; d < kColumns; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4*>(to + d * 32 + 8 * e) = f32x4{acc[d][4 * e], acc[d][4 * e + 1], acc[d][4 * e + 2], acc[d][4 * e + 3]};
  }
  lds_barrier();
  // four elements of a row a lane
  const int64_t all_rows = static_cast<int64_t>(gridDim.x / a.splits) * a.rows;
  for (int at_sum = threadIdx.x; at_sum < a.rows * (DP / 4); at_sum += W * kWave) {
    const int row = at_sum / (DP / 4), d = at_sum % (DP / 4) * 4;
    float top = kMinusInf, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) top = fmaxf(top, tops[i][row].x);
    const float from = Running::finite(top);
    f32x4 out = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float by = __builtin_amdgcn_exp2f(tops[i][row].x - from);
      sum = fmaf(tops[i][row].y, by, sum);
      out += by * *reinterpret_cast<const f32x4*>(all_sums + (i * 32 + row) * kRow + d);
    }
    out *= sum == 0.0f ? 0.0f : 1.0f / sum;
    const float lse = sum == 0.0f ? kMinusInf : top + __builtin_amdgcn_logf(sum);
    if (a.splits > 1) {
      const int64_t at_row = split * all_rows + static_cast<int64_t>(bk) * a.rows + row;
      if (d == 0) a.partial_lse[at_row] = lse;
      store_four(a.partial + at_row * a.pitch, a.pitch, d, out);
    } else {
      const int i = a.by_group.divide(row), head = kv * a.group + row - i * a.group;
      if (a.lse && d == 0) a.lse[(static_cast<int64_t>(b) * a.heads + head) * a.Sq + i] = lse * kLn2;
      store_four(const_cast<T*>(at<T>(a.out, b, i, head)), D, d, out);
    }
  }
}

// The parts of a row, each weighted by its sum of exponentials: 16 lanes a row.
template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(Attn a, int64_t all) {
  const int64_t at_row = static_cast<int64_t>(blockIdx.x) * (kThreads / 16) + threadIdx.x / 16;
  if (at_row >= all) return;
  float top = kMinusInf, sum = 0.0f;
  for (int p = 0; p < a.splits; ++p) top = fmaxf(top, a.partial_lse[p * all + at_row]);
  const float from = Running::finite(top);
  for (int p = 0; p < a.splits; ++p) sum += __builtin_amdgcn_exp2f(a.partial_lse[p * all + at_row] - from);
  const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
  const int bk = static_cast<int>(at_row / a.rows), row = static_cast<int>(at_row - static_cast<int64_t>(bk) * a.rows);
  const int b = bk / a.kv_heads, i = a.by_group.divide(row), head = (bk - b * a.kv_heads) * a.group + row - i * a.group;
  if (a.lse && threadIdx.x % 16 == 0)
    a.lse[(static_cast<int64_t>(b) * a.heads + head) * a.Sq + i] = sum == 0.0f ? kMinusInf : (from + __builtin_amdgcn_logf(sum)) * kLn2;
  T* const to = const_cast<T*>(at<T>(a.out, b, i, head));
  for (int d = threadIdx.x % 16 * 4; d < a.D; d += 64) {
    f32x4 out = {0, 0, 0, 0};
#pragma unroll 4
    for (int p = 0; p < a.splits; ++p)
      out += __builtin_amdgcn_exp2f(a.partial_lse[p * all + at_row] - from) * *reinterpret_cast<const f32x4*>(a.partial + (p * all + at_row) * a.pitch + d);
    store_four(to, a.D, d, out * by);
  }
}

}  // namespace

// The call as if it gave positions: there may be more to do then.
static WindowCall with_positions(WindowCall c) {
  static const int32_t any = 0;
  c.query_start = &any;
  return c;
}

// Launches of less than 2^32 lanes, and numbers of jobs that an int holds.
bool window_attn_takes(const WindowCall& c) {
  constexpr int64_t most = int64_t{1} << 22;
  const int64_t bk = c.B * c.kv_heads, rows = c.Sq * (c.heads / c.kv_heads);
  if (c.D > 256 || rows > INT32_MAX - kRows || up(rows, kRows) * bk > most || up(c.Sk, kRows) * bk > most) return false;
  const KeyPlan p = key_plan(with_positions(c));
  return p.blocks <= 2 * most && bk * p.jobs.sink_tiles < most / 8;
}

size_t window_attn_workspace_bytes(const WindowCall& c, tempo_dtype dt, bool back) {
  const int64_t rows = c.B * c.heads * c.Sq;
  if (!back) {
    const int splits = forward_splits(c, dt);
    return splits > 1 ? static_cast<size_t>(splits) * rows * (pitch_of(c) + 1) * sizeof(float) : 0;
  }
  const KeyPlan p = key_plan(with_positions(c));
  return static_cast<size_t>(up(2 * rows, 4) * 4 + p.partial_floats + p.further_floats) * sizeof(float);
}

tempo_status launch_window_attn_fwd(const WindowCall& c, tempo_dtype dt, hipStream_t st) {
  if (c.workspace_bytes < window_attn_workspace_bytes(c, dt, false)) return TEMPO_ERR_WORKSPACE;
  Attn a = attn_of(c);
  a.splits = forward_splits(c, dt);
  const int64_t all = c.B * c.heads * c.Sq;
  if (a.splits > 1) {
    a.partial = static_cast<float*>(c.workspace);
    a.partial_lse = a.partial + a.splits * all * a.pitch;
  }
  const int64_t blocks = c.B * c.kv_heads * a.tiles * a.splits;
  return with_type(dt, [&](auto type) {
    using T = decltype(type);
    const tempo_status s = with_width(c.D, [&](auto width) {
      constexpr int DP = decltype(width)::value, BK = sizeof(T) == 4 && DP == 64 ? 64 : 32;
      if constexpr (sizeof(T) * DP <= 512) {
        if (few(c, dt)) {
          return either(a.D == DP, [&](auto whole) {
            hipLaunchKernelGGL((few_kernel<T, DP, decltype(whole)::value>), dim3(static_cast<uint32_t>(c.B * c.kv_heads * a.splits)),
                               dim3(kFewWaves<T, DP> * kWave), 0, st, a);
            return launch_status();
          });
        }
      }
      return either(direct(c, dt, {c.k, c.v}), [&](auto straight) {
        return launch(forward_kernel<T, DP, BK, decltype(straight)::value>, blocks, st, a);
      });
    });
    if (s != TEMPO_OK || a.splits == 1) return s;
    return launch(join_kernel<T>, up(all, kThreads / 16), st, a, all);
  });
}

}  // namespace tempo
