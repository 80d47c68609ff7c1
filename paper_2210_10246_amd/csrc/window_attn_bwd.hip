// Window attention, backward.
#include "window_attn.h"

namespace tempo {
namespace {

// ---- backward by rows: delta and dq ---------------------------------------------------------------------------------------
// Three of the seven products.  Rows of 128 bfloat16 are bound by the matrix instructions (32768 tokens of 32 / 8 heads, window 4096 2.86 ms, 1090
// TFLOP/s), of 64 by the vector instructions beside them (8 x 2048 tokens of 16 heads, window 512 95 us, 475); float32 by the matrix
// instructions of one wave a SIMD and what it waits for (3 x 1021 tokens of 9 / 3 heads of 83, window 200 82 us).
template <typename T, int DP, int BK, bool DIRECT>
__global__ __launch_bounds__(kThreads, (kAtOnce<T, DP, DIRECT>)) void rows_kernel(Attn a) {
  using R = Rows<T, DP>;
  using Stream = KeyStream<T, DP, BK, DIRECT>;
  constexpr int kBlocks = BK / 32, kColumns = DP / 32;
  __shared__ __attribute__((aligned(16))) char lds[2][2][Stream::kBytes];
  const int job = in_order(blockIdx.x, gridDim.x), tile = job % a.tiles;
  const int bk = job / a.tiles, b = bk / a.kv_heads, kv = bk - b * a.kv_heads;
  const Sight s(a, b);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int first_row = tile * kRows, last_row = min(first_row + kRows, a.rows) - 1;
  const KeyTiles keys(s, a.by_group.divide(first_row), a.by_group.divide(last_row), BK);
  Stream stream(a, keys, b, kv, lds, 0, keys.count);
  const WaveRows w(a, s, first_row + wave * 32);
  const int head = kv * a.group + w.g, half = threadIdx.x % kWave / 32;
  const int64_t stat = (static_cast<int64_t>(b) * a.heads + head) * a.Sq + w.i;
  u32x4 q[R::kSteps], dout[R::kSteps];
  float delta = 0.0f;
  {
    u32x4 out[R::kSteps];
    load_half_row<T, DP>(at<T>(a.dout, b, w.i, head), half, a.D, dout);
    load_half_row<T, DP>(at<T>(a.out, b, w.i, head), half, a.D, out);
    load_half_row<T, DP>(at<T>(a.q, b, w.i, head), half, a.D, q);
    fit_half_row<T, DP>(half, a.D, dout);
    fit_half_row<T, DP>(half, a.D, out);
    fit_half_row<T, DP>(half, a.D, q);
#pragma unroll
    for (int p = 0; p < R::kSteps; ++p) {
      float x[R::V], y[R::V];
      Store<T>::unpack(dout[p], x);
      Store<T>::unpack(out[p], y);
#pragma unroll
      for (int e = 0; e < R::V; ++e) delta = fmaf(x[e], y[e], delta);
    }
    delta = across_rows<32>(delta, [](float x, float y) { return x + y; });
  }
  const bool exists = w.r0 + static_cast<int>(threadIdx.x) % 32 < a.rows;
  const float lse = a.lse[stat] * kLog2e;
  if (exists && half == 0) {
    a.stats[stat] = lse;
    a.stats[a.stat_rows + stat] = delta;
  }
  f32x16 acc[kColumns];
#pragma unroll
  for (int d = 0; d < kColumns; ++d) acc[d] = zeros();
  stream.each([&](int j0, const char* k_tile, const char* v_tile) {
    if (!w.any || w.none(s, j0, BK)) return;
    const bool all = w.all(s, j0, BK);
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
      f32x16 p[1] = {zeros()}, dp = zeros();
#pragma unroll
      for (int t = 0; t < R::kSteps; ++t) {
        p[0] = multiply<T>(R::rows(k_tile, kb * 32, t), q[t], p[0]);
        dp = multiply<T>(R::rows(v_tile, kb * 32, t), dout[t], dp);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) p[0][i] = __builtin_amdgcn_exp2f(fmaf(p[0][i], a.c, -lse)) * (dp[i] - delta);
      if (!all) w.hide(s, j0 + kb * 32, p, 0.0f);
      const Weights<T> weights(p[0]);
#pragma unroll
      for (int d = 0; d < kColumns; ++d) acc[d] = multiply_columns<T, DP>(k_tile, kb * 32, d, weights, acc[d]);
    }
  });
  if (!exists) return;
  T* const to = const_cast<T*>(at<T>(a.dq, b, w.i, head));
#pragma unroll
  for (int d = 0; d < kColumns; ++d) store_sums(to, a.D, d, acc[d], a.scale);
}

// ---- backward by keys: dk and dv ------------------------------------------------------------------------------------------
// The queries that see a tile of keys in their window, taken in blocks of BQ of one head after the other.  Those further on see only the first
// keys: jobs of their own take them for 32 of these keys at a time, the blocks dealt out to the four waves.  Where there is more than one sum for
// a key (parts of a tile's blocks, what is further on), the sums are joined in their order.  Four of the seven products, bound as by rows: the same
// calls take 4.13 ms (1000 TFLOP/s), 105 us (574) and 154 us.
enum Wanted { kBoth, kOnlyV, kOnlyK };
// bfloat16: v of the workgroup's keys in LDS, not in registers.  There a wave of rows of 128 would need more than the 256 that let two run on a
// SIMD (32768 tokens, window 4096 7.0 ms, and 4.2 in LDS), one of 64 more than the 168 that let three.
template <typename T>
constexpr bool kValuesInLds = sizeof(T) == 2;
template <typename T, int DP, bool DIRECT>
constexpr int kKeysAtOnce = DIRECT && sizeof(T) == 2 && DP == 64 ? 3 : kAtOnce<T, DP, DIRECT>;
template <typename T, int DP>
constexpr int kQueries = sizeof(T) == 2 && DP == 64 ? 64 : 32;  // of a block

template <typename T, int DP, Wanted WANTED, bool DIRECT>
__global__ __launch_bounds__(kThreads, (kKeysAtOnce<T, DP, DIRECT>)) void keys_kernel(Attn a, KeyJobs jobs) {
  using R = Rows<T, DP>;
  constexpr int BQ = kQueries<T, DP>, kBytes = R::bytes(BQ), kColumns = DP / 32;
  __shared__ __attribute__((aligned(16))) char lds[2][2][kBytes];
  __shared__ __attribute__((aligned(16))) float stats[2][2][BQ];  // lse of base 2, delta
  constexpr bool kK = WANTED != kOnlyV, kV = WANTED != kOnlyK, kInLds = kK && kValuesInLds<T>;
  __shared__ __attribute__((aligned(16))) char values[kInLds ? R::bytes(kRows) : 16];
  int64_t job = blockIdx.x;
  const bool further = job < jobs.further_jobs;
  if (!further) job = in_order(static_cast<int>(job - jobs.further_jobs), static_cast<int>(gridDim.x - jobs.further_jobs));
  const int parts = further ? jobs.further_parts : jobs.parts, tiles = further ? jobs.strips : jobs.tiles;
  const int part = static_cast<int>(job % parts), tile = static_cast<int>(job / parts % tiles);
  const int bk = static_cast<int>(job / parts / tiles), b = bk / a.kv_heads, kv = bk - b * a.kv_heads;
  const Sight s(a, b);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, half = lane / 32;
  const int key0 = tile * (further ? 32 : kRows), wave_key = key0 + (further ? 0 : wave * 32), key = wave_key + lane % 32;
  const int wave_last = wave_key + 31;
  // Queries [from, to) see key j in their window; those of [to, Sq) see it if it is one of the first.
  auto from = [&](int j) {
    const int64_t i = j - s.start;
    return j >= s.keys || i >= a.Sq ? a.Sq : i > 0 ? static_cast<int>(i) : 0;
  };
  auto to = [&](int j) {
    const int64_t i = j - s.before;
    return j >= s.keys || i <= 0 ? 0 : i < a.Sq ? static_cast<int>(i) : a.Sq;
  };
  auto beyond = [&](int j) { return j < s.sinks ? max(from(j), to(j)) : a.Sq; };
  // The job's queries, those that see some key of the wave, those that see all, and the lane's.
  int first, end, any_from, any_to, all_from, all_to, key_from, key_to;
  if (further) {
    first = any_from = beyond(key0), all_from = beyond(wave_last), key_from = beyond(key);
    end = any_to = all_to = key_to = a.Sq;
  } else {
    const int tile_last = min(key0 + kRows, s.keys) - 1;
    first = from(key0), end = key0 < s.keys ? to(tile_last) : 0;
    any_from = from(wave_key), any_to = wave_key < s.keys ? to(min(wave_last, s.keys - 1)) : 0;
    all_from = from(wave_last), all_to = wave_last < s.keys ? to(wave_key) : 0;
    key_from = from(key), key_to = to(key);
  }
  const uint32_t key_span = static_cast<uint32_t>(max(key_to - key_from, 0));
  const int blocks = first < end ? (end - first + BQ - 1) / BQ : 0;  // of a head
  const int each = static_cast<int>((static_cast<int64_t>(blocks) * a.group + parts - 1) / parts);
  const int u0 = min(part * each, blocks * a.group), u1 = min(u0 + each, blocks * a.group);
  u32x4 k[R::kSteps], v[R::kSteps];
  {
    const int there = min(key, a.Sk - 1);
    load_half_row<T, DP>(at<T>(a.k, b, there, kv), half, a.D, k);
    if constexpr (kK) load_half_row<T, DP>(at<T>(a.v, b, there, kv), half, a.D, v);
    fit_half_row<T, DP>(half, a.D, k);
    if constexpr (kK) fit_half_row<T, DP>(half, a.D, v);
    if constexpr (kInLds) {  // a wave's own rows
#pragma unroll
      for (int p = 0; p < R::kSteps; ++p) {
        const int row = wave * 32 + lane % 32, piece = 2 * p + half;
        *reinterpret_cast<u32x4*>(values + R::place(row) + ((piece ^ R::swizzle(row)) << 4)) = v[p];
      }
    }
  }
  auto value = [&](int step) {
    if constexpr (kInLds) return R::rows(values, wave * 32, step);
    else return v[step];
  };
  f32x16 dk[kK ? kColumns : 1], dv[kV ? kColumns : 1];
#pragma unroll
  for (int d = 0; d < (kK ? kColumns : 1); ++d) dk[d] = zeros();
#pragma unroll
  for (int d = 0; d < (kV ? kColumns : 1); ++d) dv[d] = zeros();
  std::conditional_t<DIRECT, Direct<T, DP, BQ>, Staged<T, DP, BQ>> qs(a.q), os(a.dout);
  float stat = 0.0f;  // of lane BQ n + i: lse (n 0) or delta (n 1) of query i of the block
  if (DIRECT && a.D < DP) {
    clear_lds(lds[0][0], 4 * kBytes);
    lds_barrier();
  }
  // Where a block is: head `g` of the group, queries from `i`.
  struct Place {
    int g, i;
  };
  auto following = [&](Place at) { return at.i + BQ < end ? Place{at.g, at.i + BQ} : Place{at.g + 1, first}; };
  auto fetch = [&](Place at_block, int into) {
    const int i0 = at_block.i, head = kv * a.group + at_block.g, last = end - 1;
    const T *q = at<T>(a.q, b, 0, head), *dout = at<T>(a.dout, b, 0, head);
    if constexpr (DIRECT) {
      if (i0 + BQ <= end) {
        qs.load(q + i0 * a.q.token, a.D, lds[into][0]);
        os.load(dout + i0 * a.dout.token, a.D, lds[into][1]);
      } else {
        qs.load_each(a.D, lds[into][0], [&](int r) { return q + min(i0 + r, last) * a.q.token; });
        os.load_each(a.D, lds[into][1], [&](int r) { return dout + min(i0 + r, last) * a.dout.token; });
      }
    } else {
      qs.load(a.D, [&](int r) { return q + min(i0 + r, last) * a.q.token; });
      os.load(a.D, [&](int r) { return dout + min(i0 + r, last) * a.dout.token; });
    }
    const int t = threadIdx.x;
    if (t < 2 * BQ) stat = a.stats[t / BQ * a.stat_rows + (static_cast<int64_t>(b) * a.heads + head) * a.Sq + min(i0 + t % BQ, last)];
  };
  auto put = [&](int into) {
    if constexpr (!DIRECT) {
      qs.store(a.D, lds[into][0]);
      os.store(a.D, lds[into][1]);
    }
    if (threadIdx.x < 2 * BQ) (&stats[into][0][0])[threadIdx.x] = stat;
  };
  Place block{0, 0};
  if (u0 < u1) {
    block = Place{u0 / blocks, first + u0 % blocks * BQ};
    fetch(block, 0);
    put(0);
  }
  for (int u = u0; u < u1; ++u) {
    const int now = (u - u0) & 1, i0 = block.i;
    if constexpr (DIRECT) landed();
    lds_barrier();  // the block is there, and the other buffer has been read
    block = following(block);
    if (u + 1 < u1) fetch(block, now ^ 1);
#pragma unroll
    for (int rb = 0; rb < BQ; rb += 32) {
      const int i1 = i0 + rb;
      if (i1 >= any_to || i1 + 32 <= any_from || (further && (u * (BQ / 32) + rb / 32) % kWaves != wave)) continue;
      const bool all = i1 >= all_from && i1 + 32 <= all_to;
      f32x16 p = zeros(), dp = zeros();
#pragma unroll
      for (int t = 0; t < R::kSteps; ++t) {
        p = multiply<T>(R::rows(lds[now][0], rb, t), k[t], p);
        if (kK) dp = multiply<T>(R::rows(lds[now][1], rb, t), value(t), dp);
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {  // queries 8 n + 4 half .. + 3
        const int r = rb + 8 * n + 4 * half;
        const f32x4 lse = *reinterpret_cast<const f32x4*>(&stats[now][0][r]), delta = *reinterpret_cast<const f32x4*>(&stats[now][1][r]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(p[4 * n + e], a.c, -lse[e]));
          p[4 * n + e] = x;
          if (kK) dp[4 * n + e] = x * (dp[4 * n + e] - delta[e]);
        }
      }
      if (!all) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool seen = static_cast<uint32_t>(i1 + key_of(i) - key_from) < key_span;
          p[i] = seen ? p[i] : 0.0f;
          if (kK) dp[i] = seen ? dp[i] : 0.0f;
        }
      }
      if constexpr (kV) {
        const Weights<T> weights(p);
#pragma unroll
        for (int d = 0; d < kColumns; ++d) dv[d] = multiply_columns<T, DP>(lds[now][1], rb, d, weights, dv[d]);
      }
      if constexpr (kK) {
        const Weights<T> weights(dp);
#pragma unroll
        for (int d = 0; d < kColumns; ++d) dk[d] = multiply_columns<T, DP>(lds[now][0], rb, d, weights, dk[d]);
      }
    }
    if (u + 1 < u1) put(now ^ 1);
  }
  if (further || parts > 1 || wave_key / 32 < jobs.strips) {
    const int64_t slot = parts > 1 ? job : static_cast<int64_t>(bk) * jobs.sink_tiles + tile;
    const int rows = further ? 32 : kRows;  // keys of a sum
    float* const into = (further ? jobs.further + (job * kWaves + wave) * 2 * 32 * a.pitch : jobs.partial + (slot * 2 * kRows + wave * 32) * a.pitch) +
                        lane % 32 * a.pitch;
    if constexpr (kK) {
#pragma unroll
      for (int d = 0; d < kColumns; ++d) store_sums(into, a.pitch, d, dk[d], a.scale);
    }
    if constexpr (kV) {
#pragma unroll
      for (int d = 0; d < kColumns; ++d) store_sums(into + static_cast<int64_t>(rows) * a.pitch, a.pitch, d, dv[d], 1.0f);
    }
  } else if (key < a.Sk) {
    if constexpr (kK) {
      T* const into = const_cast<T*>(at<T>(a.dk, b, key, kv));
#pragma unroll
      for (int d = 0; d < kColumns; ++d) store_sums(into, a.D, d, dk[d], a.scale);
    }
    if constexpr (kV) {
      T* const into = const_cast<T*>(at<T>(a.dv, b, key, kv));
#pragma unroll
      for (int d = 0; d < kColumns; ++d) store_sums(into, a.D, d, dv[d], 1.0f);
    }
  }
}

// sum += four floats of each of `count` rows, N of them on their way at a time.
template <int N>
__device__ __forceinline__ void add_parts(f32x4& sum, const float* p, int64_t step, int count) {
  for (int i = 0; i < count; i += N) {
    f32x4 v[N];
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = *reinterpret_cast<const f32x4*>(p + min(i + n, count - 1) * step);
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (i + n < count) sum += v[n];
  }
}
// The sums for a key, in their order: 32 lanes a key and gradient.  units: of 32 keys, all where tiles have parts, else the strips.
template <typename T>
__global__ __launch_bounds__(kThreads) void join_keys_kernel(Attn a, KeyJobs jobs, int units, int64_t all) {
  const int64_t n = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + threadIdx.x / 32;  // (bk, unit, gradient, key)
  if (n >= all) return;
  const int of_v = static_cast<int>(n / 32 % 2);
  const int64_t of_unit = n / 64;
  const int strip = static_cast<int>(of_unit % units), bk = static_cast<int>(of_unit / units), b = bk / a.kv_heads, kv = bk - b * a.kv_heads;
  const int key = strip * 32 + static_cast<int>(n % 32), tile = key / kRows, in_tile = key % kRows;
  if (key >= a.Sk) return;
  const int64_t of_tile = static_cast<int64_t>(bk) * (jobs.parts > 1 ? jobs.tiles : jobs.sink_tiles) + tile;
  const Heads& h = of_v ? a.dv : a.dk;
  T* const to = const_cast<T*>(at<T>(h, b, key, kv));
  const float* const parts = jobs.partial + ((of_tile * jobs.parts * 2 + of_v) * kRows + in_tile) * a.pitch;
  const float* const further = jobs.further + (((static_cast<int64_t>(bk) * jobs.strips + strip) * jobs.further_parts * kWaves * 2 + of_v) * 32 + key % 32) * a.pitch;
  const int further_sums = strip < jobs.strips ? jobs.further_parts * kWaves : 0;
  for (int d = threadIdx.x % 32 * 4; d < a.D; d += 128) {
    f32x4 sum = {0, 0, 0, 0};
    add_parts<4>(sum, parts + d, int64_t{2} * kRows * a.pitch, jobs.parts);
    add_parts<8>(sum, further + d, int64_t{2} * 32 * a.pitch, further_sums);
    store_four(to, a.D, d, sum);
  }
}

}  // namespace

tempo_status launch_window_attn_bwd(const WindowCall& c, tempo_dtype dt, hipStream_t st) {
  if (c.workspace_bytes < window_attn_workspace_bytes(c, dt, true)) return TEMPO_ERR_WORKSPACE;
  Attn a = attn_of(c);
  a.stats = static_cast<float*>(c.workspace);
  a.stat_rows = c.B * c.heads * c.Sq;
  KeyPlan p = key_plan(c);
  p.jobs.partial = a.stats + up(2 * a.stat_rows, 4) * 4;
  p.jobs.further = p.jobs.partial + p.partial_floats;
  return with_type(dt, [&](auto type) {
    using T = decltype(type);
    tempo_status s = with_width(c.D, [&](auto width) {
      constexpr int DP = decltype(width)::value, BK = sizeof(T) * DP <= 256 && sizeof(T) * DP > 128 ? 64 : 32;
      const tempo_status r = either(direct(c, dt, {c.k, c.v}), [&](auto straight) {
        return launch(rows_kernel<T, DP, BK, decltype(straight)::value>, c.B * c.kv_heads * a.tiles, st, a);
      });
      if (r != TEMPO_OK) return r;
      return either(direct(c, dt, {c.q, c.dout}), [&](auto straight) {
        constexpr bool DIRECT = decltype(straight)::value;
        if constexpr (sizeof(T) * DP > 512) {  // both gradients' sums of 256 float32 elements are more than a wave's registers
          const tempo_status of_v = launch(keys_kernel<T, DP, kOnlyV, DIRECT>, p.blocks, st, a, p.jobs);
          return of_v != TEMPO_OK ? of_v : launch(keys_kernel<T, DP, kOnlyK, DIRECT>, p.blocks, st, a, p.jobs);
        } else {
          return launch(keys_kernel<T, DP, kBoth, DIRECT>, p.blocks, st, a, p.jobs);
        }
      });
    });
    const int units = p.jobs.parts > 1 ? p.jobs.tiles * kWaves : p.jobs.strips;
    const int64_t keys = c.B * c.kv_heads * units * 2 * 32;
    if (s == TEMPO_OK && keys > 0) s = launch(join_keys_kernel<T>, up(keys, kThreads / 32), st, a, p.jobs, units, keys);
    return s;
  });
}

}  // namespace tempo
