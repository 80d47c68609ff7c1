// The place between two blocks of a pre-norm model: a norm of the block's output, its gate, the residual and the next block's norm,
//   n = post(f),  y = alpha x + beta gate n,  h = pre(y);   a norm: t^ = (t - mean) rstd (mean 0: RMS), t^ weight + bias.
// Backward from f, y and the norms' statistics, dy the gradient of y by the residual and dh that of h:
//   g = dh pre.weight,  d = dy + pre.rstd (g - y^ mean(g y^) - mean(g)),  dx = alpha d,
//   e = beta gate post.weight d,  df = post.rstd (e - f^ mean(e f^) - mean(e))         (mean(g) and mean(e) without RMS)
//   and of columns  C = sum f^ d,  F = sum d of each gate's rows,  D = sum dh y^,  E = sum dh:
//   dgate = beta (post.weight C + post.bias F),  dpost.weight = sum beta gate C,  dpost.bias = sum beta gate F,  dpre = D and E.
//
// Bound by the bytes of four tensors forward and six backward, each once: a row is held in registers by the waves of one workgroup, which
// walks rows and fetches the next while it reduces, keeps the parameters of its columns in registers and, backward, their sums, which a
// second kernel adds up in a fixed order.  8192 x 4096 bfloat16 forward 50.7 us (5.3 TB/s), 65536 x 4096 backward 546 (5.9 TB/s) and 13 for the column
// sums; 3063 x 1001 float32 backward, rows at any multiple of 4 bytes, 22 and 6.  A workgroup of 16 waves leaves 128 registers a lane, of which
// the backward spills some: rows of 513 to 1024 pieces 36 to 112 bytes a lane in bfloat16 (16384 x 8192 318 us, 5.1 TB/s, 16384 x 5120 243, 4.1), longer ones 320 to
// 576 (8192 x 16384 1168 us, 1.4 TB/s) and 40 to 220 in float32 (8192 x 8192 298 us, 5.4 TB/s); the forward only with biases, 8 to 76.
#include <algorithm>
#include <type_traits>

#include "launch_split.h"
#include "tempo_device.h"
#include "tempo_host.h"

namespace tempo {
namespace {

struct Norm {
  bool there, layer;
  const float *weight, *bias;  // null: 1 and 0
  float eps;
  float2* stats;               // [N] mean, rstd; forward: may be null
};
struct Residual {
  const void *x, *f, *y, *dy, *dh;  // backward: y is an input
  void *to_y, *h, *dx, *df;
  const float* gate;     // [groups, M] or null
  Norm post, pre;
  float alpha, beta;
  int64_t N, group_rows;  // rows of a gate
  uint32_t M;
  float inv;              // 1 / M
  int parts;              // workgroups of a gate's rows
  float* partial;         // backward: [groups * parts][sums][M]
};

template <typename T, int CH, int LANES, bool RAG>
struct Columns {
  static constexpr int V = Store<T>::kVec;
  int M, pieces, lane;
  __device__ __forceinline__ explicit Columns(int M_) : M(M_), pieces(RAG ? (M_ + V - 1) / V : M_ / V), lane(threadIdx.x) {}
  __device__ __forceinline__ int piece(int c) const { return c * LANES + lane; }
  __device__ __forceinline__ bool has(int c) const { return piece(c) < pieces; }
  __device__ __forceinline__ int at(int c) const { return piece_col<RAG, V>(piece(c), pieces, M); }
  __device__ __forceinline__ int dup(int c) const { return piece_dup<RAG, V>(piece(c), pieces, M); }
  __device__ __forceinline__ void load(const T* row, u32x4 (&to)[CH]) const {
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (has(c)) to[c] = ldg_piece<RAG>(row + at(c));
  }
  // A moved-back last piece shares elements with the piece before, which both lanes store.  Where that is another wave's, it alone stores them: in
  // place (y is x, dx is dy) it may have done so before this one loaded them, and what two lanes make of an element need not be the same to the
  // bit.  No sum takes them here.  Within a wave one instruction loads both pieces and one stores them; there single elements would
  // cost what the stores are (20000 x 101 float32 forward 9.9 us, 11.2 with them).
  __device__ __forceinline__ void store(T* row, int c, const float (&v)[V]) const {
    if (!has(c)) return;
    const int first = LANES > kWave && lane % kWave == 0 ? dup(c) : 0;
    if (!RAG || first == 0) return stg_piece<RAG>(row + at(c), Store<T>::pack(v));
#pragma unroll
    for (int i = 1; i < V; ++i)
      if (i >= first) Store<T>::store1(row + at(c) + i, v[i]);
  }
  __device__ __forceinline__ void floats(const float* p, float otherwise, float (&to)[CH][V]) const {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int i = 0; i < V; ++i) to[c][i] = otherwise;
      if (p && has(c)) load_floats_any<V>(p + at(c), to[c]);
    }
  }
  // Elements that a sum takes: those of the row, each once.
  template <typename F>
  __device__ __forceinline__ float sum(F&& of) const {
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (!has(c)) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) s += RAG && i < dup(c) ? 0.0f : of(c, i);
    }
    return s;
  }
};
// The rows of this workgroup, all of one gate: every parts-th, so that what the workgroups read and write at a time lies together
// (65536 x 4096 bfloat16 backward with its column sums 558 us; 612 where each has rows side by side).
struct Walk {
  int64_t group, first, end, step;
  __device__ __forceinline__ explicit Walk(const Residual& r) {
    group = blockIdx.x / r.parts;
    step = r.parts;
    first = group * r.group_rows + (blockIdx.x - group * r.parts);
    end = (group + 1) * r.group_rows;
  }
};

// Rows that are on their way while one is worked on: 65536 x 4096 bfloat16 backward with its column sums 558 us with two, 667 with one.
template <int CH>
constexpr int kAhead = CH == 1 ? 2 : 1;
// work(row, its turn, that modulo AHEAD as a constant)
template <int AHEAD, int I = 0, typename F>
__device__ __forceinline__ bool turns(const Walk& w, int64_t row, int turn, F&& work) {
  if constexpr (I < AHEAD) {
    if (row >= w.end) return false;
    work(row, turn, std::integral_constant<int, I>{});
    return turns<AHEAD, I + 1>(w, row + w.step, turn + 1, work);
  }
  return true;
}
template <int AHEAD, typename F>
__device__ __forceinline__ void each_row(const Walk& w, F&& work) {
  int turn = 0;
  for (int64_t row = w.first; turns<AHEAD>(w, row, turn, work); row += AHEAD * w.step) turn += AHEAD;
}

// Mean and 1 / sqrt(variance + eps) of a row; a sum at a time.
template <int LANES, typename C, typename F>
__device__ __forceinline__ float2 statistics(const C& at, const Norm& n, float inv, float* slots, F&& value) {
  float mean = 0.0f;
  if (n.layer) mean = row_reduce<LANES, false>(at.sum(value), slots) * inv;
  const float square = row_reduce<LANES, false>(at.sum([&](int c, int i) {
    const float d = value(c, i) - mean;
    return d * d;
  }), slots + LANES / kWave);
  // The compiler's square root and division: v_rsq_f32 alone is off by up to 2^-23.
  return make_float2(mean, 1.0f / sqrtf(square * inv + n.eps));
}

template <typename T, int WAVES, int CH, bool RAG, bool BIAS>
__global__ __launch_bounds__(WAVES* kWave) void forward_kernel(Residual r) {
  constexpr int V = Store<T>::kVec, LANES = WAVES * kWave;
  __shared__ float slots[2][4 * WAVES];  // of rows in turn
  const Columns<T, CH, LANES, RAG> at(r.M);
  const Walk walk(r);
  const int64_t M = r.M;
  constexpr int AHEAD = kAhead<CH>;
  u32x4 x[AHEAD][CH], f[AHEAD][CH];
  auto fetch = [&](int64_t row, int to) {
    at.load(static_cast<const T*>(r.x) + row * M, x[to]);
    at.load(static_cast<const T*>(r.f) + row * M, f[to]);
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (walk.first + i * walk.step < walk.end) fetch(walk.first + i * walk.step, i);
  float by[CH][V], more[BIAS ? CH : 1][V], weight[CH][V], bias[BIAS ? CH : 1][V];  // of f^ and of y^
  {
    float gate[CH][V];
    at.floats(r.gate ? r.gate + walk.group * M : nullptr, 1.0f, gate);
    at.floats(r.post.weight, 1.0f, by);
    at.floats(r.pre.weight, 1.0f, weight);
    if constexpr (BIAS) {
      at.floats(r.post.bias, 0.0f, more);
      at.floats(r.pre.bias, 0.0f, bias);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        by[c][i] *= r.beta * gate[c][i];
        if constexpr (BIAS) more[c][i] *= r.beta * gate[c][i];
      }
  }
  each_row<AHEAD>(walk, [&](int64_t row, int turn, auto slot) {
    u32x4 xs[CH];
    float v[CH][V], y[CH][V];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      xs[c] = x[slot][c];
      Store<T>::unpack(f[slot][c], v[c]);
    }
    if (row + AHEAD * walk.step < walk.end) fetch(row + AHEAD * walk.step, slot);
    float2 st = make_float2(0.0f, 1.0f);
    if (r.post.there) {
      st = statistics<LANES>(at, r.post, r.inv, slots[turn & 1], [&](int c, int i) { return v[c][i]; });
      if (r.post.stats && threadIdx.x == 0) r.post.stats[row] = st;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float xv[V];
      Store<T>::unpack(xs[c], xv);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float n = (v[c][i] - st.x) * st.y * by[c][i];
        if constexpr (BIAS) n += more[c][i];
        y[c][i] = fmaf(r.alpha, xv[i], n);
      }
      // The norm is of what the residual holds, which is what the backward has of it.
      Store<T>::unpack(Store<T>::pack(y[c]), y[c]);
      at.store(static_cast<T*>(r.to_y) + row * M, c, y[c]);
    }
    if (!r.pre.there) return;
    st = statistics<LANES>(at, r.pre, r.inv, slots[turn & 1] + 2 * WAVES, [&](int c, int i) { return y[c][i]; });
    if (r.pre.stats && threadIdx.x == 0) r.pre.stats[row] = st;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        y[c][i] = (y[c][i] - st.x) * st.y * weight[c][i];
        if constexpr (BIAS) y[c][i] += bias[c][i];
      }
      at.store(static_cast<T*>(r.h) + row * M, c, y[c]);
    }
  });
}

// SUMS: 2 (C, D) or 4 (C, D, F, E).
template <typename T, int WAVES, int CH, bool RAG, int SUMS>
__global__ __launch_bounds__(WAVES* kWave) void backward_kernel(Residual r) {
  constexpr int V = Store<T>::kVec, LANES = WAVES * kWave;
  __shared__ float2 slots[2][2][WAVES];  // of rows in turn
  const Columns<T, CH, LANES, RAG> at(r.M);
  const Walk walk(r);
  const int64_t M = r.M;
  constexpr int AHEAD = kAhead<CH>;
  u32x4 dys[AHEAD][CH], dhs[AHEAD][CH], fs[AHEAD][CH], ys[AHEAD][CH];
  float2 pres[AHEAD], posts[AHEAD];
  auto fetch = [&](int64_t row, int to) {
    if (r.dy) at.load(static_cast<const T*>(r.dy) + row * M, dys[to]);
    if (r.pre.there) {
      at.load(static_cast<const T*>(r.dh) + row * M, dhs[to]);
      at.load(static_cast<const T*>(r.y) + row * M, ys[to]);
      pres[to] = r.pre.stats[row];
    }
    at.load(static_cast<const T*>(r.f) + row * M, fs[to]);
    if (r.post.there) posts[to] = r.post.stats[row];
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
#pragma unroll
    for (int c = 0; c < CH; ++c) dys[i][c] = dhs[i][c] = fs[i][c] = ys[i][c] = u32x4{0, 0, 0, 0};
    pres[i] = make_float2(0.0f, 0.0f), posts[i] = make_float2(0.0f, 1.0f);
    if (walk.first + i * walk.step < walk.end) fetch(walk.first + i * walk.step, i);
  }
  float by[CH][V], weight[CH][V], sums[SUMS][CH][V];
  {
    float gate[CH][V];
    at.floats(r.gate ? r.gate + walk.group * M : nullptr, 1.0f, gate);
    at.floats(r.post.weight, 1.0f, by);
    at.floats(r.pre.weight, 1.0f, weight);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        by[c][i] *= r.beta * gate[c][i];
#pragma unroll
        for (int s = 0; s < SUMS; ++s) sums[s][c][i] = 0.0f;
      }
  }
  each_row<AHEAD>(walk, [&](int64_t row, int turn, auto slot) {
    u32x4 dy[CH], dh[CH], f[CH], y[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) dy[c] = dys[slot][c], dh[c] = dhs[slot][c], f[c] = fs[slot][c], y[c] = ys[slot][c];
    const float2 pre = pres[slot], post = posts[slot];
    if (row + AHEAD * walk.step < walk.end) fetch(row + AHEAD * walk.step, slot);
    float d[CH][V], v[CH][V], g[CH][V];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      Store<T>::unpack(dh[c], g[c]);
      Store<T>::unpack(y[c], v[c]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[c][i] = (v[c][i] - pre.x) * pre.y;
        sums[1][c][i] = fmaf(g[c][i], v[c][i], sums[1][c][i]);
        if constexpr (SUMS == 4) sums[3][c][i] += g[c][i];
        g[c][i] *= weight[c][i];
      }
    }
    float s1 = 0.0f, s2 = 0.0f;
    if (r.pre.there) {
      s1 = at.sum([&](int c, int i) { return g[c][i] * v[c][i]; });
      if (r.pre.layer) s2 = at.sum([&](int c, int i) { return g[c][i]; });
      row_sum2<LANES>(s1, s2, slots[turn & 1][0]);
    }
    s1 *= r.inv, s2 *= r.inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float out[V];
      Store<T>::unpack(dy[c], d[c]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        d[c][i] = fmaf(pre.y, g[c][i] - v[c][i] * s1 - s2, d[c][i]);
        out[i] = r.alpha * d[c][i];
      }
      at.store(static_cast<T*>(r.dx) + row * M, c, out);
      Store<T>::unpack(f[c], v[c]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[c][i] = (v[c][i] - post.x) * post.y;
        sums[0][c][i] = fmaf(v[c][i], d[c][i], sums[0][c][i]);
        if constexpr (SUMS == 4) sums[2][c][i] += d[c][i];
        g[c][i] = d[c][i] * by[c][i];
      }
    }
    s1 = s2 = 0.0f;
    if (r.post.there) {
      s1 = at.sum([&](int c, int i) { return g[c][i] * v[c][i]; });
      if (r.post.layer) s2 = at.sum([&](int c, int i) { return g[c][i]; });
      row_sum2<LANES>(s1, s2, slots[turn & 1][1]);
    }
    s1 *= r.inv, s2 *= r.inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int i = 0; i < V; ++i) g[c][i] = post.y * (g[c][i] - v[c][i] * s1 - s2);
      at.store(static_cast<T*>(r.df) + row * M, c, g[c]);
    }
  });
  if (!r.partial) return;
#pragma unroll
  for (int s = 0; s < SUMS; ++s) {
    float* const to = r.partial + (static_cast<int64_t>(blockIdx.x) * SUMS + s) * M;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (!at.has(c)) continue;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (!RAG || i >= at.dup(c)) to[at.at(c) + i] = sums[s][c][i];
    }
  }
}

// Rows of any length, longer than a workgroup's registers or shorter than a piece: element by element, read again for each step.  Columns are
// counted without a sign: the last turn passes 2^31 where M is next to it.
constexpr int kAnyThreads = 1024;
template <typename F>
__device__ __forceinline__ float sum_of_row(uint32_t M, float* slots, F&& of) {
  float s = 0.0f;
  for (uint32_t c = threadIdx.x; c < M; c += kAnyThreads) s += of(c);
  s = row_reduce<kAnyThreads, false>(s, slots);
  lds_barrier();
  return s;
}
template <typename F>
__device__ __forceinline__ float2 statistics_of_row(const Norm& n, uint32_t M, float inv, float* slots, F&& value) {
  const float mean = n.layer ? sum_of_row(M, slots, value) * inv : 0.0f;
  const float square = sum_of_row(M, slots, [&](uint32_t c) { return (value(c) - mean) * (value(c) - mean); });
  return make_float2(mean, 1.0f / sqrtf(square * inv + n.eps));
}
__device__ __forceinline__ float param(const float* p, uint32_t c, float otherwise) { return p ? p[c] : otherwise; }

template <typename T>
__global__ __launch_bounds__(kAnyThreads) void forward_any_kernel(Residual r) {
  __shared__ float slots[kAnyThreads / kWave];
  const Walk walk(r);
  const int64_t M = r.M;
  const float* gate = r.gate ? r.gate + walk.group * M : nullptr;
  for (int64_t row = walk.first; row < walk.end; row += walk.step) {
    const T *x = static_cast<const T*>(r.x) + row * M, *f = static_cast<const T*>(r.f) + row * M;
    T* const y = static_cast<T*>(r.to_y) + row * M;
    float2 st = make_float2(0.0f, 1.0f);
    if (r.post.there) {
      st = statistics_of_row(r.post, r.M, r.inv, slots, [&](uint32_t c) { return Store<T>::load1(f + c); });
      if (r.post.stats && threadIdx.x == 0) r.post.stats[row] = st;
    }
    for (uint32_t c = threadIdx.x; c < r.M; c += kAnyThreads) {
      const float g = r.beta * param(gate, c, 1.0f);
      const float n = (Store<T>::load1(f + c) - st.x) * st.y * (g * param(r.post.weight, c, 1.0f)) + g * param(r.post.bias, c, 0.0f);
      Store<T>::store1(y + c, fmaf(r.alpha, Store<T>::load1(x + c), n));
    }
    if (!r.pre.there) continue;
    st = statistics_of_row(r.pre, r.M, r.inv, slots, [&](uint32_t c) { return Store<T>::load1(y + c); });  // a lane's own
    if (r.pre.stats && threadIdx.x == 0) r.pre.stats[row] = st;
    for (uint32_t c = threadIdx.x; c < r.M; c += kAnyThreads)
      Store<T>::store1(static_cast<T*>(r.h) + row * M + c, (Store<T>::load1(y + c) - st.x) * st.y * param(r.pre.weight, c, 1.0f) +
                                                               param(r.pre.bias, c, 0.0f));
  }
}

template <typename T, int SUMS>
__global__ __launch_bounds__(kAnyThreads) void backward_any_kernel(Residual r) {
  __shared__ float slots[kAnyThreads / kWave];
  const Walk walk(r);
  const int64_t M = r.M;
  const float* gate = r.gate ? r.gate + walk.group * M : nullptr;
  float* const sums = r.partial ? r.partial + static_cast<int64_t>(blockIdx.x) * SUMS * M : nullptr;
  if (sums)
    for (uint32_t c = threadIdx.x; c < r.M; c += kAnyThreads)
      for (int s = 0; s < SUMS; ++s) sums[s * M + c] = 0.0f;
  for (int64_t row = walk.first; row < walk.end; row += walk.step) {
    auto element = [&](const void* t, uint32_t c) { return t ? Store<T>::load1(static_cast<const T*>(t) + row * M + c) : 0.0f; };
    const float2 pre = r.pre.there ? r.pre.stats[row] : make_float2(0.0f, 0.0f), post = r.post.there ? r.post.stats[row] : make_float2(0.0f, 1.0f);
    auto y_hat = [&](uint32_t c) { return r.pre.there ? (element(r.y, c) - pre.x) * pre.y : 0.0f; };
    auto f_hat = [&](uint32_t c) { return (element(r.f, c) - post.x) * post.y; };
    auto g = [&](uint32_t c) { return r.pre.there ? element(r.dh, c) * param(r.pre.weight, c, 1.0f) : 0.0f; };
    float s1 = 0.0f, s2 = 0.0f;
    if (r.pre.there) {
      s1 = sum_of_row(r.M, slots, [&](uint32_t c) { return g(c) * y_hat(c); }) * r.inv;
      if (r.pre.layer) s2 = sum_of_row(r.M, slots, g) * r.inv;
    }
    auto d = [&](uint32_t c) { return fmaf(pre.y, g(c) - y_hat(c) * s1 - s2, element(r.dy, c)); };
    auto e = [&](uint32_t c) { return d(c) * (r.beta * param(gate, c, 1.0f) * param(r.post.weight, c, 1.0f)); };
    float t1 = 0.0f, t2 = 0.0f;
    if (r.post.there) {
      t1 = sum_of_row(r.M, slots, [&](uint32_t c) { return e(c) * f_hat(c); }) * r.inv;
      if (r.post.layer) t2 = sum_of_row(r.M, slots, e) * r.inv;
    }
    for (uint32_t c = threadIdx.x; c < r.M; c += kAnyThreads) {
      const float dc = d(c), fc = f_hat(c), df = post.y * (e(c) - fc * t1 - t2);
      if (sums) {
        sums[c] = fmaf(fc, dc, sums[c]);
        if (r.pre.there) sums[M + c] = fmaf(element(r.dh, c), y_hat(c), sums[M + c]);
        if constexpr (SUMS == 4) {
          sums[2 * M + c] += dc;
          if (r.pre.there) sums[3 * M + c] += element(r.dh, c);
        }
      }
      Store<T>::store1(static_cast<T*>(r.dx) + row * M + c, r.alpha * dc);
      Store<T>::store1(static_cast<T*>(r.df) + row * M + c, df);
    }
  }
}

// The sums of all workgroups: 16 columns by 64 lanes, of which `share` take the parts of a gate's rows in turn (all of them where there is
// one gate), those of other gates at the same time; added up in a fixed order.
struct Sums {
  const float* partial;
  int64_t groups;
  int parts, sums;
  uint32_t M;
  int share;
  const float *gate, *post_weight, *post_bias;
  float beta;
  float *dgate, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
};
constexpr int kSumLanes = 64, kSumColumns = 16;
template <int SUMS>
__global__ __launch_bounds__(kSumColumns* kSumLanes) void columns_kernel(Sums s, uint32_t first_block) {
  __shared__ float of_lanes[SUMS][kSumLanes][kSumColumns];
  const int x = threadIdx.x % kSumColumns, lane = threadIdx.x / kSumColumns, in_share = lane % s.share;
  const uint32_t column = (first_block + blockIdx.x) * kSumColumns + x;
  const bool exists = column < s.M, leads = in_share == 0 && exists;
  const int at_once = kSumLanes / s.share;
  const int64_t M = s.M;
  float total[SUMS] = {};  // of a leader: dpost.weight, D, dpost.bias, E
  for (int64_t first = 0; first < s.groups; first += at_once) {
    const int64_t group = first + lane / s.share;
    float v[SUMS] = {};
    if (exists && group < s.groups) {
      const float* p = s.partial + group * s.parts * SUMS * M + column;
#pragma unroll 4
      for (int part = in_share; part < s.parts; part += s.share) {
#pragma unroll
        for (int n = 0; n < SUMS; ++n) v[n] += p[(static_cast<int64_t>(part) * SUMS + n) * M];
      }
    }
    if (s.share > 1) {
#pragma unroll
      for (int n = 0; n < SUMS; ++n) of_lanes[n][lane][x] = v[n];
      lds_barrier();
      if (leads) {
        for (int l = 1; l < s.share; ++l)
#pragma unroll
          for (int n = 0; n < SUMS; ++n) v[n] += of_lanes[n][lane + l][x];
      }
      lds_barrier();
    }
    if (leads && group < s.groups) {
      const float by = s.beta * param(s.gate ? s.gate + group * M : nullptr, column, 1.0f);
      float d = param(s.post_weight, column, 1.0f) * v[0];
      if constexpr (SUMS == 4) d += param(s.post_bias, column, 0.0f) * v[2];
      if (s.dgate) s.dgate[group * M + column] = s.beta * d;
      total[0] = fmaf(by, v[0], total[0]);
      total[1] += v[1];
      if constexpr (SUMS == 4) {
        total[2] = fmaf(by, v[2], total[2]);
        total[3] += v[3];
      }
    }
  }
#pragma unroll
  for (int n = 0; n < SUMS; ++n) of_lanes[n][lane][x] = total[n];
  lds_barrier();
  if (lane != 0 || !exists) return;
  for (int l = s.share; l < kSumLanes; l += s.share)
#pragma unroll
    for (int n = 0; n < SUMS; ++n) total[n] += of_lanes[n][l][x];
  if (s.dpost_weight) s.dpost_weight[column] = total[0];
  if (s.dpre_weight) s.dpre_weight[column] = total[1];
  if constexpr (SUMS == 4) {
    if (s.dpost_bias) s.dpost_bias[column] = total[2];
    if (s.dpre_bias) s.dpre_bias[column] = total[3];
  }
}

// ---- plans ----------------------------------------------------------------------------------------------------------------
struct Shape {
  int waves, pieces;  // 0 waves: any length
};
Shape shape_of(int64_t M, tempo_dtype dt) {
  const int V = dt == TEMPO_F32 ? 4 : 8;
  const int64_t pieces = (M + V - 1) / V;
  if (M < V || pieces > 2048) return {0, 0};
  if (pieces <= 64) return {1, 1};
  if (pieces <= 128) return {2, 1};
  if (pieces <= 256) return {4, 1};
  if (pieces <= 512) return {8, 1};
  if (pieces <= 1024) return {16, 1};
  return {16, 2};
}
// Workgroups: rows that a gate is for are cut into parts.
struct Plan {
  Shape shape;
  int64_t groups, group_rows, part_rows, parts;
};
Plan plan_of(const ResidualCall& c, tempo_dtype dt, bool back) {
  Plan p{};
  p.shape = shape_of(c.M, dt);
  p.groups = c.gate ? c.groups : 1;
  p.group_rows = c.N / p.groups;
  // 32 waves for each compute unit, and backward 8 rows each where there are as many for all of them, so that the sums are a small part of what
  // is read and written.  us with 2, 4, 8 and 12: 3063 x 1001 float32 42.8, 33.4, 29.6, 26.2, 4096 x 1024 bfloat16 30.9, 24.0, 22.0, 24.3.
  const int64_t cus = compute_units(), blocks = cus * 32 / std::max(p.shape.waves, 1);
  p.part_rows = std::max<int64_t>((c.N + blocks - 1) / blocks, 1);
  if (back) p.part_rows = std::max(p.part_rows, std::min<int64_t>(8, (c.N + cus - 1) / cus));
  p.parts = std::max<int64_t>((p.group_rows + p.part_rows - 1) / p.part_rows, 1);
  return p;
}
int sums_of(const ResidualCall& c) { return c.dpost_bias || c.dpre_bias || (c.dgate && c.post && c.post->bias) ? 4 : 2; }
bool wants_columns(const ResidualCall& c) { return c.dgate || c.dpost_weight || c.dpost_bias || c.dpre_weight || c.dpre_bias; }
Norm norm_of(const tempo_norm* n) {
  if (!n) return Norm{};
  return {true, n->kind == TEMPO_NORM_LAYER, n->weight, n->bias, n->eps, reinterpret_cast<float2*>(n->stats)};
}
Residual residual_of(const ResidualCall& c, const Plan& p) {
  Residual r{};
  r.x = c.x, r.f = c.f, r.y = c.y, r.dy = c.dy, r.dh = c.dh, r.to_y = c.to_y, r.h = c.h, r.dx = c.dx, r.df = c.df;
  r.gate = c.gate;
  r.post = norm_of(c.post), r.pre = norm_of(c.pre);
  r.alpha = c.alpha, r.beta = c.beta;
  r.N = c.N, r.M = static_cast<uint32_t>(c.M);
  r.group_rows = p.group_rows;
  r.inv = 1.0f / static_cast<float>(c.M);
  r.parts = static_cast<int>(p.parts);
  return r;
}
template <typename T, typename F>
bool with_shape(const Shape& s, int64_t M, F&& f) {
  auto by_row = [&](auto waves, auto pieces) {
    if (M % Store<T>::kVec == 0) f(waves, pieces, std::false_type{});
    else f(waves, pieces, std::true_type{});
    return true;
  };
  const std::integral_constant<int, 1> one;
  switch (s.waves) {
    case 1: return by_row(one, one);
    case 2: return by_row(std::integral_constant<int, 2>{}, one);
    case 4: return by_row(std::integral_constant<int, 4>{}, one);
    case 8: return by_row(std::integral_constant<int, 8>{}, one);
    case 16: return s.pieces == 1 ? by_row(std::integral_constant<int, 16>{}, one) : by_row(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
    default: return false;
  }
}

}  // namespace

bool residual_norm_takes(const ResidualCall& c, tempo_dtype dt) {
  const Plan p = plan_of(c, dt, false);  // more parts than backward
  return p.groups * p.parts < int64_t{1} << 22;  // launches of less than 2^32 lanes
}

size_t residual_norm_workspace_bytes(const ResidualCall& c, tempo_dtype dt) {
  const Plan p = plan_of(c, dt, true);
  return static_cast<size_t>(p.groups) * p.parts * 4 * c.M * sizeof(float);
}

tempo_status launch_residual_norm_fwd(const ResidualCall& c, tempo_dtype dt, hipStream_t st) {
  const Plan p = plan_of(c, dt, false);
  const Residual r = residual_of(c, p);
  const dim3 grid(static_cast<uint32_t>(p.groups * p.parts));
  const bool bias = (c.post && c.post->bias) || (c.pre && c.pre->bias);
  auto of_type = [&](auto type) {
    using T = decltype(type);
    const bool fits = with_shape<T>(p.shape, c.M, [&](auto waves, auto pieces, auto ragged) {
      constexpr int W = decltype(waves)::value, CH = decltype(pieces)::value;
      constexpr bool RAG = decltype(ragged)::value;
      if (bias) hipLaunchKernelGGL((forward_kernel<T, W, CH, RAG, true>), grid, dim3(W * kWave), 0, st, r);
      else hipLaunchKernelGGL((forward_kernel<T, W, CH, RAG, false>), grid, dim3(W * kWave), 0, st, r);
    });
    if (!fits) hipLaunchKernelGGL(forward_any_kernel<T>, grid, dim3(kAnyThreads), 0, st, r);
    return launch_status();
  };
  return dt == TEMPO_F32 ? of_type(float{}) : of_type(bf16_t{});
}

tempo_status launch_residual_norm_bwd(const ResidualCall& c, tempo_dtype dt, hipStream_t st) {
  const Plan p = plan_of(c, dt, true);
  Residual r = residual_of(c, p);
  const int sums = sums_of(c);
  if (wants_columns(c)) {
    if (c.workspace_bytes < static_cast<size_t>(p.groups) * p.parts * sums * c.M * sizeof(float)) return TEMPO_ERR_WORKSPACE;
    r.partial = static_cast<float*>(c.workspace);
  }
  const dim3 grid(static_cast<uint32_t>(p.groups * p.parts));
  auto of_type = [&](auto type) {
    using T = decltype(type);
    const bool fits = with_shape<T>(p.shape, c.M, [&](auto waves, auto pieces, auto ragged) {
      constexpr int W = decltype(waves)::value, CH = decltype(pieces)::value;
      constexpr bool RAG = decltype(ragged)::value;
      if (sums == 4) hipLaunchKernelGGL((backward_kernel<T, W, CH, RAG, 4>), grid, dim3(W * kWave), 0, st, r);
      else hipLaunchKernelGGL((backward_kernel<T, W, CH, RAG, 2>), grid, dim3(W * kWave), 0, st, r);
    });
    if (!fits && sums == 4) hipLaunchKernelGGL((backward_any_kernel<T, 4>), grid, dim3(kAnyThreads), 0, st, r);
    if (!fits && sums == 2) hipLaunchKernelGGL((backward_any_kernel<T, 2>), grid, dim3(kAnyThreads), 0, st, r);
    return launch_status();
  };
  const tempo_status s = dt == TEMPO_F32 ? of_type(float{}) : of_type(bf16_t{});
  if (s != TEMPO_OK || !r.partial) return s;
  int share = kSumLanes;
  while (share > 1 && kSumLanes / share < p.groups) share /= 2;
  const Sums all{r.partial, p.groups, r.parts, sums, r.M, share, c.gate, c.post ? c.post->weight : nullptr, c.post ? c.post->bias : nullptr, c.beta,
                 c.dgate, c.dpost_weight, c.dpost_bias, c.dpre_weight, c.dpre_bias};
  const dim3 lanes(kSumColumns * kSumLanes);
  const bool ok = split_launch((c.M + kSumColumns - 1) / kSumColumns, most_groups(INT64_MAX, lanes.x), [&](uint32_t first, uint32_t blocks) {
    if (sums == 4) hipLaunchKernelGGL(columns_kernel<4>, dim3(blocks), lanes, 0, st, all, first);
    else hipLaunchKernelGGL(columns_kernel<2>, dim3(blocks), lanes, 0, st, all, first);
    return launch_status() == TEMPO_OK;
  });
  return ok ? TEMPO_OK : TEMPO_ERR_LAUNCH;
}

}  // namespace tempo
