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
// second kernel adds up in a fixed order.
#include <algorithm>
#include <type_traits>

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
  int M;
  float inv;              // 1 / M
  int parts;              // workgroups of a gate's rows
  int64_t part_rows;
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
// The rows [first, end) of this workgroup, all of one gate.
struct Walk {
  int64_t group, first, end;
  __device__ __forceinline__ explicit Walk(const Residual& r) {
    group = blockIdx.x / r.parts;
    const int64_t base = group * r.group_rows, from = static_cast<int64_t>(blockIdx.x - group * r.parts) * r.part_rows;
    first = base + (from < r.group_rows ? from : r.group_rows);
    const int64_t to = from + r.part_rows;
    end = base + (to < r.group_rows ? to : r.group_rows);
  }
};

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
  u32x4 x[CH], f[CH], next_x[CH], next_f[CH];
  auto fetch = [&](int64_t row) {
    at.load(static_cast<const T*>(r.x) + row * M, next_x);
    at.load(static_cast<const T*>(r.f) + row * M, next_f);
  };
  if (walk.first < walk.end) fetch(walk.first);
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
  for (int64_t row = walk.first; row < walk.end; ++row) {
#pragma unroll
    for (int c = 0; c < CH; ++c) x[c] = next_x[c], f[c] = next_f[c];
    if (row + 1 < walk.end) fetch(row + 1);
    float v[CH][V], y[CH][V];
#pragma unroll
    for (int c = 0; c < CH; ++c) Store<T>::unpack(f[c], v[c]);
    float2 st = make_float2(0.0f, 1.0f);
    if (r.post.there) {
      st = statistics<LANES>(at, r.post, r.inv, slots[row & 1], [&](int c, int i) { return v[c][i]; });
      if (r.post.stats && threadIdx.x == 0) r.post.stats[row] = st;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float xv[V];
      Store<T>::unpack(x[c], xv);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float n = (v[c][i] - st.x) * st.y * by[c][i];
        if constexpr (BIAS) n += more[c][i];
        y[c][i] = fmaf(r.alpha, xv[i], n);
      }
      // The norm is of what the residual holds, which is what the backward has of it.
      const u32x4 w = Store<T>::pack(y[c]);
      if (at.has(c)) stg_piece<RAG>(static_cast<T*>(r.to_y) + row * M + at.at(c), w);
      Store<T>::unpack(w, y[c]);
    }
    if (!r.pre.there) continue;
    st = statistics<LANES>(at, r.pre, r.inv, slots[row & 1] + 2 * WAVES, [&](int c, int i) { return y[c][i]; });
    if (r.pre.stats && threadIdx.x == 0) r.pre.stats[row] = st;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        y[c][i] = (y[c][i] - st.x) * st.y * weight[c][i];
        if constexpr (BIAS) y[c][i] += bias[c][i];
      }
      if (at.has(c)) stg_piece<RAG>(static_cast<T*>(r.h) + row * M + at.at(c), Store<T>::pack(y[c]));
    }
  }
}

// SUMS: 2 (C, D) or 4 (C, D, F, E).
template <typename T, int WAVES, int CH, bool RAG, int SUMS>
__global__ __launch_bounds__(WAVES* kWave) void backward_kernel(Residual r) {
  constexpr int V = Store<T>::kVec, LANES = WAVES * kWave;
  __shared__ float2 slots[2][2][WAVES];  // of rows in turn
  const Columns<T, CH, LANES, RAG> at(r.M);
  const Walk walk(r);
  const int64_t M = r.M;
  u32x4 dy[CH], dh[CH], f[CH], y[CH], next_dy[CH], next_dh[CH], next_f[CH], next_y[CH];
  float2 pre, post, next_pre = make_float2(0.0f, 0.0f), next_post = make_float2(0.0f, 1.0f);
  auto fetch = [&](int64_t row) {
    if (r.dy) at.load(static_cast<const T*>(r.dy) + row * M, next_dy);
    if (r.pre.there) {
      at.load(static_cast<const T*>(r.dh) + row * M, next_dh);
      at.load(static_cast<const T*>(r.y) + row * M, next_y);
      next_pre = r.pre.stats[row];
    }
    at.load(static_cast<const T*>(r.f) + row * M, next_f);
    if (r.post.there) next_post = r.post.stats[row];
  };
#pragma unroll
  for (int c = 0; c < CH; ++c) next_dy[c] = next_dh[c] = next_f[c] = next_y[c] = u32x4{0, 0, 0, 0};
  if (walk.first < walk.end) fetch(walk.first);
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
  for (int64_t row = walk.first; row < walk.end; ++row) {
#pragma unroll
    for (int c = 0; c < CH; ++c) dy[c] = next_dy[c], dh[c] = next_dh[c], f[c] = next_f[c], y[c] = next_y[c];
    pre = next_pre, post = next_post;
    if (row + 1 < walk.end) fetch(row + 1);
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
      row_sum2<LANES>(s1, s2, slots[row & 1][0]);
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
      if (at.has(c)) stg_piece<RAG>(static_cast<T*>(r.dx) + row * M + at.at(c), Store<T>::pack(out));
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
      row_sum2<LANES>(s1, s2, slots[row & 1][1]);
    }
    s1 *= r.inv, s2 *= r.inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int i = 0; i < V; ++i) g[c][i] = post.y * (g[c][i] - v[c][i] * s1 - s2);
      if (at.has(c)) stg_piece<RAG>(static_cast<T*>(r.df) + row * M + at.at(c), Store<T>::pack(g[c]));
    }
  }
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

// Rows of any length, longer than a workgroup's registers or shorter than a piece: element by element, read again for each step.
constexpr int kAnyThreads = 1024;
template <typename F>
__device__ __forceinline__ float sum_of_row(int M, float* slots, F&& of) {
  float s = 0.0f;
  for (int c = threadIdx.x; c < M; c += kAnyThreads) s += of(c);
  s = row_reduce<kAnyThreads, false>(s, slots);
  lds_barrier();
  return s;
}
template <typename F>
__device__ __forceinline__ float2 statistics_of_row(const Norm& n, int M, float inv, float* slots, F&& value) {
  const float mean = n.layer ? sum_of_row(M, slots, value) * inv : 0.0f;
  const float square = sum_of_row(M, slots, [&](int c) { return (value(c) - mean) * (value(c) - mean); });
  return make_float2(mean, 1.0f / sqrtf(square * inv + n.eps));
}
__device__ __forceinline__ float param(const float* p, int c, float otherwise) { return p ? p[c] : otherwise; }

template <typename T>
__global__ __launch_bounds__(kAnyThreads) void forward_any_kernel(Residual r) {
  __shared__ float slots[kAnyThreads / kWave];
  const Walk walk(r);
  const int64_t M = r.M;
  const float* gate = r.gate ? r.gate + walk.group * M : nullptr;
  for (int64_t row = walk.first; row < walk.end; ++row) {
    const T *x = static_cast<const T*>(r.x) + row * M, *f = static_cast<const T*>(r.f) + row * M;
    T* const y = static_cast<T*>(r.to_y) + row * M;
    float2 st = make_float2(0.0f, 1.0f);
    if (r.post.there) {
      st = statistics_of_row(r.post, r.M, r.inv, slots, [&](int c) { return Store<T>::load1(f + c); });
      if (r.post.stats && threadIdx.x == 0) r.post.stats[row] = st;
    }
    for (int c = threadIdx.x; c < r.M; c += kAnyThreads) {
      const float g = r.beta * param(gate, c, 1.0f);
      const float n = (Store<T>::load1(f + c) - st.x) * st.y * (g * param(r.post.weight, c, 1.0f)) + g * param(r.post.bias, c, 0.0f);
      Store<T>::store1(y + c, fmaf(r.alpha, Store<T>::load1(x + c), n));
    }
    if (!r.pre.there) continue;
    st = statistics_of_row(r.pre, r.M, r.inv, slots, [&](int c) { return Store<T>::load1(y + c); });  // a lane's own
    if (r.pre.stats && threadIdx.x == 0) r.pre.stats[row] = st;
    for (int c = threadIdx.x; c < r.M; c += kAnyThreads)
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
    for (int c = threadIdx.x; c < r.M; c += kAnyThreads)
      for (int s = 0; s < SUMS; ++s) sums[s * M + c] = 0.0f;
  for (int64_t row = walk.first; row < walk.end; ++row) {
    auto element = [&](const void* t, int c) { return t ? Store<T>::load1(static_cast<const T*>(t) + row * M + c) : 0.0f; };
    const float2 pre = r.pre.there ? r.pre.stats[row] : make_float2(0.0f, 0.0f), post = r.post.there ? r.post.stats[row] : make_float2(0.0f, 1.0f);
    auto y_hat = [&](int c) { return r.pre.there ? (element(r.y, c) - pre.x) * pre.y : 0.0f; };
    auto f_hat = [&](int c) { return (element(r.f, c) - post.x) * post.y; };
    auto g = [&](int c) { return r.pre.there ? element(r.dh, c) * param(r.pre.weight, c, 1.0f) : 0.0f; };
    float s1 = 0.0f, s2 = 0.0f;
    if (r.pre.there) {
      s1 = sum_of_row(r.M, slots, [&](int c) { return g(c) * y_hat(c); }) * r.inv;
      if (r.pre.layer) s2 = sum_of_row(r.M, slots, g) * r.inv;
    }
    auto d = [&](int c) { return fmaf(pre.y, g(c) - y_hat(c) * s1 - s2, element(r.dy, c)); };
    auto e = [&](int c) { return d(c) * (r.beta * param(gate, c, 1.0f) * param(r.post.weight, c, 1.0f)); };
    float t1 = 0.0f, t2 = 0.0f;
    if (r.post.there) {
      t1 = sum_of_row(r.M, slots, [&](int c) { return e(c) * f_hat(c); }) * r.inv;
      if (r.post.layer) t2 = sum_of_row(r.M, slots, e) * r.inv;
    }
    for (int c = threadIdx.x; c < r.M; c += kAnyThreads) {
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

// The sums of all workgroups: 16 columns by 16 lanes that take every 16th part, whose sums are added in their order.
struct Sums {
  const float* partial;
  int64_t groups;
  int parts, sums, M;
  const float *gate, *post_weight, *post_bias;
  float beta;
  float *dgate, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
};
__global__ __launch_bounds__(256) void columns_kernel(Sums s) {
  __shared__ float of_lanes[4][16][17];
  const int column = blockIdx.x * 16 + threadIdx.x % 16, lane = threadIdx.x / 16;
  const bool exists = column < s.M;
  float total[4] = {0, 0, 0, 0};  // of lane 0: dpost.weight, D, dpost.bias, E
  for (int64_t group = 0; group < s.groups; ++group) {
    float v[4] = {0, 0, 0, 0};
    if (exists) {
      const float* p = s.partial + group * s.parts * s.sums * s.M + column;
      for (int part = lane; part < s.parts; part += 16)
        for (int n = 0; n < s.sums; ++n) v[n] += p[(static_cast<int64_t>(part) * s.sums + n) * s.M];
    }
    for (int n = 0; n < s.sums; ++n) of_lanes[n][lane][threadIdx.x % 16] = v[n];
    lds_barrier();
    if (lane == 0 && exists) {
      for (int n = 0; n < s.sums; ++n) {
        v[n] = 0.0f;
        for (int l = 0; l < 16; ++l) v[n] += of_lanes[n][l][threadIdx.x];
      }
      const float by = s.beta * param(s.gate ? s.gate + group * s.M : nullptr, column, 1.0f);
      if (s.dgate)
        s.dgate[group * s.M + column] = s.beta * (param(s.post_weight, column, 1.0f) * v[0] + param(s.post_bias, column, 0.0f) * v[2]);
      total[0] = fmaf(by, v[0], total[0]);
      total[1] += v[1];
      total[2] = fmaf(by, v[2], total[2]);
      total[3] += v[3];
    }
    lds_barrier();
  }
  if (lane != 0 || !exists) return;
  if (s.dpost_weight) s.dpost_weight[column] = total[0];
  if (s.dpre_weight) s.dpre_weight[column] = total[1];
  if (s.dpost_bias) s.dpost_bias[column] = total[2];
  if (s.dpre_bias) s.dpre_bias[column] = total[3];
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
  if (pieces <= 128) return {1, 2};
  if (pieces <= 256) return {2, 2};
  if (pieces <= 512) return {4, 2};
  if (pieces <= 1024) return {8, 2};
  return {16, 2};
}
// Workgroups: rows that a gate is for are cut into parts.
struct Plan {
  Shape shape;
  int64_t groups, group_rows, part_rows, parts;
};
Plan plan_of(const ResidualCall& c, tempo_dtype dt) {
  Plan p{};
  p.shape = shape_of(c.M, dt);
  p.groups = c.gate ? c.groups : 1;
  p.group_rows = c.N / p.groups;
  const int64_t blocks = int64_t{compute_units()} * 16 / std::max(p.shape.waves, 1);
  p.part_rows = std::max<int64_t>((c.N + blocks - 1) / blocks, 1);
  p.parts = std::max<int64_t>((p.group_rows + p.part_rows - 1) / p.part_rows, 1);
  p.part_rows = std::max<int64_t>((p.group_rows + p.parts - 1) / p.parts, 1);
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
  r.N = c.N, r.M = static_cast<int>(c.M);
  r.group_rows = p.group_rows;
  r.inv = 1.0f / static_cast<float>(c.M);
  r.parts = static_cast<int>(p.parts);
  r.part_rows = p.part_rows;
  return r;
}
template <typename T, typename F>
bool with_shape(const Shape& s, int64_t M, F&& f) {
  auto by_row = [&](auto waves, auto pieces) {
    if (M % Store<T>::kVec == 0) f(waves, pieces, std::false_type{});
    else f(waves, pieces, std::true_type{});
    return true;
  };
  const std::integral_constant<int, 2> two;
  switch (s.waves) {
    case 1:
      return s.pieces == 1 ? by_row(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{})
                           : by_row(std::integral_constant<int, 1>{}, two);
    case 2: return by_row(two, two);
    case 4: return by_row(std::integral_constant<int, 4>{}, two);
    case 8: return by_row(std::integral_constant<int, 8>{}, two);
    case 16: return by_row(std::integral_constant<int, 16>{}, two);
    default: return false;
  }
}

}  // namespace

bool residual_norm_takes(const ResidualCall& c, tempo_dtype dt) {
  const Plan p = plan_of(c, dt);
  return p.groups * p.parts <= int64_t{1} << 22;  // launches of less than 2^32 lanes
}

size_t residual_norm_workspace_bytes(const ResidualCall& c, tempo_dtype dt) {
  const Plan p = plan_of(c, dt);
  return static_cast<size_t>(p.groups) * p.parts * 4 * c.M * sizeof(float);
}

tempo_status launch_residual_norm_fwd(const ResidualCall& c, tempo_dtype dt, hipStream_t st) {
  const Plan p = plan_of(c, dt);
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
  const Plan p = plan_of(c, dt);
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
  const Sums all{r.partial, p.groups, r.parts, sums, r.M, c.gate, c.post ? c.post->weight : nullptr, c.post ? c.post->bias : nullptr, c.beta,
                 c.dgate, c.dpost_weight, c.dpost_bias, c.dpre_weight, c.dpre_bias};
  hipLaunchKernelGGL(columns_kernel, dim3(static_cast<uint32_t>((c.M + 15) / 16)), dim3(256), 0, st, all);
  return launch_status();
}

}  // namespace tempo
