// Rotary positions of the attention heads of q and k:
//   theta = position f_i, i < R/2;   y1 = scale (x1 cos theta - x2 sin theta), y2 = scale (x2 cos theta + x1 sin theta)
// for the pairs (x1, x2) = (x[i], x[i + R/2]) or (x[2i], x[2i + 1]); elements from R on are copied.  The backward turns the
// other way: the transposed map.
//
// Bound by the bytes of q and k, read once and written once.  Angles are made where they are used: in 64 bits, which this
// chip multiplies at the rate of 32, so that a position of any size keeps its place within the turn; no table is read, kept or
// bounded by a longest sequence.
#include "launch_split.h"
#include "tempo_device.h"
#include "tempo_host.h"

namespace tempo {
namespace {

constexpr int kThreads = 256;
constexpr int kHeadsPerLane = 4;  // heads that share the angles of a lane

// cos and sin of a turn in 64 bits.  The quarter is taken off in 64 bits, what is left, at most an eighth of a turn, goes
// through the Taylor polynomials of sin and cos (next terms below 2e-9 and 2e-10).
__device__ __forceinline__ void cos_sin(double turns, float scale, float* c, float* s) {
  const double part = turns - rint(turns);
  const double quarters = part * 4.0;
  const double q = rint(quarters);
  const float a = static_cast<float>((quarters - q) * 1.5707963267948966);
  const float z = a * a;
  float sn = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), 0.0f);
  sn = fmaf(a, sn, a);
  float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
  const int n = static_cast<int>(q);  // -2 .. 2
  const float c0 = n & 1 ? sn : cs, s0 = n & 1 ? cs : sn;
  *c = scale * ((n + 1) & 2 ? -c0 : c0);
  *s = scale * (n & 2 ? -s0 : s0);
}

struct Side {
  const void* x;
  void* y;
  int64_t x_batch, x_token, x_head, y_batch, y_token, y_head;  // elements
};
struct Rotary {
  Side q, k;
  int q_heads, heads;  // of q; of both
  const double* freqs;
  const void* positions;  // null: start, start + 1, ...
  bool wide;              // 64-bit positions
  int64_t pos_batch, pos_token, start;
  uint32_t seq, tokens;
  int R2, D;
  float scale;
  int rot_units, units;  // pieces of a head: rotated, and all
  int groups;            // lanes that share the heads of a piece
  int lanes;             // units * groups: lanes of a token
  int tokens_per_block;  // > 1: whole tokens
  uint32_t first;        // token of the first workgroup
};

// A lane owns one piece of a token's heads group, group + groups, ...: V pairs (half) or V / 2 (interleaved), or V elements
// behind the rotated ones; V elements are 16 bytes.  The last piece of each kind may have fewer.
template <typename T, bool HALF, bool BACK>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Rotary r) {
  constexpr int V = Store<T>::kVec, kPairs = HALF ? V : V / 2;
  uint32_t token, lane;
  if (r.tokens_per_block > 1) {
    const uint32_t in_block = threadIdx.x / static_cast<uint32_t>(r.lanes);
    if (in_block >= static_cast<uint32_t>(r.tokens_per_block)) return;
    token = r.first + blockIdx.x * r.tokens_per_block + in_block;
    lane = threadIdx.x - in_block * r.lanes;
  } else {
    token = r.first + blockIdx.x;
    lane = blockIdx.y * kThreads + threadIdx.x;
    if (lane >= static_cast<uint32_t>(r.lanes)) return;
  }
  if (token >= r.tokens) return;
  const uint32_t group = lane / static_cast<uint32_t>(r.units);
  const int unit = static_cast<int>(lane - group * r.units);
  const uint32_t b = token / r.seq, s = token - b * r.seq;
  const int64_t q_in = b * r.q.x_batch + s * r.q.x_token, q_to = b * r.q.y_batch + s * r.q.y_token;
  const int64_t k_in = b * r.k.x_batch + s * r.k.x_token, k_to = b * r.k.y_batch + s * r.k.y_token;
  const bool turns = unit < r.rot_units;
  const int first = (turns ? unit : unit - r.rot_units) * (turns ? kPairs : V);  // pair, or element behind the rotated ones
  const int count = min(turns ? kPairs : V, (turns ? r.R2 : r.D - 2 * r.R2) - first);
  const bool whole = count == (turns ? kPairs : V);
  const int at = turns ? (HALF ? first : 2 * first) : 2 * r.R2 + first, other = at + r.R2;  // elements; other: HALF only

  float c[kPairs], sn[kPairs];
  if (turns) {
    const int64_t p = b * r.pos_batch + s * r.pos_token;
    int64_t position = r.start;
    if (!r.positions) position += s;
    else if (r.wide) position += static_cast<const int64_t*>(r.positions)[p];
    else position += static_cast<const int32_t*>(r.positions)[p];
    const double pos = static_cast<double>(position);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const double f = r.freqs[first + min(i, count - 1)];
      cos_sin(pos * (f * 0.15915494309189535), r.scale, &c[i], &sn[i]);
      if (BACK) sn[i] = -sn[i];
    }
  }
  auto in = [&](int h) {
    return h < r.q_heads ? static_cast<const T*>(r.q.x) + q_in + h * r.q.x_head
                         : static_cast<const T*>(r.k.x) + k_in + (h - r.q_heads) * r.k.x_head;
  };
  auto out = [&](int h) {
    return h < r.q_heads ? static_cast<T*>(r.q.y) + q_to + h * r.q.y_head
                         : static_cast<T*>(r.k.y) + k_to + (h - r.q_heads) * r.k.y_head;
  };
  if (whole) {
    u32x4 w1[kHeadsPerLane], w2[kHeadsPerLane];
#pragma unroll
    for (int i = 0; i < kHeadsPerLane; ++i) {
      const int h = min(static_cast<int>(group) + i * r.groups, r.heads - 1);
      const T* x = in(h);
      w1[i] = ldg_stream_any(x + at);
      if (HALF && turns) w2[i] = ldg_stream_any(x + other);
    }
#pragma unroll
    for (int i = 0; i < kHeadsPerLane; ++i) {
      const int h = static_cast<int>(group) + i * r.groups;
      if (h >= r.heads) break;
      T* y = out(h);
      if (!turns) {
        stg_stream_any(y + at, w1[i]);
        continue;
      }
      float x1[V], x2[V], y1[V], y2[V];
      Store<T>::unpack(w1[i], x1);
      if constexpr (HALF) {
        Store<T>::unpack(w2[i], x2);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          y1[j] = fmaf(x1[j], c[j], -(x2[j] * sn[j]));
          y2[j] = fmaf(x2[j], c[j], x1[j] * sn[j]);
        }
        stg_stream_any(y + other, Store<T>::pack(y2));
      } else {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
          y1[j] = fmaf(x1[j], c[j / 2], -(x1[j + 1] * sn[j / 2]));
          y1[j + 1] = fmaf(x1[j + 1], c[j / 2], x1[j] * sn[j / 2]);
        }
      }
      stg_stream_any(y + at, Store<T>::pack(y1));
    }
    return;
  }
  for (int h = static_cast<int>(group); h < r.heads; h += r.groups) {
    const T* x = in(h);
    T* y = out(h);
    if (!turns) {
      for (int j = 0; j < count; ++j) y[at + j] = x[at + j];
      continue;
    }
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      if (j >= count) break;
      const int e1 = HALF ? at + j : at + 2 * j, e2 = HALF ? other + j : at + 2 * j + 1;
      const float a = Store<T>::load1(x + e1), d = Store<T>::load1(x + e2);
      Store<T>::store1(y + e1, fmaf(a, c[j], -(d * sn[j])));
      Store<T>::store1(y + e2, fmaf(d, c[j], a * sn[j]));
    }
  }
}

Side side(const tempo_rotary_heads* h) {
  if (!h) return Side{};
  return {h->x, h->y, h->x_batch, h->x_token, h->x_head, h->y_batch, h->y_token, h->y_head};
}

}  // namespace

tempo_status launch_rotary(const tempo_rotary_heads* q, const tempo_rotary_heads* k, const double* freqs,
                           const tempo_rotary_positions* at, int64_t B, int64_t S, int64_t D, int64_t R,
                           tempo_rotary_layout layout, float scale, bool back, tempo_dtype dt, hipStream_t st) {
  Rotary r{};
  r.q = side(q);
  r.k = side(k);
  r.q_heads = static_cast<int>(q->heads);
  r.heads = static_cast<int>(q->heads + (k ? k->heads : 0));
  r.freqs = freqs;
  r.positions = at->positions;
  r.wide = at->bits == 64;
  r.pos_batch = at->batch_stride;
  r.pos_token = at->token_stride;
  r.start = at->start;
  r.seq = static_cast<uint32_t>(S);
  r.tokens = static_cast<uint32_t>(B * S);
  r.R2 = static_cast<int>(R / 2);
  r.D = static_cast<int>(D);
  r.scale = scale;
  const bool half = layout == TEMPO_ROTARY_HALF;
  const int V = dt == TEMPO_F32 ? 4 : 8, pairs = half ? V : V / 2;
  r.rot_units = (r.R2 + pairs - 1) / pairs;
  // Elements behind the rotated ones are there already where the call is in place.
  const bool in_place = q->x == q->y && (!k || k->x == k->y);
  r.units = r.rot_units + (in_place ? 0 : (r.D - 2 * r.R2 + V - 1) / V);
  r.groups = (r.heads + kHeadsPerLane - 1) / kHeadsPerLane;
  r.lanes = r.units * r.groups;
  r.tokens_per_block = r.lanes < kThreads ? kThreads / r.lanes : 1;
  if (r.tokens_per_block == 1 && r.lanes < kThreads) r.tokens_per_block = 1;
  const int64_t blocks = (int64_t{r.tokens} + r.tokens_per_block - 1) / r.tokens_per_block;
  const int per_token = (r.lanes + kThreads - 1) / kThreads;
  auto go = [&](auto kernel) {
    const bool ok = split_launch(blocks, most_groups(blocks, kThreads * per_token), [&](uint32_t from, uint32_t count) {
      r.first = from * r.tokens_per_block;
      hipLaunchKernelGGL(kernel, dim3(count, per_token), dim3(kThreads), 0, st, r);
      return launch_status() == TEMPO_OK;
    });
    return ok ? TEMPO_OK : TEMPO_ERR_LAUNCH;
  };
  auto by_way = [&](auto f32, auto f32_back, auto bf16, auto bf16_back) {
    if (dt == TEMPO_F32) return back ? go(f32_back) : go(f32);
    return back ? go(bf16_back) : go(bf16);
  };
  if (half)
    return by_way(rotary_kernel<float, true, false>, rotary_kernel<float, true, true>, rotary_kernel<bf16_t, true, false>,
                  rotary_kernel<bf16_t, true, true>);
  return by_way(rotary_kernel<float, false, false>, rotary_kernel<float, false, true>, rotary_kernel<bf16_t, false, false>,
                rotary_kernel<bf16_t, false, true>);
}

}  // namespace tempo
