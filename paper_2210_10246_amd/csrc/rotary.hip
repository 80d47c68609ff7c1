// Rotary positions of the attention heads of q and k:
//   theta = position f_i, i < R/2;   y1 = scale (x1 cos theta - x2 sin theta), y2 = scale (x2 cos theta + x1 sin theta)
// for the pairs (x1, x2) = (x[i], x[i + R/2]) or (x[2i], x[2i + 1]); elements from R on are copied.  The backward turns the
// other way: the transposed map.
//
// Bound by the bytes of q and k, read once and written once.  Angles are made where they are used: in two numbers of 64 bits, which
// this chip multiplies at the rate of 32, so that a position of any size keeps its place within the turn; no table is read, kept or
// bounded by a longest sequence.
#include <algorithm>
#include <type_traits>

#include "launch_split.h"
#include "tempo_device.h"
#include "tempo_host.h"

namespace tempo {
namespace {

constexpr int kThreads = 256;
// Heads that share the angles of a lane, each in two pieces (half) or one: 128 bytes of a lane on their way.  One each where that leaves
// the chip short of waves and the angles, made for every head then, are few.
constexpr int heads_per_lane(bool half) { return half ? 4 : 8; }

// cos and sin of position f radians.  f / 2 pi and its product with the position are taken in two numbers of 64 bits, the second what
// the first one's rounding left out, so that less the whole turns they are good to 2^-50 at any position of 53 bits (in one number each
// the angle was off by 1.6e-4 at 2^40).  The quarter is taken off in 64 bits, what is left, at most an eighth of a turn, goes through
// the Taylor polynomials of sin and cos (next terms below 2e-9 and 2e-10).
__device__ __forceinline__ void cos_sin(double position, double f, float scale, float* c, float* s) {
#pragma clang fp contract(off)  // turns less its whole ones has to be that of the rounded product
  constexpr double inv = 0.15915494309189535, inv_rest = -9.839338337591243e-18;  // 1 / 2 pi
  const double t = f * inv, t_rest = fma(f, inv_rest, fma(f, inv, -t));
  const double turns = position * t, rest = fma(position, t_rest, fma(position, t, -turns));
  const double part = (turns - rint(turns)) + rest;
  const double quarters = part * 4.0;
  const double q = rint(quarters);
  const float a = static_cast<float>((quarters - q) * 1.5707963267948966);
  const float z = a * a;
  float sn = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), 0.0f);
  sn = fmaf(a, sn, a);
  float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
  const int n = static_cast<int>(q);  // its last two bits count
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
  uint32_t units_per_block, tokens_per_block;  // one of both is 1, or all units and several tokens
  uint32_t groups, per_tokens;                 // of heads; workgroups of the same tokens
  uint32_t first;                              // workgroup of the call that is the launch's first
  bool in_place;
};

// A lane owns one piece of HEADS heads of a token: V pairs (half) or V / 2 (interleaved), or V elements
// behind the rotated ones; V elements are 16 bytes.
// STREAM: what is written will not be in a cache when it is read.
template <typename T, bool HALF, bool BACK, int HEADS, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Rotary r) {
  constexpr int V = Store<T>::kVec, kPairs = HALF ? V : V / 2;
  // Workgroups of the same tokens follow one another; each takes heads side by side of tokens side by side, whichever of the
  // two is the nearer in memory.
  uint32_t block = blockIdx.x;
  if constexpr (STREAM) {  // a run of them on each XCD: 65536 tokens of 40 heads of 128 bfloat16 262 / 242 us
    const uint32_t each = gridDim.x / 8;
    if (block < each * 8) block = block % 8 * each + block / 8;
  }
  block += r.first;
  const uint32_t tokens = block / r.per_tokens, part = block - tokens * r.per_tokens;
  const uint32_t unit_block = part / r.groups, group = part - unit_block * r.groups;
  const uint32_t in_block = threadIdx.x / r.units_per_block, token = tokens * r.tokens_per_block + in_block;
  const int unit = static_cast<int>(unit_block * kThreads + threadIdx.x - in_block * r.units_per_block);
  if (in_block >= r.tokens_per_block || token >= r.tokens || unit >= r.units) return;
  const uint32_t b = token / r.seq, s = token - b * r.seq;
  const int64_t q_in = b * r.q.x_batch + s * r.q.x_token, q_to = b * r.q.y_batch + s * r.q.y_token;
  const int64_t k_in = b * r.k.x_batch + s * r.k.x_token, k_to = b * r.k.y_batch + s * r.k.y_token;
  const bool turns = unit < r.rot_units;
  // Of the pairs, or of the elements behind the rotated ones: the first of the piece, and how many it has.  Out of place a last
  // piece that is not whole ends where it does but begins earlier, and makes what the one before makes too; in place that could
  // have been written already.
  const int full = turns ? kPairs : V, all = turns ? r.R2 : r.D - 2 * r.R2, in_order = (turns ? unit : unit - r.rot_units) * full;
  const int first = r.in_place || all < full ? in_order : min(in_order, all - full), count = min(full, all - first);
  const int elements = turns && !HALF ? 2 * count : count;  // of a piece
  const int at = turns ? (HALF ? first : 2 * first) : 2 * r.R2 + first, other = at + r.R2;  // elements; other: HALF only
  auto in = [&](int h) {
    return h < r.q_heads ? static_cast<const T*>(r.q.x) + q_in + h * r.q.x_head
                         : static_cast<const T*>(r.k.x) + k_in + (h - r.q_heads) * r.k.x_head;
  };
  auto out = [&](int h) {
    return h < r.q_heads ? static_cast<T*>(r.q.y) + q_to + h * r.q.y_head
                         : static_cast<T*>(r.k.y) + k_to + (h - r.q_heads) * r.k.y_head;
  };
  auto load = [&](const T* p) {
    if (elements == V) return ldg_stream_any(p);
    float e[V];
#pragma unroll
    for (int j = 0; j < V; ++j) e[j] = j < elements ? Store<T>::load1(p + j) : 0.0f;
    return Store<T>::pack(e);
  };
  auto store = [&](T* p, u32x4 w) {
    if (elements == V) {
      if constexpr (STREAM) stg_stream_any(p, w);
      else *reinterpret_cast<u32x4_any*>(p) = w;
      return;
    }
    float e[V];
    Store<T>::unpack(w, e);
#pragma unroll
    for (int j = 0; j < V - 1; ++j)
      if (j < elements) Store<T>::store1(p + j, e[j]);
  };

  // All heads are on their way while the angles are made.
  u32x4 w1[HEADS], w2[HEADS];
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const T* x = in(min(static_cast<int>(group) * HEADS + i, r.heads - 1));
    w1[i] = load(x + at);
    if (HALF && turns) w2[i] = load(x + other);
  }
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
      cos_sin(pos, f, r.scale, &c[i], &sn[i]);
      if (BACK) sn[i] = -sn[i];
    }
  }
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int h = static_cast<int>(group) * HEADS + i;
    if (h >= r.heads) break;
    T* y = out(h);
    if (!turns) {
      store(y + at, w1[i]);
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
      store(y + other, Store<T>::pack(y2));
    } else {
#pragma unroll
      for (int j = 0; j < V; j += 2) {
        y1[j] = fmaf(x1[j], c[j / 2], -(x1[j + 1] * sn[j / 2]));
        y1[j + 1] = fmaf(x1[j + 1], c[j / 2], x1[j] * sn[j / 2]);
      }
    }
    store(y + at, Store<T>::pack(y1));
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
  r.in_place = q->x == q->y || (k && k->x == k->y);
  r.units = r.rot_units + (in_place ? 0 : (r.D - 2 * r.R2 + V - 1) / V);
  const int64_t pieces = int64_t{r.tokens} * r.units * r.heads;
  // us with one / several heads a lane, at 1, 2 and 4 Mi angles: half, float32, 40 heads of 128 5.9 / 7.9, 9.4 / 10.1 and 15.6 / 14.0,
  // bfloat16 5.6 / 6.1, 7.8 / 7.6 and 12.5 / 10.4; neighbours, float32 6.4 / 7.1, 10.5 / 9.7 and 17.5 / 13.6, bfloat16 (2, 4 and 8 Mi)
  // 7.6 / 7.5, 12.7 / 10.3 and 21.7 / 14.2; 12 heads of 83, 38 turned, neighbours, float32 (1 and 2 Mi) 7.2 / 8.1 and 11.8 / 10.6.
  const bool few = pieces * pairs < int64_t{compute_units()} * 8192;
  const int per_lane = few ? 1 : heads_per_lane(half);
  r.groups = (r.heads + per_lane - 1) / per_lane;
  r.units_per_block = std::min(r.units, kThreads);
  r.tokens_per_block = std::min(kThreads / r.units_per_block, r.tokens);
  r.per_tokens = r.groups * ((r.units + kThreads - 1) / kThreads);
  const int threads = (r.units_per_block * r.tokens_per_block + kWave - 1) / kWave * kWave;
  const int64_t blocks = (int64_t{r.tokens} + r.tokens_per_block - 1) / r.tokens_per_block * r.per_tokens;
  // What is written stays in the 256 MiB of cache where it is a part of that, and where lanes side by side do not write the whole of
  // each line at once.  us not streamed / streamed, 65536 tokens of 32 heads, bfloat16: halves, heads of 128 206 / 193, of 256 434 / 385,
  // of 128 in rows of 192 from 64 bytes on 292 / 260, of 128 in rows of 136 344 / 426, of 96 (halves of 96 bytes) 177 / 270, of 64 121 / 152,
  // half of a head of 128 turned 201 / 220; neighbours, heads of 128 221 / 192, in rows of 136 344 / 318, of 80 144 / 143, of 83 (95325
  // tokens of 12) 115 / 131.  4 x 2048 x 32 of 64 float32 (67 MB) 29.5 / 26.7.
  auto in_rows_of = [&](int64_t bytes, const Side& t, int64_t heads) {
    auto whole = [&](int64_t elements) { return elements * (16 / V) % bytes == 0; };
    return reinterpret_cast<uintptr_t>(t.y) % bytes == 0 && (B == 1 || whole(t.y_batch)) && (S == 1 || whole(t.y_token)) &&
           (heads == 1 || whole(t.y_head));
  };
  const int64_t row = half ? 64 : 16, run = half ? 128 : 16;
  const bool lines = (half ? r.R2 : R) * (16 / V) % run == 0 && in_rows_of(row, r.q, r.q_heads) &&
                     (!k || in_rows_of(row, r.k, k->heads));
  const bool stream = lines && pieces * (half ? 32 : 16) > (int64_t{48} << 20);
  auto go = [&](auto kernel) {
    const bool ok = split_launch(blocks, most_groups(blocks, threads), [&](uint32_t first, uint32_t count) {
      r.first = first;
      hipLaunchKernelGGL(kernel, dim3(count), dim3(threads), 0, st, r);
      return launch_status() == TEMPO_OK;
    });
    return ok ? TEMPO_OK : TEMPO_ERR_LAUNCH;
  };
  auto by_way = [&](auto type, auto halves) {
    using T = decltype(type);
    constexpr bool HALF = decltype(halves)::value;
    constexpr int HEADS = heads_per_lane(HALF);
    if (few) return back ? go(rotary_kernel<T, HALF, true, 1, false>) : go(rotary_kernel<T, HALF, false, 1, false>);
    if (stream) return back ? go(rotary_kernel<T, HALF, true, HEADS, true>) : go(rotary_kernel<T, HALF, false, HEADS, true>);
    return back ? go(rotary_kernel<T, HALF, true, HEADS, false>) : go(rotary_kernel<T, HALF, false, HEADS, false>);
  };
  if (half) return dt == TEMPO_F32 ? by_way(float{}, std::true_type{}) : by_way(bf16_t{}, std::true_type{});
  return dt == TEMPO_F32 ? by_way(float{}, std::false_type{}) : by_way(bf16_t{}, std::false_type{});
}

}  // namespace tempo
