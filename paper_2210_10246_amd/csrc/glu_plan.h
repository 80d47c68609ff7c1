// Host arithmetic of the gated unit's products: which tiles, in how many parts of k, and what of the workspace (no HIP in here).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "../../include/tempo.h"

namespace tempo {

// An operand that lies by k, rows of `n` elements, each a value of k's: pieces of 8 elements are loaded whole also where a row ends
// inside one.  The last piece of a row then ends in a later row, and that of the last rows would end behind the tensor: so many values
// of k, the last ones, are loaded element by element.  1 from 4 elements a row on, up to 7 of rows of one.
constexpr int ends_later(int n) { return n % 8 == 0 ? 0 : (8 - n % 8 + n - 1) / n; }
// Steps of `step` values of k that are loaded in whole pieces, of two operands that lie by k (n: elements of a row) or do not (n: 0).
constexpr int whole_steps(int k, int step, int a, int b) {
  const int of_a = a > 0 ? ends_later(a) : 0, of_b = b > 0 ? ends_later(b) : 0, left = k - (of_a > of_b ? of_a : of_b);
  return left > 0 ? left / step : 0;
}

// Tiles of 256, 128 or 64 rows and columns; the last three: forward only, of few rows.  Aligned: bfloat16 in rows of whole 16-byte pieces,
// else by way of registers.
enum class Size { kLarge, kMiddle, kSmall, kFewest, kFew, kFewWide };
inline int edge(Size s) { return s == Size::kLarge ? 256 : s == Size::kMiddle ? 128 : 64; }
// Few rows: their most, and the tiles' columns and values of k in a step.
constexpr int kFewestRows = 16, kFewRows = 64, kFewStep = 64;
constexpr int few_columns(Size s) { return s == Size::kFewWide ? 128 : 64; }
struct Plan {
  bool aligned;
  Size size;
  int splits, steps;
  int64_t tiles;
};
struct Shape {
  int64_t M, N, K;  // N: columns of all rows of b
  int64_t tiles(Size s) const { return ((M + edge(s) - 1) / edge(s)) * ((N + edge(s) - 1) / edge(s)); }
};
// What a tile takes, in us: `step` for 32 values of k and `tile` for its beginning and end, times the tiles of a compute unit,
// and `wait` more for every 32 values of k of the longest one, alone or not.  Measured, us of [T, H] x 2F with tiles of 256 /
// 128 / 64, bfloat16 in whole pieces: 16384 x 4096 x 11008 2390 / 3535 / 6490, 2048 x 1024 x 4096 41 / 49 / 71, 1024 x 1024 x 4096
// 35 / 26 / 39, 128 x 1024 x 4096 - / 11.0 / 6.5, 1000 x 128 x 8192 23.1 / 18.3 / 23.1; by way of registers, 128 / 64: 1021 x 1001 x
// 2729 36 / 48, 300 x 513 x 1031 15 / 8; float32 4096 x 2048 x 5504 936 / -, 1024 x 1024 x 4096 112 / 130, 512 x 512 x 1024 22 / 11.
struct Pace {
  double step, tile, wait;
  bool one;  // workgroup of a compute unit: tiles count in whole rounds
};
inline Pace pace(Size size, tempo_dtype dt, bool aligned) {
  if (dt == TEMPO_F32) return size == Size::kSmall ? Pace{0.4, 1.5, 0.2, false} : Pace{1.36, 6.0, 0.0, true};
  if (!aligned) return size == Size::kSmall ? Pace{0.17, 1.5, 0.12, false} : Pace{0.4, 5.0, 0.1, false};
  if (size == Size::kLarge) return {0.8, 12.0, 0.0, true};
  return size == Size::kMiddle ? Pace{0.225, 5.0, 0.1, false} : Pace{0.11, 1.0, 0.06, false};
}
// One plan for one or two products of a launch: the sizes of tiles, and in how many parts of k each is made where otherwise a
// few long tiles would be waited for ([32, 8192] x [8192, 1024] beside [8192, 32] x [32, 1024]: 92 us, 47 with 6 parts of the first).
inline double plan_for(const Shape* shapes, Plan* plans, int n, tempo_dtype dt, bool aligned, int cus) {
  aligned = aligned && dt == TEMPO_BF16;
  double least = 0.0;
  for (int way = 0; way < 6; ++way) {
    const Size size = way / 2 == 0 ? Size::kMiddle : way / 2 == 1 ? Size::kSmall : Size::kLarge;
    if (size == Size::kLarge && !aligned) break;
    const Pace at = pace(size, dt, aligned);
    const int bk = dt == TEMPO_F32 || (aligned && size != Size::kSmall) ? 32 : 64;
    Plan made[2];
    double tiles = 0.0, work = 0.0, longest = 0.0, join = 0.0;  // work, longest: in 32 values of k
    for (int i = 0; i < n; ++i) {
      tiles += shapes[i].tiles(size);
      work += shapes[i].tiles(size) * (shapes[i].K / 32.0);
    }
    const double share = std::max({work / cus, tiles / cus * at.tile / at.step, 8.0});
    tiles = 0.0;
    for (int i = 0; i < n; ++i) {
      const int64_t steps = std::max<int64_t>(1, (shapes[i].K + bk - 1) / bk);
      int64_t splits = way % 2 == 0 ? 1 : std::min<int64_t>(16, std::max<int64_t>(1, static_cast<int64_t>(shapes[i].K / 32.0 / share + 0.5)));
      Plan& p = made[i];
      p.aligned = aligned;
      p.size = size;
      p.steps = static_cast<int>((steps + splits - 1) / splits);
      p.splits = static_cast<int>((steps + p.steps - 1) / p.steps);
      p.tiles = shapes[i].tiles(size) * p.splits;
      tiles += p.tiles;
      longest = std::max(longest, p.steps * bk / 32.0);
      if (p.splits > 1) join += 3.0 + 8e-6 * p.splits * shapes[i].M * shapes[i].N / 4.0;  // a launch, and bytes at 4 TB/s
    }
    double here = std::max(work / cus, longest);
    if (at.one && tiles > cus) here = std::max(here, work / tiles * std::ceil(tiles / cus));
    const double cost = here * at.step + longest * at.wait + at.tile * std::max(1.0, at.one ? std::ceil(tiles / cus) : tiles / cus) + join;
    if (way == 0 || cost < least) {
      least = cost;
      for (int i = 0; i < n; ++i) plans[i] = made[i];
    }
  }
  return least;
}
// bfloat16 rows that do not all begin at multiples of 16 bytes: whether a copy with rows that do, of `bytes`, is worth what the
// products then save; plans is what is the cheaper.  us with copies / without: [8192, 1023] x 2 x 4095 forward 206 / 297, backward 383 /
// 494, [1021, 1001] x 2 x 2729 40 / 36 and 82 / 76, [513, 4095] x 2 x 11007 forward 237 / 178.
inline bool plan_padded(const Shape* shapes, Plan* plans, int n, double bytes, int cus) {
  Plan other[2];
  const double as_is = plan_for(shapes, plans, n, TEMPO_BF16, false, cus), padded = plan_for(shapes, other, n, TEMPO_BF16, true, cus);
  if (1.25 * (padded + 10.0 + bytes / 2.5e6) >= as_is) return false;
  for (int i = 0; i < n; ++i) plans[i] = other[i];
  return true;
}
inline int64_t whole_pieces(int64_t elements) { return (elements + 7) / 8 * 8; }
inline size_t partial_bytes(const Plan& p, const Shape& s) {
  return p.splits > 1 ? static_cast<size_t>(p.splits) * s.M * s.N * sizeof(float) : 0;
}
// Whether a forward of up to 64 rows is made on the tiles for few rows, in whose workgroups all of k follows on: that takes a time of
// its own however few columns W has, and the tiles above can be made in parts of k, which all compute units read.  us, those / these, on either
// side of where this changes over: 8 x 4096 x 2048 13.0 / 14.2, 1 x 4096 x 4096 20.1 / 15.4; 16 x 8192 x 2048 21.0 / 26.7, 4096 columns each 34.7
// / 32.6; 24 x 8192 x 2048 21 / 38, 24 x 4096 x 4096 20.4 / 22.3, 5504 columns each 29.0 / 24.7; 64 x 1024 x 512 6.8 / 7.2, 2048 columns
// each 8.7 / 8.4.  A step of 64 values of k is then not waited for where there are few: 64 x 512 x 2048 4.9 / 5.4, 64 x 768 x 2500 7.6 / 7.5.
inline bool few_pay(int64_t T, int64_t H, int64_t F) {
  const double steps = (H + kFewStep - 1) / kFewStep, here = 2.0 + (T <= kFewestRows ? 0.2 : 0.3) * steps;
  return (T <= kFewestRows || H > 512) && here < 5.0 + 4.0 * F * H / 4.5e6;  // W at 4.5 TB/s
}
// The three products.  Rows of x and w have H elements, of [g | u] 2F.  dx and dw are planned together whichever is wanted: the
// bits of one do not depend on the other.
struct ForwardPlan {
  Shape shape;
  Plan plan;
  bool padded = false;  // x and w copied to rows of H_pad elements
  int64_t H_pad;
  size_t x_at, bytes;   // of the copies in the workspace; all of it
  ForwardPlan(int64_t T, int64_t H, int64_t F, tempo_dtype dt, int cus) : shape{T, 2 * F, H} {
    H_pad = whole_pieces(H);
    const size_t copies = static_cast<size_t>(T + 2 * F) * H_pad * 2;
    if (dt == TEMPO_BF16 && H_pad != H) padded = plan_padded(&shape, &plan, 1, 2.0 * copies, cus);
    else plan_for(&shape, &plan, 1, dt, true, cus);
    // Up to 64 rows read W once, nothing else counts: whole lines of W's rows at a time, as much on its way as LDS holds, few rows
    // of x beside them.  us, 64 x 64 tiles of above / this: 64 x 4096 x 11008 46 / 43 (64 columns at a time 46), 24 x 8192 x 5504 60 / 45,
    // 16 x 4096 x 5504 29 / 20, 1 x 1024 x 4096 8.8 / 6.1, 1 x 1536 x 512 6.9 / 6.5.
    if (plan.aligned && !padded && T <= kFewRows && few_pay(T, H, F)) {
      // More columns at a time once 64 would make more workgroups than there are compute units: 24 x 1024 x 8192 (256 of 64 columns)
      // 8.9 us with 64, 10.3 with 128; 48 x 4096 x 9600 (300) 42.0 and 39.3, 64 x 1024 x 11008 13.8 and 12.5, 48 x 4096 x 20480 90 and 86.
      plan.size = T <= kFewestRows ? Size::kFewest : 2 * F > 64 * int64_t{cus} ? Size::kFewWide : Size::kFew;
      plan.splits = 1;
      plan.steps = static_cast<int>((H + kFewStep - 1) / kFewStep);
      plan.tiles = (2 * F + few_columns(plan.size) - 1) / few_columns(plan.size);
    }
    x_at = (partial_bytes(plan, shape) + 15) / 16 * 16;
    bytes = x_at + (padded ? copies : 0);
  }
};
struct BackwardPlan {
  Shape shapes[2];  // dx, dw
  Plan plans[2];
  bool padded = false;  // x and w copied to rows of H_pad elements if those are more than H, dgu to rows of F2_pad if more than 2F
  int64_t H_pad, F2_pad;
  size_t dx_bytes, dgu_at, x_at, bytes;
  BackwardPlan(int64_t T, int64_t H, int64_t F, tempo_dtype dt, int cus) : shapes{{T, H, 2 * F}, {2 * F, H, T}} {
    H_pad = whole_pieces(H);
    F2_pad = whole_pieces(2 * F);
    const size_t dgu_bytes = F2_pad != 2 * F ? static_cast<size_t>(T) * F2_pad * 2 : 0;
    const size_t copies = H_pad != H ? static_cast<size_t>(T + 2 * F) * H_pad * 2 : 0;
    if (dt == TEMPO_BF16 && dgu_bytes + copies > 0) padded = plan_padded(shapes, plans, 2, dgu_bytes + 2.0 * copies, cus);
    else plan_for(shapes, plans, 2, dt, true, cus);
    dx_bytes = (partial_bytes(plans[0], shapes[0]) + 15) / 16 * 16;
    dgu_at = (dx_bytes + partial_bytes(plans[1], shapes[1]) + 15) / 16 * 16;
    x_at = dgu_at + (padded ? dgu_bytes : 0);
    bytes = x_at + (padded ? copies : 0);
  }
};

}  // namespace tempo
