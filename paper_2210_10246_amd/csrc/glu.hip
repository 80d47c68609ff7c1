// The gated feed-forward unit:   [g | u] = x W^T + b,   h = act(g) u     (W [2F, H]: the rows of the gate, then those of u)
// and its backward from what is kept, [g | u]:   dg = dh u act'(g),  du = dh act(g),  h = act(g) u once more,
//   dx = [dg | du] W,   dW = [dg | du]^T x,   db = column sums of [dg | du].
//
// All products are on the matrix cores with bfloat16 operands and float32 sums.  A float32 operand is taken apart into three
// bfloat16 ones, x = x0 + x1 + x2 exactly, and of the nine products those six are made that count in float32 (the other three
// are below 2^-21 of |a| |b|).
#include <algorithm>

#include "gelu_f32.h"
#include "launch_split.h"
#include "tempo_host.h"

namespace tempo {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// ---- activations ------------------------------------------------------------------------------------------------------
struct ActGrad {
  float value, grad;
};
// act(g) and act'(g).  Beside a factor that has long been zero the other one is kept finite.
template <int KIND>
__device__ __forceinline__ ActGrad act_grad(float x) {
  const float xc = fminf(fmaxf(x, -128.0f), 128.0f);
  if constexpr (KIND == TEMPO_GLU_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x));
    return {x * s, s * fmaf(xc, 1.0f - s, 1.0f)};
  } else if constexpr (KIND == TEMPO_GLU_GELU_TANH) {
    const float k = 0.7978845608028654f, ka = k * 0.044715f;
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-2.0f * 1.4426950408889634f * x * fmaf(x * x, ka, k)));
    return {x * s, fmaf(2.0f * xc * fmaf(xc * xc, 3.0f * ka, k), s * (1.0f - s), s)};
  } else {
    const float w = x * as_f32(TEMPO_GELU_ERFC_W_SCALE);
    const float density = 0.3989422804014327f * __builtin_amdgcn_exp2f(-(w * w));  // exp(-x^2 / 2) / sqrt(2 pi)
    const float phi = gelu_erf_phi(x);
    return {x * phi, fmaf(xc, density, phi)};
  }
}
// act(g) where no branch is wanted: SiLU and the tanh form of GELU are g sigmoid(g (c0 + c1 g^2)).
template <bool ERF>
__device__ __forceinline__ float act_value(float x, float c0, float c1) {
  if constexpr (ERF) return gelu_erf_value(x);
  return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * fmaf(c1 * x, x, c0)));  // -log2(e) is part of c0 and c1
}
template <typename F>
__device__ __forceinline__ void with_kind(int kind, F&& f) {  // uniform
  if (kind == TEMPO_GLU_SILU) f(std::integral_constant<int, TEMPO_GLU_SILU>{});
  else if (kind == TEMPO_GLU_GELU_ERF) f(std::integral_constant<int, TEMPO_GLU_GELU_ERF>{});
  else f(std::integral_constant<int, TEMPO_GLU_GELU_TANH>{});
}
__device__ __forceinline__ float act_of(int kind, float x) {
  float v;
  with_kind(kind, [&](auto k) { v = act_grad<decltype(k)::value>(x).value; });
  return v;
}

// ---- one operand of a product -----------------------------------------------------------------------------------------
// R rows by BK values of k: from memory to registers a step ahead, then to LDS.  KM: element (row, k) at p[k ld + row],
// else at p[row ld + k].  LDS holds 16-byte pieces, of a row's k or of a k's rows, in an order in which the lanes of a read
// meet different banks.
template <typename T, bool KM, int R, int BK, int THREADS>
struct Operand {
  static constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kRun = (KM ? R : BK) / 8;         // pieces side by side
  static constexpr int kPieces = R * BK / 8 / THREADS;   // of a lane
  static_assert(kPieces * 8 * THREADS == R * BK && kRun >= 4, "whole pieces per lane");
  static constexpr int kPlane = R * BK * 2;              // bytes
  static constexpr int kBytes = kPlanes * kPlane;
  static constexpr int kWords = sizeof(T) / 2;           // 16-byte words of a piece in memory

  const T* p[kPieces];
  int64_t step;
  u32x4 v[kPieces][kWords];

  // row_of: row of the tile -> row in memory, one that exists
  template <typename F>
  __device__ __forceinline__ Operand(const void* base, int64_t ld, int row0, int rows, F&& row_of) {
    step = KM ? BK * ld : BK;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = i * THREADS + static_cast<int>(threadIdx.x), line = at / kRun, piece = at % kRun;
      if constexpr (KM) p[i] = static_cast<const T*>(base) + line * ld + min(row0 + piece * 8, (rows - 1) & ~7);
      else p[i] = static_cast<const T*>(base) + row_of(line) * ld + piece * 8;
    }
  }
  __device__ __forceinline__ void load(int64_t s) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
#pragma unroll
      for (int j = 0; j < kWords; ++j)
        v[i][j] = *reinterpret_cast<const u32x4_any*>(p[i] + s * step + j * (8 / kWords));
    }
  }
  // A step that ends beyond K, or whose pieces of rows may end beyond the tensor: zeros for what does not exist.
  __device__ __forceinline__ void load_rest(int64_t s, int row0, int rows, int K) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = i * THREADS + static_cast<int>(threadIdx.x), line = at / kRun, piece = at % kRun;
      const int64_t k = s * BK + (KM ? line : piece * 8);
      const int64_t left = KM ? (k < K ? rows - min(row0 + piece * 8, (rows - 1) & ~7) : 0) : K - k;
      const T* q = p[i] + s * step;
#pragma unroll
      for (int j = 0; j < kWords; ++j) {
        constexpr int E = 8 / kWords;
        u32x4 w = {0, 0, 0, 0};
        if (left >= (j + 1) * E) {
          w = *reinterpret_cast<const u32x4_any*>(q + j * E);
        } else if (left > j * E) {
          uint32_t e[4] = {0, 0, 0, 0};
#pragma unroll
          for (int n = 0; n < E; ++n) {
            if (j * E + n < left) {
              if constexpr (E == 4) e[n] = reinterpret_cast<const uint32_t*>(q)[j * E + n];
              else e[n / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(q)[j * E + n]) << (16 * (n % 2));
            }
          }
          w = u32x4{e[0], e[1], e[2], e[3]};
        }
        v[i][j] = w;
      }
    }
  }
  __device__ static __forceinline__ int swizzled(int line, int piece) {
    // 64 banks are 16 pieces: 16 lanes that read a piece each of 16 rows, or 32 that read 8 bytes each of 4 rows of k.
    if constexpr (KM) return piece ^ (kRun >= 16 ? 4 * (line & 3) : 4 * (line / 2 & 1));
    else return piece ^ (line / (16 / kRun) & (kRun - 1));
  }
  __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = i * THREADS + static_cast<int>(threadIdx.x), line = at / kRun, piece = at % kRun;
      char* to = lds + (line * kRun + swizzled(line, piece)) * 16;
      if constexpr (kPlanes == 1) {
        *reinterpret_cast<u32x4*>(to) = v[i][0];
      } else {
        u32x4 w[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t part[3][2];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const uint32_t x = v[i][j / 2][2 * (j % 2) + n];
            const float r1 = as_f32(x) - as_f32(x & 0xFFFF0000u);
            const float r2 = r1 - as_f32(as_u32(r1) & 0xFFFF0000u);
            part[0][n] = x;
            part[1][n] = as_u32(r1);
            part[2][n] = as_u32(r2);
          }
#pragma unroll
          for (int q = 0; q < 3; ++q) w[q][j] = __builtin_amdgcn_perm(part[q][1], part[q][0], 0x07060302u);
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x4*>(to + q * kPlane) = w[q];
      }
    }
  }
  // What a lane gives to a matrix instruction: values k + 8 half .. + 7 of row `row` + lane % 32, half = lane / 32.
  __device__ static __forceinline__ bf16x8 read(const char* lds, int row, int k) {
    const int lane = threadIdx.x % kWave, half = lane / 32;
    if constexpr (!KM) {
      const int line = row + lane % 32;
      return *reinterpret_cast<const bf16x8*>(lds + (line * kRun + swizzled(line, k / 8 + half)) * 16);
    } else {
      // 16 lanes read 4 values of k of 16 rows, 4 rows each, and get 4 values of k of a row each
      const int j = lane % 16, r = row + lane % 32 / 16 * 16 + j % 4 * 4, line = k + 8 * half + j / 4;
      const char* at = lds + (line * kRun + swizzled(line, r / 8)) * 16 + r % 8 * 2;
      const char* next = lds + ((line + 4) * kRun + swizzled(line + 4, r / 8)) * 16 + r % 8 * 2;
      union {
        s16x4 h[2];
        bf16x8 all;
      } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)next);
      return u.all;
    }
  }
};

// ---- products ---------------------------------------------------------------------------------------------------------
// c[m][n] = sum_k a(m, k) b(n, k); GATED: the pairs of columns f and F + f of such a c are g and u.
struct Product {
  const void *a, *b;
  int64_t lda, ldb;
  int M, N, K;        // N: F if GATED
  void* c;            // [M, N]
  float* partial;     // splits > 1: [splits, M, N] ([splits, M, 2F]) sums of k's parts
  int splits, steps;  // steps of BK values of k in a part
  const void* bias;   // GATED: [2F] or null
  void* gu;           // GATED: [M, 2F] or null
  void* h;            // GATED: [M, F]
  int kind;
  float c0, c1;       // of act_value()
};
enum Epilogue { kPlain, kSigmoid, kErf };  // kPlain: not GATED

// The order of a part's instructions: in N groups, each with its share of the matrix instructions and of what else there is.
template <int MFMA, int READS, int WRITES, int LOADS, int N, int I = 0>
__device__ __forceinline__ void groups() {
  if constexpr (I < N) {
    constexpr int m = MFMA * (I + 1) / N - MFMA * I / N, r = READS * (I + 1) / N - READS * I / N,
                  w = WRITES * (I + 1) / N - WRITES * I / N, l = LOADS * (I + 1) / N - LOADS * I / N;
    if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
    if constexpr (w > 0) __builtin_amdgcn_sched_group_barrier(0x200, w, 0);
    if constexpr (l > 0) __builtin_amdgcn_sched_group_barrier(0x020, l, 0);
    if constexpr (m > 0) __builtin_amdgcn_sched_group_barrier(0x008, m, 0);
    groups<MFMA, READS, WRITES, LOADS, N, I + 1>();
  }
}
// The reads, which the next part begins with, in the first half: they are on their way for the second half's matrix instructions.
template <int MFMA, int READS, int WRITES, int LOADS>
__device__ __forceinline__ void spread() {
  constexpr int kFirst = (MFMA + 1) / 2, kSecond = MFMA - kFirst;
  groups<kFirst, READS, 0, 0, kFirst>();
  groups<kSecond, 0, WRITES, LOADS, kSecond>();
}

template <int BM_, int BN_, int WM_, int WN_, int BK_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_;
  static constexpr int kWavesN = BN / WN, kThreads = kWave * (BM / WM) * kWavesN;
};

// 32 rows by J x 32 columns of a wave's sums to memory, through LDS of its own, so that lanes side by side store pieces side
// by side: 4 elements of a lane, in 32 rows at once, took [16384, 4096] x 2 x 11008 2877 us where this takes XXX.
// value(j, q): registers 4q .. 4q + 3 of part j, elements (m = lane % 32, n = 32 j + 8 q + 4 (lane / 32) ..) of the block;
// rows, cols: how many exist.
template <typename U, int J, typename F>
__device__ __forceinline__ void store_rows(char* lds, U* out, int64_t ld, int rows, int cols, F&& value) {
  constexpr int kRow = J * 32 * sizeof(U), kPitch = kRow + 16, E = 16 / sizeof(U), kLanes = kRow / 16, kOnce = kWave / kLanes;
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int j = 0; j < J; ++j) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      char* to = lds + lane % 32 * kPitch + (j * 32 + 8 * q + 4 * (lane / 32)) * sizeof(U);
      const f32x4 v = value(j, q);
      if constexpr (sizeof(U) == 4) *reinterpret_cast<f32x4*>(to) = v;
      else *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
  }
  wave_lds_fence();
  const int col = lane % kLanes * E, left = cols - col;
#pragma unroll
  for (int i = 0; i < 32; i += kOnce) {
    const int row = i + lane / kLanes;
    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + row * kPitch + col * sizeof(U));
    if (row >= rows || left <= 0) continue;
    U* to = out + row * ld + col;
    if (left >= E) {
      *reinterpret_cast<u32x4_any*>(to) = w;
    } else {
      float v[E];
      Store<U>::unpack(w, v);
#pragma unroll
      for (int e = 0; e < E - 1; ++e)
        if (e < left) Store<U>::store1(to + e, v[e]);
    }
  }
  wave_lds_fence();
}

template <typename T, bool AKM, bool BKM, Epilogue END, typename C>
__global__ __launch_bounds__(C::kThreads) void product_kernel(Product g) {
  constexpr bool GATED = END != kPlain;
  constexpr int BM = C::BM, BN = C::BN, BK = C::BK, WM = C::WM, WN = C::WN, FM = WM / 32, FN = WN / 32;
  static_assert(!GATED || (FN % 2 == 0 && !AKM && !BKM), "a wave has g and u of an element");
  using A = Operand<T, AKM, BM, BK, C::kThreads>;
  using B = Operand<T, BKM, BN, BK, C::kThreads>;
  constexpr int kPlanes = A::kPlanes, kBuffer = A::kBytes + B::kBytes;
  // Two objects, so that writes to one are known not to be what is read from the other.
  __shared__ __attribute__((aligned(16))) char even[kBuffer], odd[kBuffer];

  // Neighbouring workgroups go to different XCDs, each with an L2 of its own: every XCD takes a run of tiles, and these go
  // down 8 rows of tiles before the next column.
  constexpr int kCols = GATED ? BN / 2 : BN;
  const int tiles_m = (g.M + BM - 1) / BM, tiles_n = (g.N + kCols - 1) / kCols;
  const int total = gridDim.x, xcd = blockIdx.x % 8, each = total / 8, more = total % 8;
  const int tile = xcd * each + min(xcd, more) + static_cast<int>(blockIdx.x) / 8;
  const int split = tile / (tiles_m * tiles_n), in_split = tile - split * (tiles_m * tiles_n);
  const int band = in_split / (8 * tiles_n), in_band = in_split - band * (8 * tiles_n), rows = min(8, tiles_m - band * 8);
  const int m0 = (band * 8 + in_band % rows) * BM, n0 = in_band / rows * kCols;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int wm = wave / C::kWavesN * WM, wn = wave % C::kWavesN * WN;

  A a(g.a, g.lda, m0, g.M, [&](int r) { return min(m0 + r, g.M - 1); });
  B b(g.b, g.ldb, n0, g.N, [&](int r) -> int64_t {
    if constexpr (!GATED) return min(n0 + r, g.N - 1);
    const int f = min(n0 + r / WN * (WN / 2) + r % (WN / 2), g.N - 1);
    return r % WN < WN / 2 ? f : int64_t{g.N} + f;
  });
  // Steps of BK values of k that are loaded in whole pieces: where rows of a k-major operand are no multiple of a piece,
  // their last one ends in the next row, so that the last row takes no part.
  const bool over = (AKM && g.M % 8 != 0) || (BKM && g.N % 8 != 0);
  const int whole = (over ? g.K - 1 : g.K) / BK;
  const int first = split * g.steps, end = first + g.steps, last = min(end, whole);

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  constexpr int kParts = BK / 16;  // of a step, between which operands are read from LDS
  static_assert(kParts % 2 == 0, "parities below");
  bf16x8 fa[2][kPlanes][FM], fb[2][kPlanes][FN];
  auto put = [&](char* lds) {
    a.store(lds);
    b.store(lds + A::kBytes);
  };
  auto get = [&](int to, const char* la, int part) {
    const char* lb = la + A::kBytes;
#pragma unroll
    for (int q = 0; q < kPlanes; ++q) {
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[to][q][i] = A::read(la + q * A::kPlane, wm + i * 32, part * 16);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[to][q][j] = B::read(lb + q * B::kPlane, wn + j * 32, part * 16);
    }
  };
  auto multiply = [&](int from) {
    auto planes = [&](int qa, int qb) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[from][qb][j], fa[from][qa][i], acc[i][j], 0, 0, 0);
    };
    if constexpr (kPlanes == 3) {  // the small ones first
      planes(0, 2);
      planes(2, 0);
      planes(1, 1);
      planes(0, 1);
      planes(1, 0);
    }
    planes(0, 0);
  };
  if (whole * BK < g.K && end > whole && first <= whole) {  // the rest, in steps of its own
    for (int s = whole; s < end && s * int64_t{BK} < g.K; ++s) {
      a.load_rest(s, m0, g.M, g.K);
      b.load_rest(s, n0, g.N, g.K);
      put(even);
      lds_barrier();
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
        get(0, even, part);
        multiply(0);
      }
      lds_barrier();
    }
  }
  // While the matrix cores work on a part, the operands of the next one come from LDS; step s + 1 is written there in the
  // first part of s, and s + 2 is on its way from memory.  The one barrier of a step stands before its last part, whose
  // operands all waves have read by then.  No branch in here: beyond the last step that one is fetched again.
  if (first < last) {
    auto fetch = [&](int s) {
      s = min(s, last - 1);
      a.load(s);
      b.load(s);
    };
    fetch(first);
    put(even);
    fetch(first + 1);
    lds_barrier();
    get(0, even, 0);
    constexpr int kPutB = kParts > 2 ? 1 : 0, kLoadB = kParts > 2 ? 2 : 1;
    auto step = [&](int s, const char* from, char* to) {
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
        if (part == kParts - 1) {
          lds_barrier();
          get(0, to, 0);
        } else {
          get((part + 1) & 1, from, part + 1);
        }
        if (part == 0) a.store(to);
        if (part == kPutB) b.store(to + A::kBytes);
        if (part == kPutB) a.load(min(s + 2, last - 1));
        if (part == kLoadB) b.load(min(s + 2, last - 1));
        multiply(part & 1);
        constexpr int kMfma = FM * FN * (kPlanes == 3 ? 6 : 1), kReads = kPlanes * (FM * (AKM ? 2 : 1) + FN * (BKM ? 2 : 1));
        if (part == 0) spread<kMfma, kReads, kPlanes * A::kPieces, 0>();
        else if (part == 1) spread<kMfma, kReads, kPlanes * B::kPieces, A::kWords * A::kPieces>();
        else if (part == 2) spread<kMfma, kReads, 0, B::kWords * B::kPieces>();
        else spread<kMfma, kReads, 0, 0>();
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    for (int s = first; s < last; s += 2) {
      step(s, even, odd);
      if (s + 1 == last) break;
      step(s + 1, odd, even);
    }
  }

  // The bias of the tile's gates, then of the rest, behind the waves' rooms.
  constexpr int kWaves = C::kThreads / kWave, kRoom = 32 * (WN * 4 + 16);
  static_assert(kWaves % 2 == 0 && kWaves / 2 * kRoom + (GATED ? BN * 4 : 0) <= kBuffer, "a wave's rows");
  char* const room = (wave < kWaves / 2 ? even : odd) + wave % (kWaves / 2) * kRoom;
  float* const bias = reinterpret_cast<float*>(odd + kBuffer) - BN;
  lds_barrier();
  if constexpr (GATED) {
    for (int i = threadIdx.x; i < BN; i += C::kThreads) {
      const int f = min(n0 + i % (BN / 2), g.N - 1) + i / (BN / 2) * g.N;
      bias[i] = g.bias && g.splits == 1 ? Store<T>::load1(static_cast<const T*>(g.bias) + f) : 0.0f;
    }
    lds_barrier();
  }
  auto part = [&](const f32x16& v, int q) { return f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]}; };
  const int m_first = m0 + wm;
  if constexpr (!GATED) {
    const int n = n0 + wn;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = m_first + i * 32;
      auto value = [&](int j, int q) { return part(acc[i][j], q); };
      if (g.splits > 1)
        store_rows<float, FN>(room, g.partial + (static_cast<int64_t>(split) * g.M + m) * g.N + n, g.N, g.M - m, g.N - n, value);
      else
        store_rows<T, FN>(room, static_cast<T*>(g.c) + static_cast<int64_t>(m) * g.N + n, g.N, g.M - m, g.N - n, value);
    }
  } else {
    constexpr int J = FN / 2;
    const int f = n0 + wn / 2, left = g.N - f;
    const int64_t ld = 2 * static_cast<int64_t>(g.N);
    const float* const own = bias + wn / 2 + 4 * (lane / 32);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = m_first + i * 32;
      auto gate = [&](int j, int q) { return part(acc[i][j], q) + *reinterpret_cast<const f32x4*>(own + j * 32 + 8 * q); };
      auto up = [&](int j, int q) { return part(acc[i][j + J], q) + *reinterpret_cast<const f32x4*>(own + BN / 2 + j * 32 + 8 * q); };
      auto sums = [&](auto* to) {
        using U = std::remove_pointer_t<decltype(to)>;
        store_rows<U, J>(room, to + m * ld + f, ld, g.M - m, left, gate);
        store_rows<U, J>(room, to + m * ld + f + g.N, ld, g.M - m, left, up);
      };
      if (g.splits > 1) {
        sums(g.partial + static_cast<int64_t>(split) * g.M * ld);
      } else {
        if (g.gu) sums(static_cast<T*>(g.gu));
        store_rows<T, J>(room, static_cast<T*>(g.h) + static_cast<int64_t>(m) * g.N + f, g.N, g.M - m, left, [&](int j, int q) {
          f32x4 v = gate(j, q);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = act_value<END == kErf>(v[e], g.c0, g.c1);
          return v * up(j, q);
        });
      }
    }
  }
}

// The sums of the parts, in their order.
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void join_kernel(Product g) {
  const int64_t n = static_cast<int64_t>(g.M) * g.N, e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (e >= n) return;
  if constexpr (!GATED) {
    float v = 0.0f;
    for (int s = 0; s < g.splits; ++s) v += g.partial[s * n + e];
    Store<T>::store1(static_cast<T*>(g.c) + e, v);
  } else {
    const int64_t at = e / g.N * 2 * g.N + e % g.N;
    float v = 0.0f, u = 0.0f;
    for (int s = 0; s < g.splits; ++s) {
      v += g.partial[s * 2 * n + at];
      u += g.partial[s * 2 * n + at + g.N];
    }
    if (g.bias) {
      const T* bias = static_cast<const T*>(g.bias) + e % g.N;
      v += Store<T>::load1(bias);
      u += Store<T>::load1(bias + g.N);
    }
    if (g.gu) {
      Store<T>::store1(static_cast<T*>(g.gu) + at, v);
      Store<T>::store1(static_cast<T*>(g.gu) + at + g.N, u);
    }
    Store<T>::store1(static_cast<T*>(g.h) + e, act_of(g.kind, v) * u);
  }
}

// ---- the backward's elementwise part ----------------------------------------------------------------------------------
struct Gates {
  const void *dh, *gu;
  void *dgu, *h;     // h may be null
  float* sums;       // null, or [chunks, 2F]: column sums of a chunk's rows
  int64_t rows;
  int F, kind, chunk;  // chunk: rows of a workgroup
};
// A wave takes 64 pieces of 16 bytes of the columns, of `chunk` rows one after the other.
template <typename T, int KIND>
__global__ __launch_bounds__(kWave) void gates_kernel(Gates g, int64_t chunk0) {
  constexpr int V = Store<T>::kVec;
  const int f = (blockIdx.x * kWave + threadIdx.x) * V, left = g.F - f;
  if (left <= 0) return;
  const int64_t c = chunk0 + blockIdx.y, r0 = c * g.chunk, r1 = r0 + g.chunk < g.rows ? r0 + g.chunk : g.rows;
  float sg[V], su[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sg[i] = su[i] = 0.0f;
  for (int64_t r = r0; r < r1; ++r) {
    const T* dh = static_cast<const T*>(g.dh) + r * g.F + f;
    const T* gu = static_cast<const T*>(g.gu) + r * 2 * g.F + f;
    T* dgu = static_cast<T*>(g.dgu) + r * 2 * g.F + f;
    T* h = g.h ? static_cast<T*>(g.h) + r * g.F + f : nullptr;
    float d[V], x[V], u[V];
    if (left >= V) {
      Store<T>::unpack(ldg_stream_any(dh), d);
      Store<T>::unpack(*reinterpret_cast<const u32x4_any*>(gu), x);
      Store<T>::unpack(*reinterpret_cast<const u32x4_any*>(gu + g.F), u);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        d[i] = i < left ? Store<T>::load1(dh + i) : 0.0f;
        x[i] = i < left ? Store<T>::load1(gu + i) : 0.0f;
        u[i] = i < left ? Store<T>::load1(gu + g.F + i) : 0.0f;
      }
    }
    float dg[V], du[V], y[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const ActGrad a = act_grad<KIND>(x[i]);
      y[i] = a.value * u[i];
      dg[i] = d[i] * u[i] * a.grad;
      du[i] = d[i] * a.value;
      sg[i] += dg[i];
      su[i] += du[i];
    }
    if (left >= V) {
      *reinterpret_cast<u32x4_any*>(dgu) = Store<T>::pack(dg);
      *reinterpret_cast<u32x4_any*>(dgu + g.F) = Store<T>::pack(du);
      if (h) stg_stream_any(h, Store<T>::pack(y));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (i >= left) break;
        Store<T>::store1(dgu + i, dg[i]);
        Store<T>::store1(dgu + g.F + i, du[i]);
        if (h) Store<T>::store1(h + i, y[i]);
      }
    }
  }
  if (g.sums) {
    float* to = g.sums + c * 2 * g.F + f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i >= left) break;
      to[i] = sg[i];
      to[g.F + i] = su[i];
    }
  }
}
template <typename T>
__global__ __launch_bounds__(kWave) void bias_kernel(const float* sums, T* dbias, int64_t chunks, int n) {
  const int e = blockIdx.x * kWave + threadIdx.x;
  if (e >= n) return;
  float v = 0.0f;
  for (int64_t c = 0; c < chunks; ++c) v += sums[c * n + e];
  Store<T>::store1(dbias + e, v);
}

// ---- plans ------------------------------------------------------------------------------------------------------------
enum class Size { kLarge, kMiddle, kSmall };
template <typename T>
struct Tiles;
template <>
struct Tiles<bf16_t> {
  using Large = Tile<256, 256, 128, 128, 64>;
  using Middle = Tile<128, 128, 64, 64, 64>;
  using Small = Tile<64, 64, 32, 64, 64>;
};
template <>
struct Tiles<float> {
  using Large = Tile<128, 128, 64, 64, 32>;
  using Middle = Tile<128, 128, 64, 64, 32>;
  using Small = Tile<64, 64, 32, 64, 32>;
};

struct Plan {
  Size size;
  int splits, steps;
  int64_t tiles;
};
Plan plan_for(int64_t M, int64_t N, int64_t K, tempo_dtype dt) {  // N: columns of all rows of b
  const int64_t cus = compute_units();
  auto count = [&](int bm, int bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  const int bk = dt == TEMPO_F32 ? 32 : 64;
  Plan p{};
  int64_t tiles;
  if (dt == TEMPO_BF16 && count(256, 256) >= cus) p.size = Size::kLarge, tiles = count(256, 256);
  else if (count(128, 128) >= cus) p.size = Size::kMiddle, tiles = count(128, 128);
  else p.size = Size::kSmall, tiles = count(64, 64);
  const int64_t steps = std::max<int64_t>(1, (K + bk - 1) / bk);
  int64_t splits = tiles >= cus || tiles == 0 ? 1 : std::max<int64_t>(1, std::min(2 * cus / tiles, steps / 4));
  p.steps = static_cast<int>((steps + splits - 1) / splits);
  p.splits = static_cast<int>((steps + p.steps - 1) / p.steps);
  p.tiles = tiles * p.splits;
  return p;
}
size_t partial_bytes(const Plan& p, int64_t M, int64_t N) {
  return p.splits > 1 ? static_cast<size_t>(p.splits) * M * N * sizeof(float) : 0;
}

template <typename T, bool AKM, bool BKM, Epilogue END>
tempo_status launch_product(Product g, const Plan& p, hipStream_t st) {
  g.splits = p.splits;
  g.steps = p.steps;
  auto go = [&](auto tile) {
    using C = decltype(tile);
    hipLaunchKernelGGL((product_kernel<T, AKM, BKM, END, C>), dim3(static_cast<unsigned>(p.tiles)), dim3(C::kThreads), 0, st, g);
    return launch_status();
  };
  if (p.tiles == 0) return TEMPO_OK;
  tempo_status status;
  if (p.size == Size::kLarge) status = go(typename Tiles<T>::Large{});
  else if (p.size == Size::kMiddle) status = go(typename Tiles<T>::Middle{});
  else status = go(typename Tiles<T>::Small{});
  if (status != TEMPO_OK || p.splits == 1) return status;
  const int64_t n = int64_t{g.M} * g.N;
  hipLaunchKernelGGL((join_kernel<T, END != kPlain>), dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, st, g);
  return launch_status();
}

constexpr int kChunk = 32;  // rows whose column sums a wave makes
int64_t chunks_of(int64_t T) { return (T + kChunk - 1) / kChunk; }

template <typename T>
tempo_status forward(const GluCall& c, const Plan& p, hipStream_t st) {
  Product g{};
  g.a = c.x;
  g.b = c.w;
  g.lda = g.ldb = c.H;
  g.M = static_cast<int>(c.T);
  g.N = static_cast<int>(c.F);
  g.K = static_cast<int>(c.H);
  g.partial = static_cast<float*>(c.workspace);
  g.bias = c.bias;
  g.gu = c.gu;
  g.h = c.h;
  g.kind = c.kind;
  constexpr float log2e = 1.4426950408889634f, k = 0.7978845608028654f;
  if (c.kind == TEMPO_GLU_GELU_ERF) return launch_product<T, false, false, kErf>(g, p, st);
  g.c0 = c.kind == TEMPO_GLU_SILU ? -log2e : -2.0f * log2e * k;
  g.c1 = c.kind == TEMPO_GLU_SILU ? 0.0f : -2.0f * log2e * k * 0.044715f;
  return launch_product<T, false, false, kSigmoid>(g, p, st);
}

template <typename T>
tempo_status backward(const GluCall& c, const Plan& px, const Plan& pw, hipStream_t st) {
  constexpr int V = Store<T>::kVec;
  Gates e{c.dh, c.gu, c.dgu, c.h, c.dbias ? static_cast<float*>(c.workspace) : nullptr, c.T, static_cast<int>(c.F), c.kind, kChunk};
  const int64_t chunks = chunks_of(c.T);
  const unsigned across = static_cast<unsigned>((c.F + V * kWave - 1) / (V * kWave));
  auto gates = [&](auto kernel) {
    return split_launch(chunks, std::min<int64_t>(65535, most_groups(chunks, kWave * across)), [&](uint32_t first, uint32_t n) {
      hipLaunchKernelGGL(kernel, dim3(across, n), dim3(kWave), 0, st, e, int64_t{first});
      return launch_status() == TEMPO_OK;
    });
  };
  if (chunks > 0 && across > 0 &&
      !(c.kind == TEMPO_GLU_SILU ? gates(gates_kernel<T, TEMPO_GLU_SILU>)
        : c.kind == TEMPO_GLU_GELU_ERF ? gates(gates_kernel<T, TEMPO_GLU_GELU_ERF>)
                                       : gates(gates_kernel<T, TEMPO_GLU_GELU_TANH>)))
    return TEMPO_ERR_LAUNCH;
  tempo_status status = TEMPO_OK;
  if (c.dbias && c.F > 0) {
    const int n = static_cast<int>(2 * c.F);
    hipLaunchKernelGGL((bias_kernel<T>), dim3((n + kWave - 1) / kWave), dim3(kWave), 0, st, e.sums, static_cast<T*>(c.dbias), chunks, n);
    status = launch_status();
  }
  Product g{};
  g.a = c.dgu;
  g.lda = 2 * c.F;
  g.ldb = c.H;
  g.N = static_cast<int>(c.H);
  g.partial = static_cast<float*>(c.workspace);
  if (status == TEMPO_OK && c.dx) {
    g.b = c.w;
    g.M = static_cast<int>(c.T);
    g.K = static_cast<int>(2 * c.F);
    g.c = c.dx;
    status = launch_product<T, false, true, kPlain>(g, px, st);
  }
  if (status == TEMPO_OK && c.dw) {
    g.b = c.x;
    g.M = static_cast<int>(2 * c.F);
    g.K = static_cast<int>(c.T);
    g.c = c.dw;
    status = launch_product<T, true, true, kPlain>(g, pw, st);
  }
  return status;
}

}  // namespace

bool glu_takes(int64_t T, int64_t H, int64_t F) {
  const int64_t most = int64_t{1} << 30;  // of what is counted in 32 bits
  if (T > most || H > most || F > most / 2) return false;
  // tiles of 64 x 64 elements, up to 512 lanes a tile, in one launch
  auto tiles = [](int64_t M, int64_t N) { return ((M + 63) / 64) * ((N + 63) / 64); };
  return tiles(T, 2 * F) < most / 256 && tiles(T, H) < most / 256 && tiles(2 * F, H) < most / 256;
}

size_t glu_workspace_bytes(int64_t T, int64_t H, int64_t F, tempo_dtype dt, bool back) {
  if (!back) return partial_bytes(plan_for(T, 2 * F, H, dt), T, 2 * F);
  return std::max({partial_bytes(plan_for(T, H, 2 * F, dt), T, H), partial_bytes(plan_for(2 * F, H, T, dt), 2 * F, H),
                   static_cast<size_t>(chunks_of(T)) * 2 * F * sizeof(float)});
}

tempo_status launch_glu_fwd(const GluCall& c, tempo_dtype dt, hipStream_t st) {
  const Plan p = plan_for(c.T, 2 * c.F, c.H, dt);
  if (partial_bytes(p, c.T, 2 * c.F) > c.workspace_bytes) return TEMPO_ERR_WORKSPACE;
  return dt == TEMPO_F32 ? forward<float>(c, p, st) : forward<bf16_t>(c, p, st);
}

tempo_status launch_glu_bwd(const GluCall& c, tempo_dtype dt, hipStream_t st) {
  const Plan px = plan_for(c.T, c.H, 2 * c.F, dt), pw = plan_for(2 * c.F, c.H, c.T, dt);
  if ((c.dx && partial_bytes(px, c.T, c.H) > c.workspace_bytes) || (c.dw && partial_bytes(pw, 2 * c.F, c.H) > c.workspace_bytes) ||
      (c.dbias && static_cast<size_t>(chunks_of(c.T)) * 2 * c.F * sizeof(float) > c.workspace_bytes))
    return TEMPO_ERR_WORKSPACE;
  return dt == TEMPO_F32 ? backward<float>(c, px, pw, st) : backward<bf16_t>(c, px, pw, st);
}

}  // namespace tempo
