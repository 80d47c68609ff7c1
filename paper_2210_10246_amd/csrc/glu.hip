// The gated feed-forward unit:   [g | u] = x W^T + b,   h = act(g) u     (W [2F, H]: the rows of the gate, then those of u)
// and its backward from what is kept, [g | u]:   dg = dh u act'(g),  du = dh act(g),  h = act(g) u once more,
//   dx = [dg | du] W,   dW = [dg | du]^T x,   db = column sums of [dg | du].
//
// All products are on the matrix cores with bfloat16 operands and float32 sums.  A float32 operand is taken apart into three
// bfloat16 ones, x = x0 + x1 + x2 exactly (each takes the first 8 bits of what is left), and of the nine products those six are
// made that count in float32; the other three are below 2^-21 of |a| |b|.  Six products at the rate of bfloat16 are a sixth
// of its rate, half as fast again as the float32 matrix instructions: 1350 / 6 TFLOP/s and 154 for the library's, 8192^3.
//
// The products' bound is the power of the matrix cores (the clock falls from 2.4 to 1.7 GHz) and, beside it, what comes from the
// L2s; LDS is read without bank conflicts and takes a quarter of the time.  [16384, 4096] x 2 x 11008 bfloat16: forward 2.44 ms, 1210
// TFLOP/s with 1.1 GB written (2.30 ms without [g | u]; the library's plain product of that size 2.12), dx 2.17, dw 2.21 ms.
#include <algorithm>
#include <utility>

#include "gelu_f32.h"
#include "glu_plan.h"
#include "launch_split.h"
#include "tempo_host.h"

namespace tempo {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// ---- activations ------------------------------------------------------------------------------------------------------
struct ActGrad {
  float value, grad;
};
// act(g) and act'(g).  Beside a factor that has long been zero the other one is kept finite.  The argument of exp2 is rounded in 32 bits
// as g itself was: a sigmoid far on the left is off by up to |g| 2^-23 of itself (1e-5 at -80, where it is 2e-35), no more than by a last
// bit of g.
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
// act(g) where no branch is wanted: SiLU and the tanh form of GELU are g sigmoid(g (c0 + c1 g^2)).  g^2 is that of at most 128, where
// the sigmoid has long been 0 or 1: c1 is 0 for SiLU, and 0 times an infinite square would be NaN.
template <bool ERF>
__device__ __forceinline__ float act_value(float x, float c0, float c1) {
  if constexpr (ERF) return gelu_erf_value(x);
  const float xc = fminf(fmaxf(x, -128.0f), 128.0f);
  return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * fmaf(c1 * xc, xc, c0)));  // -log2(e) is part of c0 and c1
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

template <int... I, typename F>
__device__ __forceinline__ void for_each(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}

template <int... I, typename F>
__device__ __forceinline__ bool for_each_while(std::integer_sequence<int, I...>, F&& f) {
  return (f(std::integral_constant<int, I>{}) && ...);
}

// ---- one operand of a product -----------------------------------------------------------------------------------------
// R rows by BK values of k in LDS.  KM: element (row, k) at p[k ld + row], else at p[row ld + k].  LDS holds 16-byte pieces,
// of a row's k or of a k's rows, in an order in which the lanes of a read meet different banks.
template <typename T, bool KM, int R, int BK, int THREADS>
struct Operand {
  static constexpr bool kKMajor = KM;
  static constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kRun = (KM ? R : BK) / 8;         // pieces side by side
  static constexpr int kAll = R * BK / 8, kPieces = kAll < THREADS ? 1 : kAll / THREADS;  // of all lanes, and of a lane
  static_assert((kAll % THREADS == 0 || (THREADS % kAll == 0 && kAll % kWave == 0)) && (KM ? kRun >= 8 : kRun == 4 || kRun == 8),
                "whole pieces per lane");
  static constexpr int kPlane = R * BK * 2;              // bytes
  static constexpr int kBytes = kPlanes * kPlane;
  static constexpr int kWords = sizeof(T) / 2;           // 16-byte words of a piece in memory

  // 64 banks are 16 pieces.  Row by row, 16 lanes at a time read one each, in rows 0 - 3 and 12 - 15 the one and in 4 - 11 the
  // other of two neighbours, then the other way round; by k, 32 lanes read 8 bytes each of 4 rows and of 4 eight rows on.
  __device__ static __forceinline__ int swizzled(int line, int piece) {
    if constexpr (!KM && kRun == 4) return piece ^ (line / 4 & 1) * 2 ^ (line / 8 & 1) * 3;
    else if constexpr (!KM) return piece ^ (line / 2 & 7);
    else if constexpr (kRun >= 16) return piece ^ 2 * ((line & 3) + 4 * (line / 8 & 1));
    else return piece ^ 2 * ((line / 2 & 1) + 2 * (line / 8 & 1));
  }
  // What a lane gives to a matrix instruction: values k + 8 (lane / 16) .. + 7 of row `row` + lane % 16.
  __device__ static __forceinline__ bf16x8 read(const char* lds, int row, int k) {
    const int lane = threadIdx.x % kWave;
    if constexpr (!KM) {
      const int line = row + lane % 16;
      return *reinterpret_cast<const bf16x8*>(lds + (line * kRun + swizzled(line, k / 8 + lane / 16)) * 16);
    } else {
      // 16 lanes read 4 values of k of 16 rows, 4 rows each, and get 4 values of k of a row each
      const int j = lane % 16, r = row + j % 4 * 4, line = k + 8 * (lane / 16) + j / 4;
      const char* at = lds + (line * kRun + swizzled(line, r / 8)) * 16 + r % 8 * 2;
      union {
        s16x4 h[2];
        bf16x8 all;
      } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * kRun * 16));
      return u.all;
    }
  }

  // From memory: piece i of a lane is the one at this place of the LDS image; where there are fewer pieces than lanes, several
  // lanes do the same.
  __device__ static __forceinline__ int place(int i) { return (i * THREADS + static_cast<int>(threadIdx.x)) % kAll; }
  const T* p[kPieces];
  int64_t step;
  // row_of: row of the tile -> row in memory, one that exists
  template <typename F>
  __device__ __forceinline__ Operand(const void* base, int64_t ld, int row0, int rows, F&& row_of) {
    step = KM ? BK * ld : BK;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = place(i), line = at / kRun, piece = swizzled(line, at % kRun);
      if constexpr (KM) p[i] = static_cast<const T*>(base) + line * ld + min(row0 + piece * 8, (rows - 1) & ~7);
      else p[i] = static_cast<const T*>(base) + row_of(line) * ld + piece * 8;
    }
  }
  // Straight to LDS, piece i of every lane: bfloat16 at addresses that are multiples of 16 bytes.  In assembly because the
  // compiler waits for all such loads before any read of LDS; whoever calls this waits for them (landed()).  It has no output,
  // and nothing else here uses m0.
  __device__ __forceinline__ void load_lds(int i, int64_t s, char* lds) const {
    static_assert(sizeof(T) == 2, "as it is in memory");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds)) +
                        (i * THREADS + wave * kWave) % kAll * 16;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p[i] + s * step), "s"(to) : "m0", "memory");
  }
  // By way of registers.
  struct Staged {
    u32x4 v[kPieces][kWords];
  };
  __device__ __forceinline__ void load(int64_t s, Staged& to) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
#pragma unroll
      for (int j = 0; j < kWords; ++j) to.v[i][j] = *reinterpret_cast<const u32x4_any*>(p[i] + s * step + j * (8 / kWords));
    }
  }
  // A step that ends beyond K, or whose pieces of rows may end beyond the tensor: zeros for what does not exist.
  __device__ __forceinline__ void load_rest(int64_t s, int row0, int rows, int K, Staged& to) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = place(i), line = at / kRun, piece = swizzled(line, at % kRun);
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
        to.v[i][j] = w;
      }
    }
  }
  __device__ static __forceinline__ void store(const Staged& from, char* lds) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      char* to = lds + place(i) * 16;
      if constexpr (kPlanes == 1) {
        *reinterpret_cast<u32x4*>(to) = from.v[i][0];
      } else {
        u32x4 w[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t part[3][2];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const uint32_t x = from.v[i][j / 2][2 * (j % 2) + n];
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
};

// ---- products ---------------------------------------------------------------------------------------------------------
// c[m][n] = sum_k a(m, k) b(n, k); gated: the pairs of columns f and F + f of such a c are g and u.
struct Product {
  const void *a, *b;
  int64_t lda, ldb;
  int M, N, K;        // N: F if gated
  void* c;            // [M, N]
  float* partial;     // splits > 1: [splits, M, N] ([splits, M, 2F]) sums of k's parts
  int splits, steps;  // steps of BK values of k in a part
  const void* bias;   // gated: [2F] or null
  void* gu;           // gated: [M, 2F] or null
  void* h;            // gated: [M, F]
  int kind;
  float c0, c1;       // of act_value()
};
enum Epilogue { kPlain, kSigmoid, kErf };  // kPlain: not gated

// A workgroup owns BM x BN elements (gated: the g and u of BM x BN / 2), a wave WM x WN of them.
template <int BM_, int BN_, int WM_, int WN_, int BK_, int BUFS_ = 2>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, BUFS = BUFS_, FM = WM / 16, FN = WN / 16;
  static constexpr int kWavesN = BN / WN, kWaves = BM / WM * kWavesN, kThreads = kWave * kWaves;
};

// Where the workgroup's tile is.  Neighbouring workgroups go to different XCDs, each with an L2 of its own: every XCD takes a
// run of tiles, and these go down 8 rows of tiles before the next column.
template <typename C, bool GATED>
struct Place {
  static constexpr int kCols = GATED ? C::BN / 2 : C::BN;
  int split, m0, n0, wm, wn, wave;
  // Tile `block` of `total`, in the order of the launch.
  __device__ __forceinline__ Place(const Product& g, int block, int total) {
    const int tiles_m = (g.M + C::BM - 1) / C::BM, tiles_n = (g.N + kCols - 1) / kCols;
    const int xcd = block % 8, each = total / 8, more = total % 8, tile = xcd * each + min(xcd, more) + block / 8;
    split = tile / (tiles_m * tiles_n);
    const int in_split = tile - split * (tiles_m * tiles_n);
    const int band = in_split / (8 * tiles_n), in_band = in_split - band * (8 * tiles_n), rows = min(8, tiles_m - band * 8);
    m0 = (band * 8 + in_band % rows) * C::BM;
    n0 = in_band / rows * kCols;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    wm = wave / C::kWavesN * C::WM;
    wn = wave % C::kWavesN * C::WN;
  }
  // Rows of a tile's operands that exist; a wave's WN rows of b are those of g, then those of u, of WN / 2 columns of h.
  __device__ __forceinline__ int64_t a_row(const Product& g, int r) const { return min(m0 + r, g.M - 1); }
  __device__ __forceinline__ int64_t b_row(const Product& g, int r) const {
    if constexpr (!GATED) return min(n0 + r, g.N - 1);
    const int f = min(n0 + r / C::WN * (C::WN / 2) + r % (C::WN / 2), g.N - 1);
    return r % C::WN < C::WN / 2 ? f : int64_t{g.N} + f;
  }
};

// The operands of a wave for 32 values of k, and their product.
template <int PLANES, typename C>
struct Fragments {
  bf16x8 a[PLANES][C::FM], b[PLANES][C::FN];
  template <typename A, typename B>
  __device__ __forceinline__ void read(const char* la, const char* lb, int wm, int wn, int k) {
#pragma unroll
    for (int q = 0; q < PLANES; ++q) {
#pragma unroll
      for (int i = 0; i < C::FM; ++i) a[q][i] = A::read(la + q * A::kPlane, wm + i * 16, k);
#pragma unroll
      for (int j = 0; j < C::FN; ++j) b[q][j] = B::read(lb + q * B::kPlane, wn + j * 16, k);
    }
  }
  __device__ __forceinline__ void multiply(f32x4 (&acc)[C::FM][C::FN]) const {
    auto planes = [&](int qa, int qb) {
#pragma unroll
      for (int i = 0; i < C::FM; ++i)
#pragma unroll
        for (int j = 0; j < C::FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[qb][j], a[qa][i], acc[i][j], 0, 0, 0);
    };
    if constexpr (PLANES == 3) {  // the small ones first
      planes(0, 2);
      planes(2, 0);
      planes(1, 1);
      planes(0, 1);
      planes(1, 0);
    }
    planes(0, 0);
  }
};

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
  groups<kFirst, READS, 0, 0, (kFirst < 16 ? kFirst : 16)>();
  groups<kSecond, 0, WRITES, LOADS, (kSecond < 16 ? kSecond : 16)>();
}

// Blocks of 16 rows, of the N that a wave has, which fit into `bytes` of LDS in rows of `row` bytes and 16 more.
constexpr int blocks_at_once(int N, int row, int bytes) {
  return N <= 1 || 16 * N * (row + 16) <= bytes ? N : blocks_at_once(N / 2, row, bytes);
}
// 16 BLOCKS rows by J x 16 columns of a wave's sums to memory, through LDS of its own, so that lanes side by side store pieces
// side by side.  value(i, j): elements (m = 16 i + lane % 16, n = 16 j + 4 (lane / 16) ..) of them; rows, cols: how many exist.
template <typename U, int BLOCKS, int J, typename F>
__device__ __forceinline__ void store_rows(char* lds, U* out, int64_t ld, int rows, int cols, F&& value) {
  constexpr int kRow = J * 16 * sizeof(U), kPitch = kRow + 16, E = 16 / sizeof(U), kLanes = kRow / 16, kOnce = kWave / kLanes;
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      char* to = lds + (16 * i + lane % 16) * kPitch + (j * 16 + 4 * (lane / 16)) * sizeof(U);
      const f32x4 v = value(i, j);
      if constexpr (sizeof(U) == 4) *reinterpret_cast<f32x4*>(to) = v;
      else *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
  }
  wave_lds_fence();
  const int col = lane % kLanes * E, left = cols - col;
#pragma unroll
  for (int i = 0; i < 16 * BLOCKS; i += kOnce) {
    const int row = i + lane / kLanes;
    if (row >= min(rows, 16 * BLOCKS) || left <= 0) continue;
    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + row * kPitch + col * sizeof(U));
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

// A wave's sums to memory.  room: its LDS, ROOM bytes; bias: LDS for the workgroup's BN values.  All waves call it, when LDS is
// free.
template <typename T, Epilogue END, typename C, int ROOM, typename P>
__device__ __forceinline__ void finish(const Product& g, const P& at, const f32x4 (&acc)[C::FM][C::FN], char* room, float* bias) {
  constexpr int FM = C::FM, FN = C::FN, BN = C::BN;
  const int lane = threadIdx.x % kWave, m = at.m0 + at.wm;
  if constexpr (END == kPlain) {
    const int n = at.n0 + at.wn;
    auto sums = [&](auto* to) {
      using U = std::remove_pointer_t<decltype(to)>;
      constexpr int kOnce = blocks_at_once(FM, FN * 16 * sizeof(U), ROOM);
      static_assert(16 * kOnce * (FN * 16 * sizeof(U) + 16) <= ROOM, "a block's rows");
#pragma unroll
      for (int i0 = 0; i0 < FM; i0 += kOnce)
        store_rows<U, kOnce, FN>(room, to + static_cast<int64_t>(m + 16 * i0) * g.N + n, g.N, g.M - m - 16 * i0, g.N - n,
                                 [&](int i, int j) { return acc[i0 + i][j]; });
    };
    if (g.splits > 1) sums(g.partial + static_cast<int64_t>(at.split) * g.M * g.N);
    else sums(static_cast<T*>(g.c));
  } else {
    for (int i = threadIdx.x; i < BN; i += C::kThreads) {
      const int f = min(at.n0 + i % (BN / 2), g.N - 1) + i / (BN / 2) * g.N;
      bias[i] = g.bias && g.splits == 1 ? Store<T>::load1(static_cast<const T*>(g.bias) + f) : 0.0f;
    }
    lds_barrier();
    constexpr int J = FN / 2;
    const int f = at.n0 + at.wn / 2;
    const float* const own = bias + at.wn / 2 + 4 * (lane / 16);
    auto gate = [&](int i, int j) { return acc[i][j] + *reinterpret_cast<const f32x4*>(own + j * 16); };
    auto up = [&](int i, int j) { return acc[i][j + J] + *reinterpret_cast<const f32x4*>(own + BN / 2 + j * 16); };
    auto rows = [&](auto* to, int64_t ld, auto&& value) {
      using U = std::remove_pointer_t<decltype(to)>;
      constexpr int kOnce = blocks_at_once(FM, J * 16 * sizeof(U), ROOM);
      static_assert(16 * kOnce * (J * 16 * sizeof(U) + 16) <= ROOM, "a block's rows");
#pragma unroll
      for (int i0 = 0; i0 < FM; i0 += kOnce)
        store_rows<U, kOnce, J>(room, to + (m + 16 * i0) * ld + f, ld, g.M - m - 16 * i0, g.N - f,
                                [&](int i, int j) { return value(i0 + i, j); });
    };
    auto sums = [&](auto* to) {
      rows(to, 2 * static_cast<int64_t>(g.N), gate);
      rows(to + g.N, 2 * static_cast<int64_t>(g.N), up);
    };
    if (g.splits > 1) {
      sums(g.partial + static_cast<int64_t>(at.split) * g.M * 2 * g.N);
    } else {
      if (g.gu) sums(static_cast<T*>(g.gu));
      rows(static_cast<T*>(g.h), g.N, [&](int i, int j) {
        f32x4 v = gate(i, j);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = act_value<END == kErf>(v[e], g.c0, g.c1);
        return v * up(i, j);
      });
    }
  }
}

template <typename C>
__device__ __forceinline__ void clear(f32x4 (&acc)[C::FM][C::FN]) {
#pragma unroll
  for (int i = 0; i < C::FM; ++i)
#pragma unroll
    for (int j = 0; j < C::FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
}
// The steps from `whole` on, one after the other, through one buffer.
template <typename A, typename B, typename C, typename P>
__device__ __forceinline__ void rest_of_k(const Product& g, const P& at, const A& a, const B& b, int whole, int end, char* lds,
                                          f32x4 (&acc)[C::FM][C::FN]) {
  for (int s = whole; s < end && s * int64_t{C::BK} < g.K; ++s) {
    typename A::Staged va;
    typename B::Staged vb;
    a.load_rest(s, at.m0, g.M, g.K, va);
    b.load_rest(s, at.n0, g.N, g.K, vb);
    A::store(va, lds);
    B::store(vb, lds + A::kBytes);
    lds_barrier();
#pragma unroll
    for (int k = 0; k < C::BK; k += 32) {
      Fragments<A::kPlanes, C> f;
      f.template read<A, B>(lds, lds + A::kBytes, at.wm, at.wn, k);
      f.multiply(acc);
    }
    lds_barrier();
  }
}

// Any type, size and address: operands by way of registers, two buffers in LDS.  While the matrix cores work on 32 values of
// k, the operands of the next ones come from LDS; behind the one barrier of a step, when all waves have read what it held,
// a buffer gets the step after the next, and the one behind that is on its way from memory.
// Two buffers that are two objects, so that writes to one are known not to be what is read from the other.
template <typename T, bool AKM, bool BKM, Epilogue END, typename C>
__device__ __forceinline__ void product_tile(const Product& g, int block, int total, char* even, char* odd) {
  using A = Operand<T, AKM, C::BM, C::BK, C::kThreads>;
  using B = Operand<T, BKM, C::BN, C::BK, C::kThreads>;
  constexpr int kPlanes = A::kPlanes, kBuffer = A::kBytes + B::kBytes, kParts = C::BK / 32;
  const Place<C, END != kPlain> at(g, block, total);
  const A a(g.a, g.lda, at.m0, g.M, [&](int r) { return at.a_row(g, r); });
  const B b(g.b, g.ldb, at.n0, g.N, [&](int r) { return at.b_row(g, r); });
  const int whole = whole_steps(g.K, C::BK, AKM ? g.M : 0, BKM ? g.N : 0);
  const int first = at.split * g.steps, end = first + g.steps, last = min(end, whole);
  f32x4 acc[C::FM][C::FN];
  clear<C>(acc);
  if (end > whole) rest_of_k<A, B, C>(g, at, a, b, max(whole, first), end, even, acc);
  if (first < last) {
    typename A::Staged va;
    typename B::Staged vb;
    Fragments<kPlanes, C> f[2];
    // No branch around the loads: behind one, the compiler waits for all that are under way.  Beyond the last step they
    // fetch that one again.
    auto fetch = [&](int s) {
      a.load(min(s, last - 1), va);
      b.load(min(s, last - 1), vb);
    };
    auto put = [&](char* lds) {
      A::store(va, lds);
      B::store(vb, lds + A::kBytes);
    };
    fetch(first);
    put(even);
    fetch(first + 1);
    put(odd);
    fetch(first + 2);
    lds_barrier();
    f[0].template read<A, B>(even, even + A::kBytes, at.wm, at.wn, 0);
    auto step = [&](int s, char* from, char* to, int parity) {
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
        const int now = (parity * kParts + part) & 1;
        constexpr int kMfma = C::FM * C::FN * (kPlanes == 3 ? 6 : 1);
        constexpr int kReads = kPlanes * (C::FM * (AKM ? 2 : 1) + C::FN * (BKM ? 2 : 1));
        if (part == kParts - 1) {
          lds_barrier();
          f[now ^ 1].template read<A, B>(to, to + A::kBytes, at.wm, at.wn, 0);
          put(from);
          fetch(s + 3);
          f[now].multiply(acc);
          spread<kMfma, kReads, kPlanes*(A::kPieces + B::kPieces), A::kWords * A::kPieces + B::kWords * B::kPieces>();
        } else {
          f[now ^ 1].template read<A, B>(from, from + A::kBytes, at.wm, at.wn, (part + 1) * 32);
          f[now].multiply(acc);
          spread<kMfma, kReads, 0, 0>();
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    for (int s = first; s < last; s += 2) {
      step(s, even, odd, 0);
      if (s + 1 == last) break;
      step(s + 1, odd, even, 1);
    }
    lds_barrier();
  }
  constexpr int kRoom = (kBuffer - C::BN * 4) / ((C::kWaves + 1) / 2) & ~15;
  finish<T, END, C, kRoom>(g, at, acc, (at.wave % 2 == 0 ? even : odd) + at.wave / 2 * kRoom,
                           reinterpret_cast<float*>(odd + kBuffer) - C::BN);
}

// Waits until all but the last N loads of the wave have come (and for nothing else).
template <int N>
__device__ __forceinline__ void landed() {
  static_assert(N < 64, "six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0xF70);
}
// bfloat16 whose rows begin at multiples of 16 bytes: memory to LDS without registers, BUFS - 1 steps ahead.
template <bool AKM, bool BKM, Epilogue END, typename C>
__device__ __forceinline__ void aligned_tile(const Product& g, int block, int total, char* lds) {
  using A = Operand<bf16_t, AKM, C::BM, C::BK, C::kThreads>;
  using B = Operand<bf16_t, BKM, C::BN, C::BK, C::kThreads>;
  constexpr int BUFS = C::BUFS, kParts = C::BK / 32, kBuffer = A::kBytes + B::kBytes, kLoads = A::kPieces + B::kPieces;
  const Place<C, END != kPlain> at(g, block, total);
  const A a(g.a, g.lda, at.m0, g.M, [&](int r) { return at.a_row(g, r); });
  const B b(g.b, g.ldb, at.n0, g.N, [&](int r) { return at.b_row(g, r); });
  const int whole = g.K / C::BK, first = at.split * g.steps, end = first + g.steps, last = min(end, whole);
  f32x4 acc[C::FM][C::FN];
  clear<C>(acc);
  if (end > whole) rest_of_k<A, B, C>(g, at, a, b, max(whole, first), end, lds, acc);
  if (first < last) {
    Fragments<1, C> f[2];
    auto load = [&](int i, int s, int buffer) {  // piece i of step s, beyond the last one that one's again
      char* const to = lds + buffer * kBuffer;
      if (i < A::kPieces) a.load_lds(i, min(s, last - 1), to);
      else b.load_lds(i - A::kPieces, min(s, last - 1), to + A::kBytes);
    };
    auto read = [&](int i, int to, int buffer, int k) {  // operand i of a wave
      const char* const from = lds + buffer * kBuffer;
      if (i < C::FN) f[to].b[0][i] = B::read(from + A::kBytes, at.wn + i * 16, k);
      else f[to].a[0][i - C::FN] = A::read(from, at.wm + (i - C::FN) * 16, k);
    };
    // Buffer s % BUFS has been read when all waves have come to the barrier of step s + 1; what step s loads goes to that of
    // s - 1.  The next step's operands are read in the first half of the matrix instructions, to have come by the end.
    auto step = [&](int s, auto turn) {
      constexpr int kMfma = C::FM * C::FN, kHalf = (kMfma + 1) / 2, kReads = C::FM + C::FN, buffer = turn % BUFS;
      landed<(BUFS - 3) * kLoads>();
      lds_barrier();
      for_each(std::make_integer_sequence<int, kParts * kMfma>{}, [&](auto count) {
        constexpr int part = count / kMfma, n = count % kMfma, i = n / C::FN, j = n % C::FN, now = (turn * kParts + part) & 1;
        for_each(std::make_integer_sequence<int, kReads>{}, [&](auto r) {
          if constexpr (r * kHalf / kReads == n) {
            if constexpr (part + 1 < kParts) read(r, now ^ 1, buffer, (part + 1) * 32);
            else read(r, now ^ 1, (buffer + 1) % BUFS, 0);
          }
        });
        for_each(std::make_integer_sequence<int, kLoads>{}, [&](auto l) {
          if constexpr ((2 * l + 1) * kParts * kMfma / (2 * kLoads) == count) load(l, s + BUFS - 1, (buffer + BUFS - 1) % BUFS);
        });
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[now].b[0][j], f[now].a[0][i], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
#pragma unroll
    for (int s = 0; s < BUFS - 1; ++s)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load(i, first + s, s);
    landed<(BUFS - 2) * kLoads>();
    lds_barrier();
#pragma unroll
    for (int i = 0; i < C::FM + C::FN; ++i) read(i, 0, 0, 0);
    constexpr int kTurns = BUFS * kParts % 2 == 0 ? BUFS : 2 * BUFS;  // buffers and operands' registers come round
    for (int s = first; s < last; s += kTurns) {
      const bool all = for_each_while(std::make_integer_sequence<int, kTurns>{}, [&](auto turn) {
        step(s + turn, turn);
        return s + turn + 1 < last;
      });
      if (!all) break;
    }
    landed<0>();
    lds_barrier();
  }
  constexpr int kRoom = (BUFS * kBuffer - C::BN * 4) / C::kWaves & ~15;
  finish<bf16_t, END, C, kRoom>(g, at, acc, lds + at.wave * kRoom, reinterpret_cast<float*>(lds + BUFS * kBuffer) - C::BN);
}

template <typename T, bool AKM, bool BKM, Epilogue END, typename C, bool ALIGNED>
__device__ __forceinline__ void any_tile(const Product& g, int block, int total, char* even, char* odd) {
  if constexpr (ALIGNED) aligned_tile<AKM, BKM, END, C>(g, block, total, even);
  else product_tile<T, AKM, BKM, END, C>(g, block, total, even, odd);
}
#define TEMPO_GLU_LDS(T, C, ALIGNED)                                                                                        \
  constexpr int kOne = (C::BM + C::BN) * C::BK * 2 * (sizeof(T) == 4 ? 3 : 1);                                              \
  __shared__ __attribute__((aligned(16))) char even[ALIGNED ? C::BUFS * kOne : kOne], odd[ALIGNED ? 16 : kOne]
template <typename T, bool AKM, bool BKM, Epilogue END, typename C, bool ALIGNED>
__global__ __launch_bounds__(C::kThreads) void product_kernel(Product g) {
  TEMPO_GLU_LDS(T, C, ALIGNED);
  any_tile<T, AKM, BKM, END, C, ALIGNED>(g, blockIdx.x, gridDim.x, even, odd);
}
// dx and dw, which need nothing of each other, in one launch.
template <typename T, typename C, bool ALIGNED>
__global__ __launch_bounds__(C::kThreads) void both_kernel(Product dx, Product dw, int dx_tiles) {
  TEMPO_GLU_LDS(T, C, ALIGNED);
  const int block = blockIdx.x;
  if (block < dx_tiles) any_tile<T, false, true, kPlain, C, ALIGNED>(dx, block, dx_tiles, even, odd);
  else any_tile<T, true, true, kPlain, C, ALIGNED>(dw, block - dx_tiles, gridDim.x - dx_tiles, even, odd);
}
#undef TEMPO_GLU_LDS

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

// Rows of `columns` bfloat16 elements, those of `first`, then those of `second`, copied to rows of `pieces` 16-byte pieces, zeros
// behind them.
__global__ __launch_bounds__(256) void pad_kernel(const bf16_t* first, uint32_t first_rows, const bf16_t* second, uint32_t rows,
                                                  int columns, uint32_t pieces, u32x4* to) {
  const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = at / pieces, column = (at - row * pieces) * 8;
  if (row >= rows) return;
  const bf16_t* from = (row < first_rows ? first + static_cast<int64_t>(row) * columns
                                         : second + static_cast<int64_t>(row - first_rows) * columns) + column;
  const int left = columns - static_cast<int>(column);
  u32x4 w;
  if (left >= 8) {
    w = *reinterpret_cast<const u32x4_any*>(from);
  } else {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? Store<bf16_t>::load1(from + e) : 0.0f;
    w = Store<bf16_t>::pack(v);
  }
  to[at] = w;
}

// ---- the backward's elementwise part ----------------------------------------------------------------------------------
// dg and du are rounded to the storage type before dx and dw: one operand of a matrix instruction each, as an autograd that keeps its
// tensors in that type has them.  In two bfloat16 parts they would count in float32, at twice the products: of [8192, 1024] x 2 x 4096 dx and dw are
// off by 2.34e-3 of their norm, by 1.66e-3 (their own rounding alone) with dgu in float32.  dbias is summed before the rounding.
struct Gates {
  const void *dh, *gu;
  void *dgu, *h;     // h may be null
  float* sums;       // null, or [groups, 2F]: column sums of a workgroup's rows
  int64_t rows;
  int F, kind, chunk;  // chunk: rows of a wave
  void* pad;           // null, or dgu once more, in rows of pad_ld elements
  int64_t pad_ld;
};
// A wave takes 64 pieces of 16 bytes of the columns, of `chunk` rows one after the other, the four of a workgroup those of
// neighbouring rows, whose sums they add up.
constexpr int kGateWaves = 4;
template <typename T, int KIND>
__global__ __launch_bounds__(kGateWaves* kWave) void gates_kernel(Gates g, int64_t group0) {
  constexpr int V = Store<T>::kVec;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, f = (blockIdx.x * kWave + lane) * V, left = g.F - f;
  const int64_t group = group0 + blockIdx.y, r0 = (group * kGateWaves + wave) * g.chunk;
  const int64_t r1 = left <= 0 ? r0 : r0 + g.chunk < g.rows ? r0 + g.chunk : g.rows;
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
    T* pad = g.pad ? static_cast<T*>(g.pad) + r * g.pad_ld + f : nullptr;
    if (left >= V) {
      const u32x4 wg = Store<T>::pack(dg), wu = Store<T>::pack(du);
      *reinterpret_cast<u32x4_any*>(dgu) = wg;
      *reinterpret_cast<u32x4_any*>(dgu + g.F) = wu;
      if (h) stg_stream_any(h, Store<T>::pack(y));
      if (pad) {
        *reinterpret_cast<u32x4_any*>(pad) = wg;
        *reinterpret_cast<u32x4_any*>(pad + g.F) = wu;
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (i >= left) break;
        Store<T>::store1(dgu + i, dg[i]);
        Store<T>::store1(dgu + g.F + i, du[i]);
        if (h) Store<T>::store1(h + i, y[i]);
        if (pad) {
          Store<T>::store1(pad + i, dg[i]);
          Store<T>::store1(pad + g.F + i, du[i]);
        }
      }
    }
  }
  if (g.sums) {  // uniform
    __shared__ float of_waves[kGateWaves][2 * V][kWave];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      of_waves[wave][i][lane] = sg[i];
      of_waves[wave][V + i][lane] = su[i];
    }
    lds_barrier();
    float* const to = g.sums + group * 2 * g.F + f;
#pragma unroll
    for (int n = 0; n < 2 * V / kGateWaves; ++n) {
      const int i = wave * (2 * V / kGateWaves) + n, column = i % V;
      const float v = (of_waves[0][i][lane] + of_waves[1][i][lane]) + (of_waves[2][i][lane] + of_waves[3][i][lane]);
      if (column < left) to[i / V * g.F + column] = v;
    }
  }
}
// The groups' sums of 64 columns, a quarter of the groups a wave, then the quarters.
template <typename T>
__global__ __launch_bounds__(4 * kWave) void bias_kernel(const float* sums, T* dbias, int64_t groups, int n) {
  __shared__ float quarters[4 * kWave];
  const int e = blockIdx.x * kWave + threadIdx.x % kWave, quarter = threadIdx.x / kWave;
  const int64_t each = (groups + 3) / 4, first = quarter * each, last = first + each < groups ? first + each : groups;
  float v = 0.0f;
  if (e < n) {
#pragma unroll 8
    for (int64_t c = first; c < last; ++c) v += sums[c * n + e];
  }
  quarters[threadIdx.x] = v;
  lds_barrier();
  if (quarter == 0 && e < n) {
    const float* q = quarters + threadIdx.x;
    Store<T>::store1(dbias + e, (q[0] + q[kWave]) + (q[2 * kWave] + q[3 * kWave]));
  }
}

// ---- the tiles of plans (glu_plan.h) ----------------------------------------------------------------------------------
// Register path: what has any type or address.  Aligned path: bfloat16 in rows of whole 16-byte pieces.
template <typename T>
using Middle = Tile<128, 128, 64, 64, sizeof(T) == 4 ? 32 : 64>;
template <typename T>
using Small = Tile<64, 64, 32, 32, sizeof(T) == 4 ? 32 : 64>;
using AlignedLarge = Tile<256, 256, 128, 128, 32, 4>;
using AlignedMiddle = Tile<128, 128, 64, 64, 32, 4>;
using AlignedSmall = Tile<64, 64, 32, 32, 64, 4>;
using AlignedFewest = Tile<16, 64, 16, 32, 64, 8>;
using AlignedFew = Tile<64, 64, 64, 32, 64, 5>;
using AlignedFewWide = Tile<64, 128, 64, 32, 64, 6>;

static_assert(AlignedFewest::BM == kFewestRows && AlignedFew::BM == kFewRows && AlignedFewWide::BM == kFewRows &&
                  AlignedFewest::BN == few_columns(Size::kFewest) && AlignedFew::BN == few_columns(Size::kFew) &&
                  AlignedFewWide::BN == few_columns(Size::kFewWide) && AlignedFewest::BK == kFewStep && AlignedFew::BK == kFewStep &&
                  AlignedFewWide::BK == kFewStep,
              "the plan's");

template <typename T, bool GATED, typename F>
tempo_status with_tile(const Plan& p, F&& f) {
  if (!p.aligned) return p.size == Size::kSmall ? f(Small<T>{}, std::false_type{}) : f(Middle<T>{}, std::false_type{});
  if constexpr (sizeof(T) == 2) {
    if constexpr (GATED) {
      if (p.size == Size::kFewest) return f(AlignedFewest{}, std::true_type{});
      if (p.size == Size::kFew) return f(AlignedFew{}, std::true_type{});
      if (p.size == Size::kFewWide) return f(AlignedFewWide{}, std::true_type{});
    }
    if (p.size == Size::kLarge) return f(AlignedLarge{}, std::true_type{});
    return p.size == Size::kMiddle ? f(AlignedMiddle{}, std::true_type{}) : f(AlignedSmall{}, std::true_type{});
  }
  return TEMPO_ERR_UNSUPPORTED;
}
template <typename T, bool GATED>
tempo_status join(const Product& g, hipStream_t st) {
  if (g.splits == 1) return TEMPO_OK;
  const int64_t n = int64_t{g.M} * g.N;
  hipLaunchKernelGGL((join_kernel<T, GATED>), dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, st, g);
  return launch_status();
}
template <typename T, bool AKM, bool BKM, Epilogue END>
tempo_status launch_product(Product g, const Plan& p, hipStream_t st) {
  if (p.tiles == 0) return TEMPO_OK;
  g.splits = p.splits;
  g.steps = p.steps;
  const tempo_status status = with_tile<T, END != kPlain>(p, [&](auto tile, auto aligned) {
    using C = decltype(tile);
    hipLaunchKernelGGL((product_kernel<T, AKM, BKM, END, C, decltype(aligned)::value>), dim3(static_cast<unsigned>(p.tiles)),
                       dim3(C::kThreads), 0, st, g);
    return launch_status();
  });
  return status == TEMPO_OK ? join<T, END != kPlain>(g, st) : status;
}
template <typename T>
tempo_status launch_both(Product dx, Product dw, const Plan* p, hipStream_t st) {
  dx.splits = p[0].splits, dx.steps = p[0].steps;
  dw.splits = p[1].splits, dw.steps = p[1].steps;
  tempo_status status = with_tile<T, false>(p[0], [&](auto tile, auto aligned) {
    using C = decltype(tile);
    hipLaunchKernelGGL((both_kernel<T, C, decltype(aligned)::value>), dim3(static_cast<unsigned>(p[0].tiles + p[1].tiles)),
                       dim3(C::kThreads), 0, st, dx, dw, static_cast<int>(p[0].tiles));
    return launch_status();
  });
  if (status == TEMPO_OK) status = join<T, false>(dx, st);
  return status == TEMPO_OK ? join<T, false>(dw, st) : status;
}

// Rows that a wave of the backward's elementwise part takes: 32, fewer where they would make less than 16 waves per compute unit,
// and not fewer than 4, so that the column sums of a workgroup's rows are few beside the rows.
int chunk_of(int64_t T, int64_t F, tempo_dtype dt) {
  const int64_t across = (F + (dt == TEMPO_F32 ? 4 : 8) * kWave - 1) / ((dt == TEMPO_F32 ? 4 : 8) * kWave);
  return static_cast<int>(std::min<int64_t>(32, std::max<int64_t>(4, T * across / (16 * int64_t{compute_units()}))));
}
int64_t groups_of(int64_t T, int chunk) { return (T + kGateWaves * chunk - 1) / (kGateWaves * chunk); }
size_t sums_bytes(int64_t T, int64_t F, tempo_dtype dt) {
  return static_cast<size_t>(groups_of(T, chunk_of(T, F, dt))) * 2 * F * sizeof(float);
}

// The rows of first, then those of second; either may have none.
tempo_status pad(const void* first, int64_t first_rows, const void* second, int64_t second_rows, int64_t columns, int64_t ld, void* to,
                 hipStream_t st) {
  const int64_t rows = first_rows + second_rows, pieces = ld / 8;
  if (rows == 0) return TEMPO_OK;
  hipLaunchKernelGGL(pad_kernel, dim3(static_cast<unsigned>((rows * pieces + 255) / 256)), dim3(256), 0, st,
                     static_cast<const bf16_t*>(first), static_cast<uint32_t>(first_rows), static_cast<const bf16_t*>(second),
                     static_cast<uint32_t>(rows), static_cast<int>(columns), static_cast<uint32_t>(pieces), static_cast<u32x4*>(to));
  return launch_status();
}
template <typename T>
tempo_status forward(const GluCall& c, const ForwardPlan& p, hipStream_t st) {
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
  if (p.padded) {
    char* const to = static_cast<char*>(c.workspace) + p.x_at;
    const tempo_status status = pad(c.x, c.T, c.w, 2 * c.F, c.H, p.H_pad, to, st);
    if (status != TEMPO_OK) return status;
    g.a = to;
    g.b = to + c.T * p.H_pad * 2;
    g.lda = g.ldb = p.H_pad;
  }
  constexpr float log2e = 1.4426950408889634f, k = 0.7978845608028654f;
  if (c.kind == TEMPO_GLU_GELU_ERF) return launch_product<T, false, false, kErf>(g, p.plan, st);
  g.c0 = c.kind == TEMPO_GLU_SILU ? -log2e : -2.0f * log2e * k;
  g.c1 = c.kind == TEMPO_GLU_SILU ? 0.0f : -2.0f * log2e * k * 0.044715f;
  return launch_product<T, false, false, kSigmoid>(g, p.plan, st);
}

template <typename T>
tempo_status backward(const GluCall& c, const BackwardPlan& p, hipStream_t st) {
  constexpr int V = Store<T>::kVec;
  Gates e{c.dh, c.gu, c.dgu, c.h, c.dbias ? static_cast<float*>(c.workspace) : nullptr, c.T, static_cast<int>(c.F), c.kind,
          chunk_of(c.T, c.F, sizeof(T) == 4 ? TEMPO_F32 : TEMPO_BF16)};
  const int64_t row_groups = groups_of(c.T, e.chunk);
  char* const workspace = static_cast<char*>(c.workspace);
  const bool copied = p.padded && p.F2_pad != 2 * c.F && (c.dx || c.dw);
  if (copied) {
    e.pad = workspace + p.dgu_at;
    e.pad_ld = p.F2_pad;
    if (c.dbias) e.sums = reinterpret_cast<float*>(workspace + p.bytes);  // else where the products' parts will be
  }
  const unsigned across = static_cast<unsigned>((c.F + V * kWave - 1) / (V * kWave));
  auto gates = [&](auto kernel) {
    constexpr int kThreads = kGateWaves * kWave;
    return split_launch(row_groups, std::min<int64_t>(65535, most_groups(row_groups, kThreads * across)), [&](uint32_t first, uint32_t n) {
      hipLaunchKernelGGL(kernel, dim3(across, n), dim3(kThreads), 0, st, e, int64_t{first});
      return launch_status() == TEMPO_OK;
    });
  };
  if (row_groups > 0 && across > 0 &&
      !(c.kind == TEMPO_GLU_SILU ? gates(gates_kernel<T, TEMPO_GLU_SILU>)
        : c.kind == TEMPO_GLU_GELU_ERF ? gates(gates_kernel<T, TEMPO_GLU_GELU_ERF>)
                                       : gates(gates_kernel<T, TEMPO_GLU_GELU_TANH>)))
    return TEMPO_ERR_LAUNCH;
  tempo_status status = TEMPO_OK;
  if (c.dbias && c.F > 0) {
    const int n = static_cast<int>(2 * c.F);
    hipLaunchKernelGGL((bias_kernel<T>), dim3((n + kWave - 1) / kWave), dim3(4 * kWave), 0, st, e.sums, static_cast<T*>(c.dbias), row_groups, n);
    status = launch_status();
  }
  if (status != TEMPO_OK || c.H == 0) return status;
  Product dx{}, dw{};
  dx.a = dw.a = c.dgu;
  dx.lda = dw.lda = 2 * c.F;
  dx.ldb = dw.ldb = c.H;
  dx.N = dw.N = static_cast<int>(c.H);
  dx.M = dw.K = static_cast<int>(c.T);
  dx.K = dw.M = static_cast<int>(2 * c.F);
  dx.b = c.w;
  dx.c = c.dx;
  dx.partial = static_cast<float*>(c.workspace);
  dw.b = c.x;
  dw.c = c.dw;
  dw.partial = dx.partial + p.dx_bytes / sizeof(float);
  const bool x = c.dx && c.T > 0, w = c.dw && c.F > 0;
  if (copied) {
    dx.a = dw.a = e.pad;
    dx.lda = dw.lda = p.F2_pad;
  }
  if (p.padded && p.H_pad != c.H) {
    char* const to = workspace + p.x_at;
    status = pad(c.x, w ? c.T : 0, c.w, x ? 2 * c.F : 0, c.H, p.H_pad, to, st);
    if (status != TEMPO_OK) return status;
    dw.b = to;
    dx.b = to + (w ? c.T : 0) * p.H_pad * 2;
    dx.ldb = dw.ldb = p.H_pad;
  }
  if (x && w) return launch_both<T>(dx, dw, p.plans, st);
  if (x) return launch_product<T, false, true, kPlain>(dx, p.plans[0], st);
  return w ? launch_product<T, true, true, kPlain>(dw, p.plans[1], st) : TEMPO_OK;
}

}  // namespace

bool glu_takes(int64_t T, int64_t H, int64_t F) {
  const int64_t most = int64_t{1} << 30;  // of what is counted in 32 bits
  if (T > most || H > most || F > most / 2) return false;
  // Two products of tiles of 64 x 64 elements, 256 lanes each, make 2^31 of the 2^32 lanes that a launch may have; parts of k are made
  // of few tiles.
  auto tiles = [](int64_t M, int64_t N) { return ((M + 63) / 64) * ((N + 63) / 64); };
  return tiles(T, 2 * F) < most / 256 && tiles(T, H) < most / 256 && tiles(2 * F, H) < most / 256;
}

size_t glu_workspace_bytes(int64_t T, int64_t H, int64_t F, tempo_dtype dt, bool back) {
  if (!back) return ForwardPlan(T, H, F, dt, compute_units()).bytes;
  const BackwardPlan p(T, H, F, dt, compute_units());
  return p.padded ? p.bytes + sums_bytes(T, F, dt) : std::max(p.bytes, sums_bytes(T, F, dt));
}

tempo_status launch_glu_fwd(const GluCall& c, tempo_dtype dt, hipStream_t st) {
  const ForwardPlan p(c.T, c.H, c.F, dt, compute_units());
  if (p.bytes > c.workspace_bytes) return TEMPO_ERR_WORKSPACE;
  return dt == TEMPO_F32 ? forward<float>(c, p, st) : forward<bf16_t>(c, p, st);
}

tempo_status launch_glu_bwd(const GluCall& c, tempo_dtype dt, hipStream_t st) {
  const BackwardPlan p(c.T, c.H, c.F, dt, compute_units());
  const size_t products = c.dx || c.dw ? p.bytes : 0, sums = c.dbias ? sums_bytes(c.T, c.F, dt) : 0;
  if ((p.padded ? products + sums : std::max(products, sums)) > c.workspace_bytes) return TEMPO_ERR_WORKSPACE;
  return dt == TEMPO_F32 ? backward<float>(c, p, st) : backward<bf16_t>(c, p, st);
}

}  // namespace tempo
