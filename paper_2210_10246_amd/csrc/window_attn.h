// Attention with a sliding window and first tokens that stay visible, forward and backward, without a matrix of scores in memory:
//   s_ij = scale q_i . k_j of the keys that row i sees,  lse_i = ln sum_j exp s_ij,  p_ij = exp(s_ij - lse_i),  out_i = sum_j p_ij v_j;
//   delta_i = dout_i . out_i,  ds_ij = p_ij (dout_i . v_j - delta_i) scale,
//   dq_i = sum_j ds_ij k_j,  dk_j = sum_i ds_ij q_i,  dv_j = sum_i p_ij dout_i.
// Row i of a sequence stands at position P = query_start + i and sees the keys j <= P, j < key_len with j > P - window or j < sinks.
//
// The query heads that share a key head are rows of one problem: row r is query r / group of head r % group of them, so that a key is
// read once for all of them, in a call for a single token too, and the gradients of a shared head are one sum.
//
// All products are on the matrix cores, 32 x 32 at a time, and made so that what a lane gets of one is what it has to give to the next:
// of S^T = K Q^T lane n holds 16 keys of row n % 32, which is how a matrix instruction takes P^T for O^T = V^T P^T, whatever the
// order of the keys, so long as the other operand has the same one.  Maximum, sum and what rescales the output are then one number a
// lane.  The backward is made twice from S, once by rows (dq) and once by keys (dk, dv): 14 D operations a pair and not 10, but each
// gradient is summed in one place in a fixed order, without atomics.
#ifndef TEMPO_WINDOW_ATTN_H_
#define TEMPO_WINDOW_ATTN_H_

#include <algorithm>
#include <type_traits>

#include "tempo_device.h"
#include "tempo_host.h"

namespace tempo {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kRows = 32 * kWaves;  // rows (or keys, in the backward by keys) of a workgroup, 32 of a wave
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMinusInf = -__builtin_inff();

struct Heads {
  const void* p;
  int64_t batch, token, head;  // elements
};
struct Attn {
  Heads q, k, v, out, dout, dq, dk, dv;
  float* lse;          // [B, heads, Sq]
  float* stats;        // backward: lse of base 2, then delta, [2, B, heads, Sq]
  int64_t stat_rows;   // B heads Sq
  const int32_t *key_len, *query_start;
  int Sq, Sk, heads, kv_heads, group, rows, D;  // rows: Sq * group
  FastDiv by_group;
  int64_t window;  // positions go up to 2^32
  int sinks;
  float scale, c;  // c: scale log2(e)
  int tiles, splits;
  int pitch;                     // floats of a row of sums in the workspace: D up to whole pieces
  float *partial, *partial_lse;  // splits > 1: [splits, B kv_heads, rows, pitch] and [splits, B kv_heads, rows], of base 2
};

// Which keys the queries of a sequence see.
struct Sight {
  int64_t start, before;  // position of the first query, and of the last key before its window
  int keys, sinks;
  __device__ __forceinline__ Sight(const Attn& a, int b) {
    keys = a.key_len ? min(max(a.key_len[b], 0), a.Sk) : a.Sk;
    start = a.query_start ? a.query_start[b] : int64_t{a.Sk} - a.Sq;
    before = start - a.window;
    sinks = min(a.sinks, keys);
  }
  // keys [begin, end) and those below min(sinks, end)
  __device__ __forceinline__ int end(int i) const {
    const int64_t e = start + i + 1;
    return e <= 0 ? 0 : e < keys ? static_cast<int>(e) : keys;
  }
  __device__ __forceinline__ int begin(int i) const {
    const int64_t e = before + i + 1;
    return e <= 0 ? 0 : e < INT32_MAX ? static_cast<int>(e) : INT32_MAX;
  }
};

// ---- matrices in LDS ----------------------------------------------------------------------------------------------------
// Rows of DP elements in pieces of 16 bytes.  A matrix instruction takes 32 rows by two pieces (lane n: row n % 32, piece 2 s + n / 32)
// or, transposed, 32 columns by the rows that a lane's sums of the other product lie in (4 (n / 32) + 0 .. 3 of each eight).
// Pieces are stored in another order in each row, in bfloat16 rows of 16 pieces and more with a gap behind every fourth row, so that the
// lanes of a read meet different banks.
template <typename T, int DP>
struct Rows {
  // pieces of a row, room for them, a power of two, and matrix instructions that take two of them each
  static constexpr int V = Store<T>::kVec, P = DP / V, kRoom = P <= 8 ? 8 : P <= 16 ? 16 : P <= 32 ? 32 : 64, kSteps = P / 2;
  static constexpr int kPitch = kRoom * 16, kGap = sizeof(T) == 2 && kRoom >= 16 ? 16 : 0;
  static constexpr int bytes(int rows) { return rows * kPitch + rows / 4 * kGap; }
  __device__ static __forceinline__ int swizzle(int row) {
    if constexpr (sizeof(T) == 4) return (row >> 2 & 1) << 3 | (row & 3) | (row >> 3 & 1) << 2;
    else if constexpr (kRoom == 8) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
    else return (row & 3) << 2;
  }
  __device__ static __forceinline__ int place(int row) { return row * kPitch + row / 4 * kGap; }
  __device__ static __forceinline__ u32x4 rows(const char* lds, int row0, int step) {
    const int lane = threadIdx.x % kWave, row = lane % 32, piece = 2 * step + lane / 32;
    return *reinterpret_cast<const u32x4*>(lds + bytes(row0) + place(row) + ((piece ^ swizzle(row)) << 4));
  }
};

// 32 x 32 sums += 32 rows x two pieces of each operand.
template <typename T>
__device__ __forceinline__ f32x16 multiply(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(as_f32(a[e]), as_f32(b[e]), c, 0, 0, 0);
    return c;
  }
}

// The 16 sums of a lane as operands of the next product.  bfloat16: rounded, as its other operand is; the sums that they go into
// are over hundreds of them.
template <typename T>
struct Weights;
template <>
struct Weights<bf16_t> {
  u32x4 w[2];
  __device__ __forceinline__ explicit Weights(const f32x16& p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 4][i % 4] = pack_bf16(p[2 * i], p[2 * i + 1]);
  }
};
template <>
struct Weights<float> {
  f32x16 w;
  __device__ __forceinline__ explicit Weights(const f32x16& p) : w(p) {}
};

// sums[columns 32 block .. + 31] += transposed 32 rows of LDS x weights
template <typename T, int DP>
__device__ __forceinline__ f32x16 multiply_columns(const char* lds, int row0, int block, const Weights<T>& w, f32x16 c) {
  using R = Rows<T, DP>;
  const int lane = threadIdx.x % kWave;
  if constexpr (sizeof(T) == 2) {
    // 16 lanes read 4 rows of 16 columns, 4 columns each, and get 4 rows of a column each
    const int j = lane % 16, line = 4 * (lane / 32) + j / 4, piece = block * 4 + (lane / 16 & 1) * 2 + (j % 4) / 2;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      union {
        s16x4 h[2];
        bf16x8 all;
      } a;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int r = 16 * u + 8 * n;  // rows beyond `line`, whose order of pieces is that of line but for rows of 8 pieces
        a.h[n] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + R::bytes(row0 + r) + R::place(line) +
                                                                      ((piece ^ R::swizzle(R::kGap ? line : line + r)) << 4) + (j & 1) * 8));
      }
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.all, __builtin_bit_cast(bf16x8, w.w[u]), c, 0, 0, 0);
    }
  } else {
    const int column = block * 32 + lane % 32;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = row0 + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
      const float a = *reinterpret_cast<const float*>(lds + R::place(r) + ((column / 4 ^ R::swizzle(r)) << 4) + column % 4 * 4);
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w.w[i], c, 0, 0, 0);
    }
  }
  return c;
}

// Piece `piece` of a row of D elements at any address: what is loaded, by all lanes at once, and what the piece then is.  A piece that the row ends
// in is loaded from earlier on, and its elements are moved to their places once they have come, those behind the row become 0.  With a branch for
// such pieces beside the load, the wave waits for each load there: one token of 16 sequences, 4096 keys of 32 / 8 heads of 83 float32 181 us,
// 275 with it; 2 x 1000 tokens of 8 / 2 heads of 125 bfloat16 backward 114 us, 159 with it.
template <typename T, bool STREAM = false, bool WHOLE = false>
__device__ __forceinline__ u32x4 load_piece(const T* row, int piece, int D) {
  constexpr int V = Store<T>::kVec;
  if (!WHOLE && D < V) {
    float e[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float x = Store<T>::load1(row + min(j, D - 1));
      e[j] = j < D ? x : 0.0f;
    }
    return Store<T>::pack(e);
  }
  const T* const p = row + (WHOLE ? piece * V : min(piece * V, D - V));
  return STREAM ? ldg_stream_any(p) : *reinterpret_cast<const u32x4_any*>(p);
}
template <typename T>
__device__ __forceinline__ u32x4 fitted(u32x4 v, int piece, int D, int DP) {
  constexpr int V = Store<T>::kVec;
  if (D == DP) return v;
  const int left = D - piece * V;
  if (D % V != 0 && D > V) {
    const int by = left > 0 && left < V ? V - left : 0;  // elements
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = by & 1 ? v[n] >> 16 | (n < 3 ? v[n + 1] << 16 : 0) : v[n];
    }
#pragma unroll
    for (int words = 1; words < 4; words *= 2) {
      const bool moves = by * static_cast<int>(sizeof(T)) / 4 & words;
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = moves ? (n + words < 4 ? v[n + words] : 0) : v[n];
    }
  }
#pragma unroll
  for (int n = 0; n < 4; ++n) v[n] = left > 0 ? v[n] : 0;
  return v;
}
// Every second piece of a row, from `first` on.
template <typename T, int DP>
__device__ __forceinline__ void load_half_row(const T* row, int first, int D, u32x4 (&to)[Rows<T, DP>::kSteps]) {
#pragma unroll
  for (int p = 0; p < Rows<T, DP>::kSteps; ++p) to[p] = load_piece<T>(row, 2 * p + first, D);
}
template <typename T, int DP>
__device__ __forceinline__ void fit_half_row(int first, int D, u32x4 (&v)[Rows<T, DP>::kSteps]) {
#pragma unroll
  for (int p = 0; p < Rows<T, DP>::kSteps; ++p) v[p] = fitted<T>(v[p], 2 * p + first, D, DP);
}

// N rows of a matrix on their way to LDS by way of registers.
template <typename T, int DP, int N>
struct Staged {
  using R = Rows<T, DP>;
  static constexpr int kPieces = N * R::kRoom / kThreads;
  static_assert(N * R::kRoom % kThreads == 0, "whole pieces a lane");
  u32x4 v[kPieces];
  __device__ __forceinline__ explicit Staged(const Heads&) {}
  // of: row -> its elements
  template <typename F>
  __device__ __forceinline__ void load(int D, F&& of) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = i * kThreads + static_cast<int>(threadIdx.x), row = at / R::kRoom, piece = at % R::kRoom ^ R::swizzle(row);
      v[i] = load_piece<T>(of(row), piece, D);
    }
  }
  __device__ __forceinline__ void store(int D, char* lds) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = i * kThreads + static_cast<int>(threadIdx.x), row = at / R::kRoom, piece = at % R::kRoom ^ R::swizzle(row);
      *reinterpret_cast<u32x4*>(lds + R::place(row) + at % R::kRoom * 16) = fitted<T>(v[i], piece, D, DP);
    }
  }
};

// Waits until all of the wave's loads have come (and for nothing else).
__device__ __forceinline__ void landed() { __builtin_amdgcn_s_waitcnt(0xF70); }
// N rows of a matrix from memory to LDS without registers: rows that begin at multiples of 16 bytes, D a multiple of a piece.  In assembly
// because the compiler waits for all such loads before any read of LDS; whoever calls this waits for them.  It has no output, and nothing else
// here uses m0.  Lanes of pieces behind D load nothing, and what LDS holds there stays.
template <typename T, int DP, int N>
struct Direct {
  using R = Rows<T, DP>;
  static constexpr int kPieces = N * R::kRoom / kThreads;
  static_assert(R::kGap == 0 || R::kRoom * 4 % kWave == 0 || kWave % (R::kRoom * 4) == 0, "no gap within what a wave loads");
  uint32_t offset[kPieces];  // bytes from the first row
  __device__ __forceinline__ Direct(const Heads& h) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      offset[i] = static_cast<uint32_t>(row(i)) * static_cast<uint32_t>(h.token * sizeof(T)) + static_cast<uint32_t>(piece(i)) * 16;
  }
  __device__ static __forceinline__ int row(int i) { return (i * kThreads + static_cast<int>(threadIdx.x)) / R::kRoom; }
  __device__ static __forceinline__ int piece(int i) {
    return (i * kThreads + static_cast<int>(threadIdx.x)) % R::kRoom ^ R::swizzle(row(i));
  }
  __device__ static __forceinline__ uint32_t to(char* lds, int i) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds)) +
           R::place((i * kThreads + wave * kWave) / R::kRoom) + (i * kThreads + wave * kWave) % R::kRoom * 16;
  }
  // first: the first row (uniform)
  __device__ __forceinline__ void load(const T* first, int D, char* lds) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (R::kRoom * R::V == D || piece(i) * R::V < D)
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" ::"v"(offset[i]), "s"(to(lds, i)), "s"(first) : "m0", "memory");
  }
  // of: row -> its elements
  template <typename F>
  __device__ __forceinline__ void load_each(int D, char* lds, F&& of) const {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const T* const p = of(row(i)) + piece(i) * R::V;
      if (R::kRoom * R::V == D || piece(i) * R::V < D)
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(to(lds, i)) : "m0", "memory");
    }
  }
};
__device__ __forceinline__ void clear_lds(char* lds, int bytes) {
  for (int i = threadIdx.x * 16; i < bytes; i += kThreads * 16) *reinterpret_cast<u32x4*>(lds + i) = u32x4{0, 0, 0, 0};
}

template <typename T>
__device__ __forceinline__ const T* at(const Heads& h, int b, int token, int head) {
  return static_cast<const T*>(h.p) + b * h.batch + token * h.token + head * h.head;
}

// Four neighbouring elements of a row of D.
template <typename T>
__device__ __forceinline__ void store_four(T* row, int D, int d, f32x4 v) {
  const int left = D - d;
  if (left >= 4) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_any*>(row + d) = v;
    else *reinterpret_cast<u32x2_any*>(row + d) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) Store<T>::store1(row + d + e, v[e]);
  }
}
// A lane's sums of column block `block`: 8 (i / 4) + 4 (lane / 32) + i % 4 are four neighbours each.
template <typename T>
__device__ __forceinline__ void store_sums(T* row, int D, int block, const f32x16& s, float by) {
  const int d = block * 32 + 4 * (static_cast<int>(threadIdx.x) % kWave / 32);
#pragma unroll
  for (int n = 0; n < 4; ++n) store_four(row, D, d + 8 * n, f32x4{s[4 * n], s[4 * n + 1], s[4 * n + 2], s[4 * n + 3]} * by);
}
__device__ __forceinline__ f32x16 zeros() { return f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0}; }

// Neighbouring workgroups go to different XCDs, each with an L2 of its own: every XCD takes a run of them.
__device__ __forceinline__ int in_order(int block, int total) {
  const int xcd = block % 8, each = total / 8, more = total % 8;
  return xcd * each + min(xcd, more) + block / 8;
}

// The key tiles that the rows of a workgroup see: those of the first keys, then those of the window.
struct KeyTiles {
  int of_sinks, first, count;
  int low, high, sinks;  // seen by some row: [low, high) and those below sinks
  __device__ __forceinline__ KeyTiles(const Sight& s, int i0, int i1, int keys) {
    low = s.begin(i0);
    high = s.end(i1);
    sinks = min(s.sinks, high);
    of_sinks = (sinks + keys - 1) / keys;
    first = max(low / keys, of_sinks);
    count = of_sinks + (low < high ? max((high + keys - 1) / keys - first, 0) : 0);
  }
  __device__ __forceinline__ int key(int n, int keys) const { return (n < of_sinks ? n : first + n - of_sinks) * keys; }
  // Whether some row sees key j of a tile; if none does, one beside it that is seen, whose elements are then in its place: of a key that
  // is not looked at nothing is known, and 0 times it need not be 0.
  __device__ __forceinline__ bool all(int j0, int keys) const { return j0 + keys <= high && (j0 >= low || j0 + keys <= sinks); }
  __device__ __forceinline__ int seen(int j) const {
    if (j < sinks || (j >= low && j < high)) return j;
    return low < high ? min(max(j, low), high - 1) : sinks - 1;
  }
};

// The tiles of k and v that the rows of a workgroup see, one after the other through two buffers: while one is worked on, the next is on
// its way.  DIRECT: without registers.
template <typename T, int DP, int BK, bool DIRECT>
struct KeyStream {
  static constexpr int kBytes = Rows<T, DP>::bytes(BK);
  const Attn& a;
  const KeyTiles& keys;
  const T *k, *v;  // of key 0
  char (*lds)[2][kBytes];
  int n0, n1;
  std::conditional_t<DIRECT, Direct<T, DP, BK>, Staged<T, DP, BK>> ks, vs;
  // Tiles [n0, n1); the first one is on its way from here on.
  __device__ __forceinline__ KeyStream(const Attn& a_, const KeyTiles& keys_, int b, int kv, char (*lds_)[2][kBytes], int n0_, int n1_)
      : a(a_), keys(keys_), k(at<T>(a_.k, b, 0, kv)), v(at<T>(a_.v, b, 0, kv)), lds(lds_), n0(n0_), n1(n1_), ks(a_.k), vs(a_.v) {
    if (DIRECT && a.D < DP) {
      clear_lds(lds[0][0], 4 * kBytes);
      lds_barrier();
    }
    if (n0 < n1) fetch(n0, 0);
  }
  __device__ __forceinline__ void fetch(int n, int to) {
    const int j0 = keys.key(n, BK);
    if constexpr (DIRECT) {
      if (keys.all(j0, BK)) {
        ks.load(k + j0 * a.k.token, a.D, lds[to][0]);
        vs.load(v + j0 * a.v.token, a.D, lds[to][1]);
      } else {
        ks.load_each(a.D, lds[to][0], [&](int r) { return k + keys.seen(j0 + r) * a.k.token; });
        vs.load_each(a.D, lds[to][1], [&](int r) { return v + keys.seen(j0 + r) * a.v.token; });
      }
    } else {
      ks.load(a.D, [&](int r) { return k + keys.seen(j0 + r) * a.k.token; });
      vs.load(a.D, [&](int r) { return v + keys.seen(j0 + r) * a.v.token; });
    }
  }
  __device__ __forceinline__ void put(int to) {
    if constexpr (!DIRECT) {
      ks.store(a.D, lds[to][0]);
      vs.store(a.D, lds[to][1]);
    }
  }
  // work(tile's first key, its k, its v)
  template <typename F>
  __device__ __forceinline__ void each(F&& work) {
    if (n0 < n1) put(0);
    for (int n = n0; n < n1; ++n) {
      const int now = (n - n0) & 1;
      if constexpr (DIRECT) landed();
      lds_barrier();  // the tile is there, and the other buffer has been read
      if (n + 1 < n1) fetch(n + 1, now ^ 1);
      work(keys.key(n, BK), lds[now][0], lds[now][1]);
      if (n + 1 < n1) put(now ^ 1);
    }
  }
};

// The key (or query) of a lane's sum i.
__device__ __forceinline__ int key_of(int i) { return 8 * (i / 4) + 4 * (static_cast<int>(threadIdx.x) % kWave / 32) + i % 4; }

// What a wave's 32 rows see of keys [j0, j0 + n).
struct WaveRows {
  int r0, row, i, g;        // the wave's first row, the lane's, its query and head
  bool any;                 // rows that exist
  int begin, end;           // of the lane
  int first_begin, last_begin, first_end, last_end;
  __device__ __forceinline__ WaveRows(const Attn& a, const Sight& s, int r0_) : r0(r0_), any(r0_ < a.rows) {
    const int lane = threadIdx.x % kWave, last = a.rows - 1;
    row = min(r0 + lane % 32, last);
    i = a.by_group.divide(row);
    g = row - i * a.group;
    begin = s.begin(i);
    end = s.end(i);
    const int i0 = a.by_group.divide(min(r0, last)), i1 = a.by_group.divide(min(r0 + 31, last));
    first_begin = s.begin(i0), last_begin = s.begin(i1), first_end = s.end(i0), last_end = s.end(i1);
  }
  __device__ __forceinline__ bool none(const Sight& s, int j0, int n) const {
    return j0 >= last_end || (j0 + n <= first_begin && j0 >= s.sinks);
  }
  __device__ __forceinline__ bool all(const Sight& s, int j0, int n) const {
    return j0 + n <= first_end && (j0 >= last_begin || j0 + n <= s.sinks);
  }
  // Of the sums of keys from j0 on, those of keys that the row does not see become `otherwise`.
  template <int BLOCKS>
  __device__ __forceinline__ void hide(const Sight& s, int j0, f32x16 (&p)[BLOCKS], float otherwise) const {
    if (j0 >= s.sinks) {  // one stretch of keys
      const uint32_t from = j0 + key_of(0) - begin, span = max(end - begin, 0);
#pragma unroll
      for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) p[kb][i] = from + (kb * 32 + 8 * (i / 4) + i % 4) < span ? p[kb][i] : otherwise;
    } else {
#pragma unroll
      for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = j0 + kb * 32 + key_of(i);
          p[kb][i] = j < end && (j >= begin || j < s.sinks) ? p[kb][i] : otherwise;
        }
    }
  }
};

// Waves on a SIMD: two where their registers allow it.
template <typename T, int DP, bool DIRECT>
constexpr int kAtOnce = DIRECT && sizeof(T) * DP <= 256 ? 2 : 1;

// ---- plans ----------------------------------------------------------------------------------------------------------------
// Jobs of the backward by keys.
struct KeyJobs {
  int tiles, parts;                // of kRows keys; parts of a tile's blocks of queries
  int sink_tiles;                  // tiles that have first keys whose sums go on
  int strips, further_parts;       // of 32 first keys
  int64_t further_jobs;
  float *partial, *further;        // [job][2][kRows][pitch] (one part: of the sink tiles, for the strips' keys), [job][4][2][32][pitch]
};

int64_t up(int64_t n, int64_t by) { return (n + by - 1) / by; }
int64_t pitch_of(const WindowCall& c) { return up(c.D, 4) * 4; }

// Up to 32 rows for a key head: the kernel for few, of rows whose keys, values and sums a wave can hold; bfloat16 of more than 192 elements spills 124 bytes a
// lane there.  One token over 4096 keys of 256, 48 sequences of 32 / 8 heads: 358 us, 387 by the kernel for many; 16 of 8 / 8 heads 136 and 114.
bool few(const WindowCall& c, tempo_dtype dt) {
  return c.Sq * (c.heads / c.kv_heads) <= 32 && c.D <= (dt == TEMPO_F32 ? 128 : 256);
}
// Parts of the keys of a forward: enough workgroups for the chip where there are few rows, of at least two tiles of keys each.
int forward_splits(const WindowCall& c, tempo_dtype dt) {
  const int64_t rows = c.Sq * (c.heads / c.kv_heads), blocks = up(rows, kRows) * c.B * c.kv_heads;
  const int64_t span = std::min(c.Sk, c.window + c.Sq) + std::min(c.sinks, c.Sk), most = std::max<int64_t>(up(span, 128), 1);
  if (blocks > 0 && few(c, dt)) {
    const int64_t waves = c.D * (dt == TEMPO_F32 ? 4 : 2) <= 256 ? 8 : 4;
    return static_cast<int>(std::max<int64_t>(1, std::min({up(span, 32 * waves * 4), up(3 * compute_units(), blocks), int64_t{64}})));
  }
  if (blocks == 0 || blocks >= compute_units()) return 1;
  return static_cast<int>(std::min<int64_t>(std::min<int64_t>(most, 64), up(2 * compute_units(), blocks)));
}
struct KeyPlan {
  KeyJobs jobs;
  int64_t blocks, partial_floats, further_floats;
};
KeyPlan key_plan(const WindowCall& c) {
  KeyPlan p{};
  const int64_t group = c.heads / c.kv_heads, bk = c.B * c.kv_heads, tiles = up(c.Sk, kRows), cus = compute_units();
  const int64_t span = up(std::min(c.Sq, c.window + kRows), 32) * group, all = up(c.Sq, 32) * group;  // blocks of queries
  // Workgroups for each compute unit: 1.5, so that the parts' sums cost less than an even end is worth.
  const int64_t want = up(3 * cus / 2, std::max<int64_t>(bk * tiles, 1));
  p.jobs.tiles = static_cast<int>(tiles);
  p.jobs.parts = static_cast<int>(std::max<int64_t>(1, std::min({want, up(span, 4), int64_t{64}})));
  // Without positions of the caller's the last query stands at the last key: none is further on than a window that holds all keys.
  if (c.sinks > 0 && c.Sq > 0 && (c.query_start || c.window < c.Sk)) {
    p.jobs.strips = static_cast<int>(up(std::min(c.sinks, c.Sk), 32));
    p.jobs.sink_tiles = static_cast<int>(up(p.jobs.strips, kWaves));
    const int64_t part = 2 * std::max<int64_t>(up(span, p.jobs.parts), 1);  // two of a wave's blocks for one of the others'
    p.jobs.further_parts = static_cast<int>(std::max<int64_t>(1, std::min(up(all, part), up(4 * cus, std::max<int64_t>(bk * p.jobs.strips, 1)))));
  }
  p.jobs.further_jobs = bk * p.jobs.strips * p.jobs.further_parts;
  p.blocks = p.jobs.further_jobs + bk * tiles * p.jobs.parts;
  p.partial_floats = bk * (p.jobs.parts > 1 ? tiles * p.jobs.parts : p.jobs.sink_tiles) * 2 * kRows * pitch_of(c);
  p.further_floats = p.jobs.further_jobs * kWaves * 2 * 32 * pitch_of(c);
  return p;
}

Heads heads_of(const tempo_attn_heads* h) { return h ? Heads{h->p, h->batch, h->token, h->head} : Heads{}; }
Attn attn_of(const WindowCall& c) {
  Attn a{};
  a.q = heads_of(c.q), a.k = heads_of(c.k), a.v = heads_of(c.v), a.out = heads_of(c.out);
  a.dout = heads_of(c.dout), a.dq = heads_of(c.dq), a.dk = heads_of(c.dk), a.dv = heads_of(c.dv);
  a.lse = c.lse;
  a.key_len = c.key_len, a.query_start = c.query_start;
  a.Sq = static_cast<int>(c.Sq), a.Sk = static_cast<int>(c.Sk), a.heads = static_cast<int>(c.heads), a.kv_heads = static_cast<int>(c.kv_heads);
  a.group = a.heads / a.kv_heads;
  a.rows = a.Sq * a.group;
  a.D = static_cast<int>(c.D);
  a.pitch = static_cast<int>(pitch_of(c));
  a.by_group = FastDiv(static_cast<uint32_t>(a.group));
  a.window = c.window;
  a.sinks = static_cast<int>(std::min<int64_t>(c.sinks, c.Sk));
  a.scale = c.scale;
  a.c = c.scale * kLog2e;
  a.tiles = static_cast<int>(up(a.rows, kRows));
  a.splits = 1;
  return a;
}

// Kernels of each width: with rows of 192 elements in those of 256, 2 x 1000 tokens of 8 / 2 heads, window 300, bfloat16 backward take 269 us (138 in
// their own), float32 768 (457), 16 tokens over 4096 keys of 32 / 8 heads 163 (82).
template <typename F>
tempo_status with_width(int64_t D, F&& f) {
  if (D <= 64) return f(std::integral_constant<int, 64>{});
  if (D <= 96) return f(std::integral_constant<int, 96>{});
  if (D <= 128) return f(std::integral_constant<int, 128>{});
  if (D <= 192) return f(std::integral_constant<int, 192>{});
  return f(std::integral_constant<int, 256>{});
}
template <typename F>
tempo_status with_type(tempo_dtype dt, F&& f) {
  return dt == TEMPO_F32 ? f(float{}) : f(bf16_t{});
}
// Whether rows of all of these can go to LDS without registers.
bool direct(const WindowCall& c, tempo_dtype dt, std::initializer_list<const tempo_attn_heads*> of) {
  const int64_t size = dt == TEMPO_F32 ? 4 : 2, piece = 16 / size;
  if (c.D % piece != 0) return false;
  for (const tempo_attn_heads* h : of)
    if (reinterpret_cast<uintptr_t>(h->p) % 16 != 0 || h->batch % piece != 0 || h->token % piece != 0 || h->head % piece != 0 ||
        h->token * size > INT32_MAX / 64)
      return false;
  return true;
}
template <typename F>
tempo_status either(bool which, F&& f) {
  return which ? f(std::true_type{}) : f(std::false_type{});
}
template <typename K, typename... Args>
tempo_status launch(K kernel, int64_t blocks, hipStream_t st, const Args&... args) {
  if (blocks == 0) return TEMPO_OK;
  hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, st, args...);
  return launch_status();
}

}  // namespace
}  // namespace tempo

#endif  // TEMPO_WINDOW_ATTN_H_
