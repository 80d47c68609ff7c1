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
#include <algorithm>
#include <type_traits>

#include "launch_split.h"
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
  int window, sinks;
  float scale, c;  // c: scale log2(e)
  int tiles, splits;
  int pitch;                     // floats of a row of sums in the workspace: D up to whole pieces
  float *partial, *partial_lse;  // splits > 1: [splits, B kv_heads, rows, pitch] and [splits, B kv_heads, rows], of base 2
};

// Which keys the queries of a sequence see.
struct Sight {
  int64_t start;
  int keys, window, sinks;
  __device__ __forceinline__ Sight(const Attn& a, int b) : window(a.window) {
    keys = a.key_len ? min(max(a.key_len[b], 0), a.Sk) : a.Sk;
    start = a.query_start ? a.query_start[b] : int64_t{a.Sk} - a.Sq;
    sinks = min(a.sinks, keys);
  }
  // keys [begin, end) and those below min(sinks, end)
  __device__ __forceinline__ int end(int i) const {
    const int64_t e = start + i + 1;
    return e <= 0 ? 0 : e < keys ? static_cast<int>(e) : keys;
  }
  __device__ __forceinline__ int begin(int i) const {
    const int64_t e = start + i + 1 - window;
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
// Four neighbouring floats of a row of D; zeros behind its end.
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

// ---- forward ------------------------------------------------------------------------------------------------------------
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
constexpr int kAtOnce = DIRECT && sizeof(T) * DP <= 256 ? 2 : 1;
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
struct KeyJobs {
  int tiles, parts;                // of kRows keys; parts of a tile's blocks of queries
  int sink_tiles;                  // tiles that have first keys whose sums go on
  int strips, further_parts;       // of 32 first keys
  int64_t further_jobs;
  float *partial, *further;        // [job][2][kRows][pitch] (one part: of the sink tiles, for the strips' keys), [job][4][2][32][pitch]
};
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
    const int64_t i = j + int64_t{s.window} - s.start;
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

// ---- plans ----------------------------------------------------------------------------------------------------------------
int64_t up(int64_t n, int64_t by) { return (n + by - 1) / by; }
int64_t pitch_of(const WindowCall& c) { return up(c.D, 4) * 4; }

// Up to 32 rows for a key head: the kernel for few, where a wave's registers hold what it needs.
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
  a.window = static_cast<int>(std::min<int64_t>(c.window, INT32_MAX));
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
