// Attention over whole prompts and its gradients.
//
//   forward   S = scale Q K^T,  O = softmax(S) V   one pass over the keys with a running maximum and sum for each row
//   backward  P = exp(S - lse),  dV = P^T dO,  dS = P (dO V^T - delta),  dQ = scale dS K,  dK = scale dS^T Q,
//             delta = dO . O for each row.
//
// The backward pass is two kernels: one whose workgroups own queries (dQ) and one whose workgroups own keys (dK, dV, over all
// query heads of a group).  They compute S and dO V^T twice, seven products instead of five, and need no sums between workgroups: no
// atomics, the same bits from run to run.
//
// A workgroup is four waves.  What it owns (16 or 32 rows a wave) stays in registers as matrix operands; what it walks over
// goes through the LDS in tiles, the next one on its way while one is multiplied.  A tile is kept once, as rows; its
// transposed operands come from the LDS's transposing reads (16-bit types).  Rows in the LDS are
// whole multiples of 128 bytes, their 16-byte pieces exchanged by the row's number so that both kinds of reads
// reach all banks (`place`).
#pragma once

#include "squant_att.h"

namespace squant {
namespace att {

struct PromptArgs {
  Strided q, k, v, o;     // o: the output, or in a backward pass its gradient's
  Strided d_o, dq, dk, dv;
  float* lse;             // [heads][q rows]
  float* delta;           // the same
  Packed queries, keys;
  int32_t heads, kv_heads, group, dim;
  int32_t causal;
  float scale, scale2;    // scale2: times log2(e), never 0 (a hidden score's minus infinity stays one)
};

template <class T, int DP> struct TileOf {
  static constexpr int kPiece = 16 / (int)sizeof(T);                     // elements of 16 bytes
  static constexpr int kPieces = DP / kPiece;                            // of a row
  static constexpr int kRowBytes = (DP * (int)sizeof(T) + 127) / 128 * 128;
  // Byte address of piece c of row r.  Eight rows' same piece lie in eight different 16-byte columns of 128 bytes, four
  // rows' same pair of pieces in four different 32-byte columns.
  static __device__ __forceinline__ int place(int r, int c) {
    return r * kRowBytes + ((c ^ (((r & 3) << 1) | ((r >> 2) & 1))) << 4);
  }
};

// A tile of ROWS rows on its way from memory: pieces behind `count` rows or `dim` elements are zeros.
template <class T, int DP, int ROWS> struct Staged {
  typedef TileOf<T, DP> TL;
  static constexpr int kEach = ROWS * TL::kPieces / kThreads;
  static_assert(ROWS * TL::kPieces % kThreads == 0, "");
  uint4v piece[kEach];
  __device__ __forceinline__ void load(const Strided& s, int64_t row0, int head, int count, int dim) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = (int)threadIdx.x + i * kThreads, r = at / TL::kPieces, c = at % TL::kPieces;
      piece[i] = uint4v{0, 0, 0, 0};
      if (r < count && c * TL::kPiece < dim) piece[i] = load_any<uint4v>(element<T>(s, row0 + r, head) + c * TL::kPiece);
    }
  }
  __device__ __forceinline__ void store(char* tile) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = (int)threadIdx.x + i * kThreads;
      *reinterpret_cast<uint4v*>(tile + TL::place(at / TL::kPieces, at % TL::kPieces)) = piece[i];
    }
  }
  // Whether some element is an infinity or NaN.
  __device__ __forceinline__ bool odd() const {
    uint32_t top = 0, high = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (sizeof(T) == 4) {
          top = max(top, piece[i][w] & 0x7fffffffu);
        } else {
          top = max(top, piece[i][w] & 0x7fffu);
          high = max(high, piece[i][w] & 0x7fff0000u);
        }
      }
    if constexpr (sizeof(T) == 4) return top >= 0x7f800000u;
    constexpr uint32_t first = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
    return top >= first || high >= first << 16;
  }
};

// Operand rows r0 .. r0 + 15 of a tile, contraction elements 32 ks .. 32 ks + 31 of the row.
template <class T, int DP> __device__ __forceinline__ typename MatrixOf<T>::type::frag row_operand(const char* tile, int r0, int ks) {
  typedef TileOf<T, DP> TL;
  typedef typename MatrixOf<T>::type::frag frag;
  const int lane = (int)threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  if constexpr (sizeof(T) == 2) {
    return __builtin_bit_cast(frag, *reinterpret_cast<const uint4v*>(tile + TL::place(r0 + n, 4 * ks + g)));
  } else {
    const float4v a = *reinterpret_cast<const float4v*>(tile + TL::place(r0 + n, 8 * ks + 2 * g));
    const float4v b = *reinterpret_cast<const float4v*>(tile + TL::place(r0 + n, 8 * ks + 2 * g + 1));
    return frag{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
}

// Operand rows = elements 16 f .. 16 f + 15 of a tile's rows, contraction over its rows r0 .. r0 + 31 in the order of two
// results side by side.
template <class T, int DP> __device__ __forceinline__ typename MatrixOf<T>::type::frag turned_operand(const char* tile, int r0, int f) {
  typedef TileOf<T, DP> TL;
  typedef typename MatrixOf<T>::type::frag frag;
  const int lane = (int)threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  if constexpr (sizeof(T) == 2) {
    typedef short short4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4v* lds_t;
    // lanes 4 r .. 4 r + 3 of sixteen name the 16 elements of row r; lane n gets element n of the four rows
    const int r = r0 + 4 * g + (n >> 2), c = 2 * f + ((n & 3) >> 1), in = (n & 1) * 8;
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(tile + TL::place(r, c) + in));
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(tile + TL::place(r + 16, c) + in));
    typedef short short8v __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(frag, short8v{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
  } else {
    frag o;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      o[j] = *reinterpret_cast<const float*>(tile + TL::place(r0 + 4 * g + (j & 3) + 16 * (j >> 2), 4 * f + (n >> 2)) + (n & 3) * 4);
    return o;
  }
}

// Two results side by side, rounded to the element type: the operand of the next product.
template <class T> __device__ __forceinline__ typename MatrixOf<T>::type::frag as_operand(const float4v& a, const float4v& b) {
  typename MatrixOf<T>::type::frag o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = (T)a[i], o[4 + i] = (T)b[i];
  return o;
}

// Operand columns from memory: 8 elements a lane from row `row` on; zeros past `dim` or where the row is none.
template <class T, int KS>
__device__ __forceinline__ void own_operand(typename MatrixOf<T>::type::frag (&o)[KS], const Strided& s, int64_t row, int head, bool live, int dim) {
  typedef typename MatrixOf<T>::type::frag frag;
  const int g = ((int)threadIdx.x & 63) >> 4;
  const T* p = element<T>(s, row, head) + 8 * g;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    o[ks] = frag{};
    if (live && 32 * ks + 8 * g < dim) o[ks] = load_any<frag>(p + 32 * ks);
  }
}

// What a lane holds of a finished column: elements 16 f + 4 g + i of a row.
template <class T, int F>
__device__ __forceinline__ void store_column(const Strided& s, int64_t row, int head, int dim, const float4v (&acc)[F], float by) {
  const int g = ((int)threadIdx.x & 63) >> 4;
  T* p = element<T>(s, row, head) + 4 * g;
#pragma unroll
  for (int f = 0; f < F; ++f) {
    if (16 * f + 4 * g >= dim) continue;
    struct Four { T v[4]; };
    Four o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = (T)(acc[f][i] * by);
    store_any(p + 16 * f, o);
  }
}

// Weights of binary16 calls are held times 2^14, so that small ones keep their bits.
template <class T> constexpr float weight_unit() { return __is_same(T, _Float16) ? 14.0f : 0.0f; }

template <class T, int DP, int QT, int BK, int WAVES_EU>
__global__ __launch_bounds__(kThreads, WAVES_EU) void prompt_forward(PromptArgs a) {
  typedef typename MatrixOf<T>::type M;
  typedef typename M::frag frag;
  typedef TileOf<T, DP> TL;
  constexpr int KS = DP / 32, F = DP / 16, TT = BK / 16, kRows = 64 * QT, kTile = BK * TL::kRowBytes;
  extern __shared__ __attribute__((aligned(128))) char tiles[];  // [2][keys, values], [2] flags
  int* const odd_flags = reinterpret_cast<int*>(tiles + 4 * kTile);
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int turn = (int)(blockIdx.x % (uint32_t)a.heads), kv_head = turn % a.kv_heads, head = kv_head * a.group + turn / a.kv_heads;
  Tile tile = find_tile(a.queries, blockIdx.x / (uint32_t)a.heads, 1, kRows);
  if (tile.sequence < 0) return;
  // the longest tiles of a causal sequence first
  const int seq = tile.sequence, first = (tile.tiles - 1 - tile.index) * kRows;
  const int rows = a.queries.length(seq), q0 = a.queries.start(seq);
  const int keys = seq < a.queries.count ? a.keys.length(seq) : 0, k0 = a.keys.start(min(seq, a.keys.count));
  const int shift = keys - rows;
  auto sees = [&](int r) { return a.causal ? min(max(r + shift + 1, 0), keys) : keys; };
  const int mine = first + wave * 16 * QT;
  int seen[QT];
  frag q[QT][KS];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = mine + 16 * t + n;
    const bool live = r < rows;
    seen[t] = live ? sees(r) : 0;
    own_operand<T, KS>(q[t], a.q, q0 + (live ? r : 0), head, live, a.dim);
  }
  const int wave_least = mine < rows ? sees(mine) : keys;  // keys that all rows of the wave see
  const int wave_most = mine < rows ? sees(min(mine + 16 * QT, rows) - 1) : 0;
  const int most = sees(min(first + kRows, rows) - 1), least = sees(first);
  const int steps = (most + BK - 1) / BK;

  float4v o[QT][F];
  float largest[QT], sum[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    largest[t] = -kInfinity, sum[t] = 0.0f;
#pragma unroll
    for (int f = 0; f < F; ++f) o[t][f] = float4v{0, 0, 0, 0};
  }
  Staged<T, DP, BK> sk, sv;
  auto put = [&](int j) {
    char* at = tiles + (j & 1) * 2 * kTile;
    sk.store(at);
    sv.store(at + kTile);
    // a value that some row of the workgroup does not see
    if ((j + 1) * BK > least && lanes_where(sv.odd()) && lane == 0) odd_flags[j & 1] = j + 1;
  };
  if (threadIdx.x < 2) odd_flags[threadIdx.x] = 0;
  if (steps > 0) {
    sk.load(a.k, k0, kv_head, keys, a.dim);
    sv.load(a.v, k0, kv_head, keys, a.dim);
  }
  __syncthreads();
  if (steps > 0) put(0);
  __syncthreads();
#pragma unroll 1
  for (int j = 0; j < steps; ++j) {
    if (j + 1 < steps) {
      sk.load(a.k, k0 + (j + 1) * BK, kv_head, keys - (j + 1) * BK, a.dim);
      sv.load(a.v, k0 + (j + 1) * BK, kv_head, keys - (j + 1) * BK, a.dim);
    }
    const char* kt = tiles + (j & 1) * 2 * kTile;
    const char* vt = kt + kTile;
    if (j * BK < wave_most) {
      float4v s[TT][QT];
#pragma unroll
      for (int tt = 0; tt < TT; ++tt) {
#pragma unroll
        for (int t = 0; t < QT; ++t) s[tt][t] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const frag k = row_operand<T, DP>(kt, 16 * tt, ks);
#pragma unroll
          for (int t = 0; t < QT; ++t) s[tt][t] = M::mma(k, q[t][ks], s[tt][t]);
        }
      }
      const bool some_hidden = (j + 1) * BK > wave_least;
      if (some_hidden) {
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
          for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (j * BK + 16 * tt + 4 * g + i >= seen[t]) s[tt][t][i] = -kInfinity;
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float m = s[0][t][0];
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) m = fmaxf(m, s[tt][t][i]);
        m = over_groups_max(m) * a.scale2;
        if (lanes_where(m > largest[t])) {
          const float more = fmaxf(m, largest[t]);
          const float shrink = more == -kInfinity ? 1.0f : exp2_fast(largest[t] - more);
          sum[t] *= shrink;
#pragma unroll
          for (int f = 0; f < F; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[t][f][i] *= shrink;
          largest[t] = more;
        }
        const float base = largest[t] == -kInfinity ? 0.0f : weight_unit<T>() - largest[t];
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[tt][t][i] = exp2_fast(__builtin_fmaf(s[tt][t][i], a.scale2, base));
            sum[t] += s[tt][t][i];
          }
      }
      frag p[QT][TT / 2];
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int kk = 0; kk < TT / 2; ++kk) p[t][kk] = as_operand<T>(s[2 * kk][t], s[2 * kk + 1][t]);
      const bool odd = some_hidden && __builtin_amdgcn_readfirstlane(odd_flags[j & 1]) == j + 1;
      if (!odd) {
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
          for (int kk = 0; kk < TT / 2; ++kk) {
            const frag v = turned_operand<T, DP>(vt, 32 * kk, f);
#pragma unroll
            for (int t = 0; t < QT; ++t) o[t][f] = M::mma(v, p[t][kk], o[t][f]);
          }
      } else {
        // a weight of 0 would not keep an infinity or NaN out: token by token, rows that do not see it left out
#pragma unroll
        for (int kk = 0; kk < TT / 2; ++kk)
#pragma unroll 1
          for (int token = 0; token < 32; ++token)
#pragma unroll
            for (int f = 0; f < F; ++f) {
              frag v = turned_operand<T, DP>(vt, 32 * kk, f);
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (4 * g + (e & 3) + 16 * (e >> 2) != token) v[e] = (T)0.0f;
#pragma unroll
              for (int t = 0; t < QT; ++t) {
                const float4v one = M::mma(v, p[t][kk], float4v{0, 0, 0, 0});
                if (j * BK + 32 * kk + token < seen[t]) o[t][f] += one;
              }
            }
      }
    }
    if (j + 1 < steps) put(j + 1);
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = mine + 16 * t + n;
    const float total = over_groups_sum(sum[t]);
    if (r >= rows) continue;
    store_column<T, F>(a.o, q0 + r, head, a.dim, o[t], total == 0.0f ? 0.0f : 1.0f / total);
    if (a.lse && g == 0)
      a.lse[(int64_t)head * a.queries.rows + q0 + r] =
          total == 0.0f ? -kInfinity : (largest[t] - weight_unit<T>() + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

// delta[h][r] = dO . O: 16 lanes a row and head.
template <class T> __global__ __launch_bounds__(kThreads) void prompt_delta(PromptArgs a) {
  const int64_t at = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 16;
  if (at >= (int64_t)a.queries.rows * a.heads) return;
  const int64_t row = at / a.heads;
  const int head = (int)(at - row * a.heads), lane = (int)threadIdx.x & 15;
  float sum = 0.0f;
  for (int d = lane * 8; d < a.dim; d += 128) {
    struct Eight { T v[8]; };
    const Eight x = load_any<Eight>(element<T>(a.o, row, head) + d), y = load_any<Eight>(element<T>(a.d_o, row, head) + d);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf((float)x.v[i], (float)y.v[i], sum);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) a.delta[(int64_t)head * a.queries.rows + row] = sum;
}

// Binary16 gradients: dS is held times 2^e, e running for the wave (a tile with a larger one lowers it, and the sums with it): its
// largest magnitude stays below 2^15, and 2^-39 of the largest so far is still told from 0.
__device__ __forceinline__ int gradient_exponent(uint32_t top) {
  return top == 0 ? 126 : min(14 - ((int)(top >> 23) - 127), 126);
}

// KEYS: the workgroup owns keys and values and walks over queries (dK, dV); otherwise it owns queries and walks over keys (dQ).
// First operands: keys and queries; second: values and the output's gradient.
template <class T, int DP, int OT, int BS, bool KEYS>
__global__ __launch_bounds__(kThreads) void prompt_backward(PromptArgs a) {
  typedef typename MatrixOf<T>::type M;
  typedef typename M::frag frag;
  typedef TileOf<T, DP> TL;
  constexpr int KS = DP / 32, F = DP / 16, TT = BS / 16, kRows = 64 * OT, kTile = BS * TL::kRowBytes;
  extern __shared__ __attribute__((aligned(128))) char tiles[];  // [2][first, second], [2][2][BS] row statistics
  float* const stats = reinterpret_cast<float*>(tiles + 4 * kTile);
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const uint32_t heads = (uint32_t)(KEYS ? a.kv_heads : a.heads);
  const int turn = (int)(blockIdx.x % heads);
  const int kv_head = KEYS ? turn : turn % a.kv_heads, head0 = kv_head * a.group + (KEYS ? 0 : turn / a.kv_heads);
  const Packed& own = KEYS ? a.keys : a.queries;
  const Tile tile = find_tile(own, blockIdx.x / heads, 1, kRows);
  if (tile.sequence < 0) return;
  const int seq = tile.sequence, first = (KEYS ? tile.index : tile.tiles - 1 - tile.index) * kRows;
  const bool real = seq < own.count;
  const int rows = real || !KEYS ? a.queries.length(min(seq, a.queries.count)) : 0, q0 = a.queries.start(min(seq, a.queries.count));
  const int keys = real || KEYS ? a.keys.length(min(seq, a.keys.count)) : 0, k0 = a.keys.start(min(seq, a.keys.count));
  const int own_count = KEYS ? keys : rows, own0 = KEYS ? k0 : q0;
  const int walk_count = KEYS ? (real ? rows : 0) : (real ? keys : 0), walk0 = KEYS ? q0 : k0;
  const int shift = keys - rows;  // query i sees key j if j <= i + shift
  const Strided& own1 = KEYS ? a.k : a.q;
  const Strided& own2 = KEYS ? a.v : a.d_o;
  const Strided& walk1 = KEYS ? a.q : a.k;
  const Strided& walk2 = KEYS ? a.d_o : a.v;

  const int mine = first + wave * 16 * OT;
  frag x1[OT][KS], x2[OT][KS];
  float own_lse[OT], own_delta[OT];
#pragma unroll
  for (int t = 0; t < OT; ++t) {
    const int r = mine + 16 * t + n;
    const bool live = r < own_count;
    const int64_t at = own0 + (live ? r : 0);
    const int head = KEYS ? kv_head : head0;
    own_operand<T, KS>(x1[t], own1, at, head, live, a.dim);
    own_operand<T, KS>(x2[t], own2, at, head, live, a.dim);
    own_lse[t] = own_delta[t] = 0.0f;
    if (!KEYS && live) {
      const float l = a.lse[(int64_t)head0 * a.queries.rows + at];
      own_lse[t] = l == -kInfinity ? kInfinity : l * kLog2E;
      own_delta[t] = a.delta[(int64_t)head0 * a.queries.rows + at];
    }
  }
  float4v acc1[OT][F], acc2[KEYS ? OT : 1][KEYS ? F : 1];
#pragma unroll
  for (int t = 0; t < OT; ++t)
#pragma unroll
    for (int f = 0; f < F; ++f) {
      acc1[t][f] = float4v{0, 0, 0, 0};
      if constexpr (KEYS) acc2[t][f] = float4v{0, 0, 0, 0};
    }
  int ds_e = 126;

  // tiles walked over: keys up to the last that a row of ours sees; queries from the first that sees one of ours
  int from = 0, to = walk_count;
  if (a.causal) {
    if (KEYS) from = min(max(first - shift, 0), walk_count) / BS * BS;
    else to = min(max(min(first + kRows, rows) + shift, 0), walk_count);
  }
  const int per_head = to > from ? (to - from + BS - 1) / BS : 0;
  const int steps = KEYS ? per_head * a.group : per_head;

  Staged<T, DP, BS> s1, s2;
  float row_stat = 0.0f;
  auto load = [&](int j) {
    const int member = KEYS ? j / per_head : 0, at = from + (j - member * per_head) * BS;
    const int head = KEYS ? head0 + member : kv_head;
    s1.load(walk1, walk0 + at, head, walk_count - at, a.dim);
    s2.load(walk2, walk0 + at, head, walk_count - at, a.dim);
    if (KEYS && threadIdx.x < 2 * BS) {
      const int r = at + (int)threadIdx.x % BS;
      row_stat = 0.0f;
      if (r < walk_count) {
        const float* p = (int)threadIdx.x < BS ? a.lse : a.delta;
        row_stat = p[(int64_t)head * a.queries.rows + walk0 + r];
        if ((int)threadIdx.x < BS) row_stat = row_stat == -kInfinity ? kInfinity : row_stat * kLog2E;
      }
    }
  };
  auto put = [&](int j) {
    char* at = tiles + (j & 1) * 2 * kTile;
    s1.store(at);
    s2.store(at + kTile);
    if (KEYS && threadIdx.x < 2 * BS) stats[(j & 1) * 2 * BS + threadIdx.x] = row_stat;
  };
  if (steps > 0) {
    load(0);
    put(0);
  }
  __syncthreads();
#pragma unroll 1
  for (int j = 0; j < steps; ++j) {
    if (j + 1 < steps) load(j + 1);
    const int member = KEYS ? j / per_head : 0, at = from + (j - member * per_head) * BS;
    const char* t1 = tiles + (j & 1) * 2 * kTile;
    const char* t2 = t1 + kTile;
    // scores (base 2) and dO V^T: rows are the tile's, columns ours
    float4v s[TT][OT], d[TT][OT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
#pragma unroll
      for (int t = 0; t < OT; ++t) s[tt][t] = d[tt][t] = float4v{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const frag y1 = row_operand<T, DP>(t1, 16 * tt, ks), y2 = row_operand<T, DP>(t2, 16 * tt, ks);
#pragma unroll
        for (int t = 0; t < OT; ++t) {
          s[tt][t] = M::mma(y1, x1[t][ks], s[tt][t]);
          d[tt][t] = M::mma(y2, x2[t][ks], d[tt][t]);
        }
      }
    }
    bool some_hidden = at + BS > walk_count || mine + 16 * OT > own_count;
    if (a.causal) some_hidden = some_hidden || (KEYS ? mine + 16 * OT - 1 > at + shift : at + BS - 1 > mine + shift);
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
      float4v tile_lse, tile_delta;
      if constexpr (KEYS) {
        tile_lse = *reinterpret_cast<const float4v*>(stats + (j & 1) * 2 * BS + 16 * tt + 4 * g);
        tile_delta = *reinterpret_cast<const float4v*>(stats + (j & 1) * 2 * BS + BS + 16 * tt + 4 * g);
      }
#pragma unroll
      for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lse = KEYS ? tile_lse[i] : own_lse[t], delta = KEYS ? tile_delta[i] : own_delta[t];
          float p = exp2_fast(__builtin_fmaf(s[tt][t][i], a.scale2, weight_unit<T>() - lse));
          float ds = p * (d[tt][t][i] - delta);
          if (some_hidden) {
            const int theirs = at + 16 * tt + 4 * g + i, ours = mine + 16 * t + n;
            const int query = KEYS ? theirs : ours, key = KEYS ? ours : theirs;
            const bool visible = query < rows && key < keys && (!a.causal || key <= query + shift);
            p = visible ? p : 0.0f;
            ds = visible ? ds : 0.0f;
          }
          s[tt][t][i] = p;
          d[tt][t][i] = ds;
        }
    }
    if constexpr (__is_same(T, _Float16)) {
      float top = 0.0f;
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int t = 0; t < OT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(d[tt][t][i]));
      if (lanes_where(top * power_of_two(ds_e) >= 32768.0f)) {
        uint32_t m = magnitude(top);
        m = m < 0x7f800000u ? m : 0u;
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, w));
        const int e = min(ds_e, __builtin_amdgcn_readfirstlane(gradient_exponent(m)));
#pragma unroll
        for (int t = 0; t < OT; ++t)
#pragma unroll
          for (int f = 0; f < F; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc1[t][f][i] = ldexpf(acc1[t][f][i], e - ds_e);
        ds_e = e;
      }
      const float unit = power_of_two(ds_e);
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int t = 0; t < OT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) d[tt][t][i] *= unit;
    }
#pragma unroll
    for (int kk = 0; kk < TT / 2; ++kk) {
      frag ds[OT], p[OT];
#pragma unroll
      for (int t = 0; t < OT; ++t) {
        ds[t] = as_operand<T>(d[2 * kk][t], d[2 * kk + 1][t]);
        if constexpr (KEYS) p[t] = as_operand<T>(s[2 * kk][t], s[2 * kk + 1][t]);
      }
#pragma unroll
      for (int f = 0; f < F; ++f) {
        const frag y1 = turned_operand<T, DP>(t1, 32 * kk, f);
#pragma unroll
        for (int t = 0; t < OT; ++t) acc1[t][f] = M::mma(y1, ds[t], acc1[t][f]);
        if constexpr (KEYS) {
          const frag y2 = turned_operand<T, DP>(t2, 32 * kk, f);
#pragma unroll
          for (int t = 0; t < OT; ++t) acc2[t][f] = M::mma(y2, p[t], acc2[t][f]);
        }
      }
    }
    if (j + 1 < steps) put(j + 1);
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < OT; ++t) {
    const int r = mine + 16 * t + n;
    if (r >= own_count) continue;
    float by = a.scale;
    if constexpr (__is_same(T, _Float16)) {
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc1[t][f][i] = ldexpf(acc1[t][f][i], -ds_e - (int)weight_unit<T>());
    }
    store_column<T, F>(KEYS ? a.dk : a.dq, own0 + r, KEYS ? kv_head : head0, a.dim, acc1[t], by);
    if constexpr (KEYS) store_column<T, F>(a.dv, own0 + r, kv_head, a.dim, acc2[t], __is_same(T, _Float16) ? 0.00006103515625f : 1.0f);
  }
}

// Rows a wave owns and rows of a tile, by type and (padded) head size: what fits registers and LDS.
struct PromptShape {
  int rows;       // of a workgroup
  int walked;     // of a tile
  size_t lds;
};
typedef void (*prompt_t)(PromptArgs);
struct PromptKernel {
  prompt_t run;
  PromptShape shape;
};

template <class T, int DP, int QT, int BK, int WAVES_EU> PromptKernel forward_of() {
  return {prompt_forward<T, DP, QT, BK, WAVES_EU>, {64 * QT, BK, (size_t)4 * BK * TileOf<T, DP>::kRowBytes + 16}};
}
template <class T, int DP, int OT, int BS, bool KEYS> PromptKernel backward_of() {
  return {prompt_backward<T, DP, OT, BS, KEYS>, {64 * OT, BS, (size_t)4 * BS * TileOf<T, DP>::kRowBytes + 16 * BS}};
}

// By the head's size.
PromptKernel prompt_forward_bf16(int dim);
PromptKernel prompt_forward_f16(int dim);
PromptKernel prompt_forward_f32(int dim);
PromptKernel prompt_keys_bf16(int dim);
PromptKernel prompt_keys_f16(int dim);
PromptKernel prompt_keys_f32(int dim);
PromptKernel prompt_queries_bf16(int dim);
PromptKernel prompt_queries_f16(int dim);
PromptKernel prompt_queries_f32(int dim);
prompt_t prompt_delta_kernel(int type);

template <class T> PromptKernel forward_for(int dim) {
  if constexpr (sizeof(T) == 2) {
    if (dim <= 64) return forward_of<T, 64, 2, 64, 2>();
    if (dim <= 96) return forward_of<T, 96, 2, 64, 2>();
    if (dim <= 128) return forward_of<T, 128, 2, 64, 2>();
    if (dim <= 192) return forward_of<T, 192, 1, 32, 2>();
    return forward_of<T, 256, 1, 32, 2>();
  } else {
    if (dim <= 64) return forward_of<T, 64, 1, 32, 2>();
    if (dim <= 96) return forward_of<T, 96, 1, 32, 2>();
    if (dim <= 128) return forward_of<T, 128, 1, 32, 2>();
    if (dim <= 192) return forward_of<T, 192, 1, 32, 1>();
    return forward_of<T, 256, 1, 32, 1>();
  }
}
template <class T, bool KEYS> PromptKernel backward_for(int dim) {
  if constexpr (sizeof(T) == 2) {
    if (dim <= 64) return backward_of<T, 64, 2, 32, KEYS>();
    if (dim <= 96) return backward_of<T, 96, 2, 64, KEYS>();
    if (dim <= 128) return backward_of<T, 128, 2, 32, KEYS>();
    if (dim <= 192) return backward_of<T, 192, 1, 32, KEYS>();
    return backward_of<T, 256, 1, 32, KEYS>();
  } else {
    if (dim <= 64) return backward_of<T, 64, 1, 32, KEYS>();
    if (dim <= 96) return backward_of<T, 96, 1, 32, KEYS>();
    if (dim <= 128) return backward_of<T, 128, 1, 32, KEYS>();
    if (dim <= 192) return backward_of<T, 192, 1, 32, KEYS>();
    return backward_of<T, 256, 1, 32, KEYS>();
  }
}

}  // namespace att
}  // namespace squant
