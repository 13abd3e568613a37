// Attention over whole prompts and its gradients.
//
//   forward   S = scale Q K^T,  O = softmax(S) V   one pass over the keys with a running maximum and sum for each row
//   backward  P = exp(S - lse),  dV = P^T dO,  dS = P (dO V^T - delta),  dQ = scale dS K,  dK = scale dS^T Q,
//             delta = dO . O for each row.
//
// The backward pass is two kernels: one whose workgroups own queries (dQ) and one whose workgroups own keys (dK, dV, over all
// query heads of a group).  They compute S and dO V^T twice, seven products instead of five (16-bit types eight: P K beside dS K, for
// delta), and need no sums between workgroups: no atomics, the same bits from run to run.
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
  int32_t by_length;      // the order of tiles
  float scale, scale2;    // scale2: times log2(e), never 0 (a hidden score's minus infinity stays one)
  // walks that are cut into `splits` (the grid's y): their sums, [splits][rows][heads][1 or 2][dim], and, forward, the rows' largest
  // scores (base 2) and sums of weights, [splits][rows][heads]
  int32_t splits;
  float* partial;
  float2* stats;
};

template <class T, int DP> struct TileOf {
  static constexpr int kPiece = 16 / (int)sizeof(T);                     // elements of 16 bytes
  static constexpr int kPieces = DP / kPiece;                            // of a row
  static constexpr int kRowBytes = (DP * (int)sizeof(T) + 127) / 128 * 128;
  // Byte address of piece c of row r.  The LDS serves 256 bytes at once: 16 rows' same piece (operands of rows), or 8 rows' same
  // pair of pieces (transposing reads), lie in different columns of 256 bytes.
  static __device__ __forceinline__ int turn(int r) {
    return kRowBytes % 256 == 0 ? ((r & 7) << 1) ^ (((r >> 3) & 1) * 9) : (r & 6) ^ (((r >> 3) & 1) * 5);
  }
  static __device__ __forceinline__ int place(int r, int c) { return r * kRowBytes + ((c ^ turn(r)) << 4); }
};

constexpr bool keeps_offsets(int dim) { return dim < 256; }

// Tiles of ROWS rows on their way from memory to the LDS.  DIRECT: without passing through registers, which takes rows at
// multiples of 16 bytes; otherwise by registers.  A row past the last is the last one again, a piece past the head's elements the
// first one: both meet zeros or are hidden.  Bytes of the tile are dealt to lanes in their order, 16 each.
template <class T, int DP, int ROWS, int WAVES, bool DIRECT> struct Loader {
  typedef TileOf<T, DP> TL;
  static constexpr int kBytes = ROWS * TL::kRowBytes;
  static constexpr int kEach = kBytes / (WAVES * 1024);
  static_assert(kBytes % (WAVES * 1024) == 0, "");
  uint32_t offset[kEach];  // of full tiles, bytes from the tile's first row
  uint4v piece[DIRECT ? 1 : kEach];

  static __device__ __forceinline__ int first(int i) { return (__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * kEach + i) * 1024; }
  static __device__ __forceinline__ int position(int i) { return first(i) + ((int)threadIdx.x & 63) * 16; }
  static __device__ __forceinline__ uint32_t offset_of(int i, uint32_t row_bytes, int last, int dim) {
    const int at = position(i), r = at / TL::kRowBytes;
    int c = (at % TL::kRowBytes >> 4) ^ TL::turn(r);
    if (c * TL::kPiece >= dim) c = 0;
    return (uint32_t)min(r, last) * row_bytes + (uint32_t)(c << 4);
  }
  __device__ __forceinline__ void begin(uint32_t row_bytes, int dim) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) offset[i] = offset_of(i, row_bytes, ROWS, dim);
  }
  template <class OFFSET> __device__ __forceinline__ void take(const char* from, char* tile, OFFSET off) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if constexpr (DIRECT)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + off(i)),
                                         (__attribute__((address_space(3))) void*)(tile + first(i)), 16, 0, 0);
      else
        piece[i] = load_any<uint4v>(from + off(i));
    }
  }
  // `from`: the tile's first row; `count`: rows from there on, at least one.  KEPT: full tiles by the offsets kept.  The loops of
  // hidden steps, and all of the largest heads, make them anew: they have no registers for them, and reading them back from memory waits
  // for what is on its way, each time (forward of 34 sequences of 300 tokens, 32 heads of 128: 131 us, 103; of 8192 tokens, 16
  // heads of 256: 697, 580).  Heads of 192 keep them (488, 512 without).
  template <bool KEPT> __device__ __forceinline__ void issue(const char* from, char* tile, int count, uint32_t row_bytes, int dim, Constant<KEPT>) {
    if (KEPT && count >= ROWS) take(from, tile, [&](int i) { return offset[i]; });
    else take(from, tile, [&](int i) { return offset_of(i, row_bytes, min(count, ROWS) - 1, dim); });
  }
  // Before the barrier behind which the tile is read.
  __device__ __forceinline__ void land(char* tile) const {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) *reinterpret_cast<uint4v*>(tile + position(i)) = piece[i];
    }
  }
  // Whether this lane's part of a tile has an infinity or NaN.
  static __device__ __forceinline__ bool odd(const char* tile) {
    uint32_t top = 0, high = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint4v v = *reinterpret_cast<const uint4v*>(tile + position(i));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (sizeof(T) == 4) {
          top = max(top, v[w] & 0x7fffffffu);
        } else {
          top = max(top, v[w] & 0x7fffu);
          high = max(high, v[w] & 0x7fff0000u);
        }
      }
    }
    if constexpr (sizeof(T) == 4) return top >= 0x7f800000u;
    constexpr uint32_t first = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
    return top >= first || high >= first << 16;
  }
};
__device__ __forceinline__ void tiles_are_here() { __builtin_amdgcn_s_waitcnt(0x0F70); }  // vmcnt(0)

// Where a lane reads operands, in bytes from a tile's beginning.  Pieces are exchanged within runs of 8 or 16, so what an
// operand's place adds to a lane's is one exclusive or and an offset of the instruction.
template <class T, int DP> struct Lanes {
  typedef TileOf<T, DP> TL;
  static constexpr int kRun = TL::kRowBytes % 256 == 0 ? 15 : 7;
  int row, turned;
  __device__ __forceinline__ Lanes() {
    const int lane = (int)threadIdx.x & 63, n = lane & 15, g = lane >> 4, r = 4 * g + (n >> 2);
    row = n * TL::kRowBytes + (((sizeof(T) == 2 ? g : 2 * g) ^ TL::turn(n)) << 4);
    turned = sizeof(T) == 2 ? r * TL::kRowBytes + ((((n & 3) >> 1) ^ TL::turn(r)) << 4) + (n & 1) * 8 : 0;
  }
  static __device__ __forceinline__ int piece(int at, int c) { return (at ^ ((c & kRun) << 4)) + ((c & ~kRun) << 4); }
};

// Operand rows r0 .. r0 + 15 of a tile, contraction elements 32 ks .. 32 ks + 31 of the row.  `at`: the lane's `row` and the tile.
template <class T, int DP>
__device__ __forceinline__ typename MatrixOf<T>::type::frag row_operand(const char* tiles, int at, int r0, int ks) {
  typedef Lanes<T, DP> L;
  typedef typename MatrixOf<T>::type::frag frag;
  const int o = r0 * L::TL::kRowBytes;
  if constexpr (sizeof(T) == 2) {
    return __builtin_bit_cast(frag, *reinterpret_cast<const uint4v*>(tiles + L::piece(at, 4 * ks) + o));
  } else {
    const float4v a = *reinterpret_cast<const float4v*>(tiles + L::piece(at, 8 * ks) + o);
    const float4v b = *reinterpret_cast<const float4v*>(tiles + L::piece(at, 8 * ks + 1) + o);
    return frag{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
}

// Operand rows = elements 16 f .. 16 f + 15 of a tile's rows, contraction over its rows r0 .. r0 + 31 in the order of two
// results side by side.  `at`: the lane's `turned` and the tile.
template <class T, int DP>
__device__ __forceinline__ typename MatrixOf<T>::type::frag turned_operand(const char* tiles, int at, int r0, int f) {
  typedef Lanes<T, DP> L;
  typedef typename L::TL TL;
  typedef typename MatrixOf<T>::type::frag frag;
  if constexpr (sizeof(T) == 2) {
    typedef short short4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4v* lds_t;
    // lanes 4 r .. 4 r + 3 of sixteen name the 16 elements of row r; lane n gets element n of the four rows
    const char* p = tiles + L::piece(at, 2 * f) + r0 * TL::kRowBytes;
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)p);
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(p + 16 * TL::kRowBytes));
    typedef short short8v __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(frag, short8v{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
  } else {
    const int lane = (int)threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    frag o;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      o[j] = *reinterpret_cast<const float*>(tiles + at + TL::place(r0 + 4 * g + (j & 3) + 16 * (j >> 2), 4 * f + (n >> 2)) + (n & 3) * 4);
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

// Weights of binary16 calls are held times 2^7, so that small ones keep their bits.
template <class T> constexpr float weight_unit() { return __is_same(T, _Float16) ? 7.0f : 0.0f; }

// Asks the compiler to keep 8 reads from the LDS ahead of a step's matrix instructions: FIRST reads with EACH of them behind every
// read, then SECOND with EACH behind every SECOND_STEP.  Left to itself it reads two operands and waits for them (dK and dV of
// 10239 tokens, 32 heads of 128: 720 us, 612 with this).
template <int FIRST, int SECOND, int EACH, int SECOND_STEP> __device__ __forceinline__ void interleave() {
  constexpr int kAhead = 8 < FIRST ? 8 : FIRST, kRead = 0x100, kMatrix = 0x008;
  __builtin_amdgcn_sched_group_barrier(kRead, kAhead, 0);
#pragma unroll
  for (int i = 0; i < FIRST - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMatrix, EACH, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
  }
#pragma unroll
  for (int i = 0; i < SECOND / SECOND_STEP; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMatrix, EACH, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, SECOND_STEP, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kMatrix, kAhead * EACH, 0);
}

// A row's running maximum (base 2) may be passed by this much before sums are scaled down to a new one: weights, held times
// 2^forward_unit, stay below 1 (binary16: 2^15), so that sums of values leave binary32 no sooner than with weights of at most 1.  Without it most steps of a long sequence have a row of the wave's 32 whose maximum moves.
constexpr float kSlack = 8.0f;
template <class T> constexpr float forward_unit() { return __is_same(T, _Float16) ? weight_unit<T>() : -kSlack; }
template <class T> constexpr float without_unit() { return __is_same(T, _Float16) ? 0x1p-7f : 0x1p8f; }

// The tile of a workgroup, and the rows that its sequence walks over.
//
// Where there are more workgroups than run at once, sequences with longer walks come first (and, `by_tile`, tiles with longer ones over all sequences):
// what is left for the end is short, and the compute units end together.  10239 tokens in seven causal sequences of 261
// to 4096, the second longest in the fifth place, 32 heads of 128 on 8: forward 322 us in their own order, 301; dK and dV 632, 569
// (its walks are 64 tiles times four heads, and few).  Forward takes whole sequences: tile by tile, ten of 1024 tokens, which
// all begin and end together then, took 158 us, 148 otherwise.
// With T a tile's rows, tile i of a sequence (the first being its longest walk) is on level
//   by_tile: max(0, min(ceil(walked / T), its tiles - i)),  else ceil(walked / T),
// its walk's length in tiles.  A lane for each sequence knows how many of its tiles lie above a level; the level at which they
// are more than `id` is searched by halves.

// Workgroups that count as run at once: two a compute unit, as heads of 128 have them.  Heads of 64 run three or four, 192 and 256 in
// binary32 one; plans that knew that have not been measured.
constexpr int kRunAtOnce = 512;
// Where piece i of a walk's steps (less than 2^27) begins.
__device__ __forceinline__ int piece_of(int steps, uint32_t i, int splits) { return (int)((uint32_t)steps * i / (uint32_t)splits); }

struct PromptTile {
  int sequence;  // -1: this tile is no one's
  int index, tiles;
  int start, length;  // its sequence's rows
  int walk_start, walk_length;
};
// Sums over the lanes up to each, by moves within the vector registers: within 16 lanes, then of those before.
__device__ __forceinline__ int up_to_lane(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}
__device__ __forceinline__ int over_lanes_sum(int v) { return __builtin_amdgcn_readlane(up_to_lane(v), 63); }

__device__ __forceinline__ PromptTile find_walk(const Packed& own, const Packed& walk, bool by_length, bool by_tile, int id, int tile) {
  PromptTile t;
  if (!own.starts || own.count >= 63) {
    const Tile f = find_tile(own, id, 1, tile);
    t.sequence = f.sequence;
    if (t.sequence < 0) return t;
    auto one = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    t.index = one(f.index), t.tiles = one(f.tiles), t.start = one(f.start), t.length = one(f.length);
    t.walk_start = one(walk.start(min(t.sequence, walk.count))), t.walk_length = one(t.sequence < own.count ? walk.length(t.sequence) : 0);
    return t;
  }
  const int lane = (int)(threadIdx.x & 63u), here = min(lane, own.count);
  const int own_at = own.starts[here], walk_at = walk.starts[here];
  auto inside = [](const Packed& p, int at) { return min(max(at, 0), p.rows); };
  const int start = inside(own, own_at), walk_start = inside(walk, walk_at);
  // the next lane's
  const int end = __builtin_amdgcn_update_dpp(0, start, 0x130, 0xf, 0xf, false), walk_end = __builtin_amdgcn_update_dpp(0, walk_start, 0x130, 0xf, 0xf, false);
  const bool real = lane < own.count;
  const int length = lane > own.count ? 0 : max((real ? end : own.rows) - start, 0), walk_length = real ? max(walk_end - walk_start, 0) : 0;
  auto in_tiles = [&](int n) { return (int)(((uint32_t)n + (uint32_t)tile - 1) / (uint32_t)tile); };
  const int cap = in_tiles(walk_length);
  t.sequence = -1;
  if (by_length && (by_tile || lanes_where(real && cap != __builtin_amdgcn_readfirstlane(cap)))) {
    const int tiles = in_tiles(length), top = by_tile && real ? tiles : 0x40000000;
    auto above = [&](int level) { return level < 0 ? tiles : cap > level ? min(max(top - level, 0), tiles) : 0; };
    if (id >= over_lanes_sum(tiles)) return t;
    // tiles above `high` are no more than id, those above `low` more
    int low = -1, high = in_tiles(walk.rows);
    while (high - low > 1) {
      const int middle = (high + low) / 2;
      if (over_lanes_sum(above(middle)) <= id) high = middle;
      else low = middle;
    }
    const int before = above(high), at = id - over_lanes_sum(before), upto = up_to_lane(above(high - 1) - before);
    t.sequence = (int)__builtin_ctzll(lanes_where(upto > at));
    t.index = __builtin_amdgcn_readlane(before, t.sequence) + at - (t.sequence ? __builtin_amdgcn_readlane(upto, t.sequence - 1) : 0);
  } else {
    // as find_tile does
    const int place = start / tile + lane;
    t.sequence = __popcll(lanes_where(lane <= own.count && place <= id)) - 1;
    if (t.sequence < 0) return t;
    t.index = id - __builtin_amdgcn_readlane(place, t.sequence);
  }
  t.start = __builtin_amdgcn_readlane(start, t.sequence), t.length = __builtin_amdgcn_readlane(length, t.sequence);
  t.walk_start = __builtin_amdgcn_readlane(walk_start, t.sequence), t.walk_length = __builtin_amdgcn_readlane(walk_length, t.sequence);
  t.index = __builtin_amdgcn_readfirstlane(t.index), t.tiles = __builtin_amdgcn_readfirstlane(in_tiles(t.length));
  if (t.index < 0 || t.index >= t.tiles) t.sequence = -1;
  return t;
}

// One row against keys `from` to `to` - 1 by a wave, the largest score taken off before it is multiplied: for rows with far scores, which are
// seldom.  A lane for each key, then for each element.
template <class T, int DP>
__device__ __forceinline__ void far_row(const PromptArgs& a, int64_t q_row, int head, int kv_head, int64_t k0, int from, int to) {
  constexpr int E = (DP + 63) / 64;
  const int lane = (int)threadIdx.x & 63;
  const T* q = element<T>(a.q, q_row, head);
  auto score = [&](int t) {
    const T* k = element<T>(a.k, k0 + t, kv_head);
    float s = 0.0f;
#pragma unroll 4
    for (int d = 0; d < a.dim; d += 8) {
      float x[8], y[8];
      load8(q + d, x);
      load8(k + d, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x[i], y[i], s);
    }
    return s;
  };
  float top = -kInfinity;
#pragma unroll 1
  for (int t = from + lane; t < to; t += 64) top = fmaxf(top, score(t));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float none = top == -kInfinity ? 0.0f : top;
  float total = 0.0f, sum[E] = {};
#pragma unroll 1
  for (int t0 = from; t0 < to; t0 += 64) {
    const float w = t0 + lane < to ? exp2_fast((score(t0 + lane) - none) * a.scale2) : 0.0f;
    total += w;
    const int count = min(64, to - t0);
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      const T* v = element<T>(a.v, k0 + t0 + i, kv_head);
      const float one = __shfl(w, i);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (lane + 64 * e < a.dim) sum[e] = __builtin_fmaf(one, (float)v[lane + 64 * e], sum[e]);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o);
  const float largest = top * a.scale2;
  if (a.splits > 1) {
    const float unit = 1.0f / without_unit<T>();
    const int64_t at = ((int64_t)blockIdx.y * a.queries.rows + q_row) * a.heads + head;
    if (lane == 0) a.stats[at] = make_float2(largest, total * unit);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (lane + 64 * e < a.dim) a.partial[at * a.dim + lane + 64 * e] = sum[e] * unit;
    return;
  }
  T* o = element<T>(a.o, q_row, head);
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (lane + 64 * e < a.dim) o[lane + 64 * e] = (T)(total == 0.0f ? 0.0f : sum[e] / total);
  if (a.lse && lane == 0) a.lse[(int64_t)head * a.queries.rows + q_row] = total == 0.0f ? -kInfinity : (largest + __builtin_amdgcn_logf(total)) * kLn2;
}

// All rows of a wave.  The arguments and the tile are found anew, from a pointer that the compiler does not know: kept through the loops before,
// they would put others' registers into memory.
template <class T, int DP, int QT, int BK, int WAVES> __device__ __forceinline__ void far_rows() {
  typedef const __attribute__((address_space(4))) PromptArgs* args_t;
  args_t p = (args_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  const PromptArgs& a = *(const PromptArgs*)p;
  constexpr int kRows = 16 * WAVES * QT;
  const int turn = (int)(blockIdx.x % (uint32_t)a.heads), kv_head = turn % a.kv_heads, head = kv_head * a.group + turn / a.kv_heads;
  const PromptTile tile = find_walk(a.queries, a.keys, a.by_length, false, (int)(blockIdx.x / (uint32_t)a.heads), kRows);
  const int first = (tile.tiles - 1 - tile.index) * kRows, rows = tile.length, keys = tile.walk_length;
  auto sees = [&](int r) { return a.causal ? min(max(r + keys - rows + 1, 0), keys) : keys; };
  const int all_steps = (sees(min(first + kRows, rows) - 1) + BK - 1) / BK;
  int begin = 0, steps = all_steps;
  if (a.splits > 1) begin = piece_of(all_steps, blockIdx.y, a.splits), steps = piece_of(all_steps, blockIdx.y + 1, a.splits);
  const int mine = first + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 16 * QT;
#pragma unroll 1
  for (int r = mine; r < min(mine + 16 * QT, rows); ++r)
    far_row<T, DP>(a, tile.start + r, head, kv_head, tile.walk_start, begin * BK, min(sees(r), steps * BK));
}

template <class T, int DP, int QT, int BK, int WAVES, int OCCUPANCY, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, OCCUPANCY) void prompt_forward(PromptArgs a) {
  typedef typename MatrixOf<T>::type M;
  typedef typename M::frag frag;
  typedef TileOf<T, DP> TL;
  typedef Loader<T, DP, BK, WAVES, DIRECT> Load;
  constexpr int KS = DP / 32, F = DP / 16, TT = BK / 16, kRows = 16 * WAVES * QT, kTile = BK * TL::kRowBytes;
  constexpr bool kKept = keeps_offsets(DP);
  extern __shared__ __attribute__((aligned(1024))) char tiles[];  // [2][keys, values], a flag
  int* const odd_flag = reinterpret_cast<int*>(tiles + 4 * kTile);
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int turn = (int)(blockIdx.x % (uint32_t)a.heads), kv_head = turn % a.kv_heads, head = kv_head * a.group + turn / a.kv_heads;
  const PromptTile tile = find_walk(a.queries, a.keys, a.by_length, false, (int)(blockIdx.x / (uint32_t)a.heads), kRows);
  if (tile.sequence < 0) return;
  // the longest tiles of a causal sequence first
  const int first = (tile.tiles - 1 - tile.index) * kRows;
  const int rows = tile.length, q0 = tile.start, keys = tile.walk_length, k0 = tile.walk_start;
  const int shift = keys - rows;
  auto sees = [&](int r) { return a.causal ? min(max(r + shift + 1, 0), keys) : keys; };
  const int mine = first + wave * 16 * QT;
  frag q[QT][KS];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = mine + 16 * t + n;
    const bool live = r < rows;
    own_operand<T, KS>(q[t], a.q, q0 + (live ? r : 0), head, live, a.dim);
  }
  const int wave_most = mine < rows ? sees(min(mine + 16 * QT, rows) - 1) : 0;
  const int most = sees(min(first + kRows, rows) - 1);
  const int all_steps = (most + BK - 1) / BK;
  int begin = 0, steps = all_steps;
  if (a.splits > 1) begin = piece_of(all_steps, blockIdx.y, a.splits), steps = piece_of(all_steps, blockIdx.y + 1, a.splits);
  const int whole = min(first + kRows <= rows ? sees(first) / BK : 0, steps);  // steps of which all rows see all keys

  float4v o[QT][F];
  float largest[QT], sum[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    largest[t] = -kInfinity, sum[t] = 0.0f;
#pragma unroll
    for (int f = 0; f < F; ++f) o[t][f] = float4v{0, 0, 0, 0};
  }
  const uint32_t k_bytes = (uint32_t)a.k.row * sizeof(T), v_bytes = (uint32_t)a.v.row * sizeof(T);
  const char* const k_from = (const char*)element<T>(a.k, k0, kv_head);
  const char* const v_from = (const char*)element<T>(a.v, k0, kv_head);
  Load lk, lv;
  const Lanes<T, DP> at;
  lk.begin(k_bytes, a.dim);
  lv.begin(v_bytes, a.dim);
  auto issue = [&](int j, auto kept) {
    char* at = tiles + (j & 1) * 2 * kTile;
    lk.issue(k_from + (int64_t)j * BK * k_bytes, at, keys - j * BK, k_bytes, a.dim, kept);
    lv.issue(v_from + (int64_t)j * BK * v_bytes, at + kTile, keys - j * BK, v_bytes, a.dim, kept);
  };
  auto land = [&](int j) {
    char* at = tiles + (j & 1) * 2 * kTile;
    lk.land(at);
    lv.land(at + kTile);
    if (DIRECT) tiles_are_here();
  };
  if (steps > begin) {
    issue(begin, Constant<kKept>{});
    land(begin);
  }
  __syncthreads();

  bool far = false;  // whether a row of the wave met far scores
  // Keys from step j on that the lane's row t sees, made anew: kept, they would be put into memory.  Rows past the last hold zeros.
  auto seen_from = [&](int j, int t) {
    const int left = keys - j * BK;
    return a.causal ? min(max(mine + 16 * t + shift + 1 - j * BK + n, -j * BK), left) : left;
  };
  auto step = [&](int j, auto some_hidden) {
    constexpr bool kHidden = decltype(some_hidden)::value;
    const int kt = at.row + (j & 1) * 2 * kTile, vt = at.turned + (j & 1) * 2 * kTile + kTile;
    bool odd = false;
    if constexpr (kHidden) {
      // a weight of 0 would not keep an infinity or NaN of a hidden value out
      if (threadIdx.x == 0) *odd_flag = 0;
      __syncthreads();
      if (lanes_where(Load::odd(tiles + (j & 1) * 2 * kTile + kTile)) && lane == 0) *odd_flag = 1;
      __syncthreads();
      odd = __builtin_amdgcn_readfirstlane(*odd_flag) != 0;
      if (j * BK >= wave_most) return;
    }
    float4v s[TT][QT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
#pragma unroll
      for (int t = 0; t < QT; ++t) s[tt][t] = float4v{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const frag k = row_operand<T, DP>(tiles, kt, 16 * tt, ks);
#pragma unroll
        for (int t = 0; t < QT; ++t) s[tt][t] = M::mma(k, q[t][ks], s[tt][t]);
      }
    }
    if constexpr (kHidden) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const int here = seen_from(j, t) - 4 * g;
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * tt + i >= here) s[tt][t][i] = -kInfinity;
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float m = s[0][t][0];
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, s[tt][t][i]);
      m = over_groups_max(m) * a.scale2;
      if (lanes_where(m > largest[t] + kSlack)) {
        const float more = fmaxf(m, largest[t]);
        const float shrink = more == -kInfinity ? 1.0f : exp2_fast(largest[t] - more);
        sum[t] *= shrink;
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][f][i] *= shrink;
        largest[t] = more;
        far |= far_scores(more);
      }
      const float base = largest[t] == -kInfinity ? 0.0f : forward_unit<T>() - largest[t];
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
    if (!odd) {
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int kk = 0; kk < TT / 2; ++kk) {
          const frag v = turned_operand<T, DP>(tiles, vt, 32 * kk, f);
#pragma unroll
          for (int t = 0; t < QT; ++t) o[t][f] = M::mma(v, p[t][kk], o[t][f]);
        }
    } else {
      // token by token, rows that do not see it left out
#pragma unroll
      for (int kk = 0; kk < TT / 2; ++kk)
#pragma unroll 1
        for (int token = 0; token < 32; ++token)
#pragma unroll
          for (int f = 0; f < F; ++f) {
            frag v = turned_operand<T, DP>(tiles, vt, 32 * kk, f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (4 * g + (e & 3) + 16 * (e >> 2) != token) v[e] = (T)0.0f;
#pragma unroll
            for (int t = 0; t < QT; ++t) {
              const float4v one = M::mma(v, p[t][kk], float4v{0, 0, 0, 0});
              if (32 * kk + token < seen_from(j, t)) o[t][f] += one;
            }
          }
    }
  };
  int j = begin;
#pragma unroll 1
  for (; j < whole; ++j) {
    if (j + 1 < steps) issue(j + 1, Constant<kKept>{});
    step(j, Constant<false>{});
    if (j + 1 < steps) land(j + 1);
    __syncthreads();
  }
#pragma unroll 1
  for (; j < steps; ++j) {
    if (j + 1 < steps) issue(j + 1, Constant<false>{});
    step(j, Constant<true>{});
    if (j + 1 < steps) land(j + 1);
    __syncthreads();
  }
  if (__builtin_expect(far, false)) {
    // whatever that takes: a branch in the loops costs all others 1 to 5 %
    far_rows<T, DP, QT, BK, WAVES>();
    return;
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = mine + 16 * t + n;
    const float total = over_groups_sum(sum[t]);
    if (r >= rows) continue;
    if (a.splits > 1) {
      const int64_t at = ((int64_t)blockIdx.y * a.queries.rows + q0 + r) * a.heads + head;
      if (g == 0) a.stats[at] = make_float2(largest[t], total);
      float* p = a.partial + at * a.dim + 4 * g;
#pragma unroll
      for (int f = 0; f < F; ++f)
        if (16 * f + 4 * g < a.dim) *reinterpret_cast<float4v*>(p + 16 * f) = o[t][f];
      continue;
    }
    store_column<T, F>(a.o, q0 + r, head, a.dim, o[t], total == 0.0f ? 0.0f : 1.0f / total);
    if (a.lse && g == 0)
      a.lse[(int64_t)head * a.queries.rows + q0 + r] =
          total == 0.0f ? -kInfinity : (largest[t] + __builtin_amdgcn_logf(total * without_unit<T>())) * kLn2;
  }
}

// Binary16 gradients: dS is held times 2^e, e running for the wave (a tile with a larger one lowers it, and the sums with it): its
// largest magnitude stays below 2^15, and 2^-39 of the largest so far is still told from 0.
__device__ __forceinline__ int gradient_exponent(uint32_t top) {
  return top == 0 ? 126 : min(14 - ((int)(top >> 23) - 127), 126);
}

// KEYS: the workgroup owns keys and values and walks over queries (dK, dV); otherwise it owns queries and walks over keys (dQ).
// First operands: keys and queries; second: values and the output's gradient.
//
// delta.  The dQ kernel has dO in registers and reads O beside it; the other kernel reads what it leaves (a launch of its own for
// delta took 28 us for 10239 rows of 32 heads of 128).  dS's rows add up to 0.  delta from the output as it was stored is off by its rounding (and the weights' in it), by
// the same for all of a row's keys: with binary16 and bfloat16 as much as everything else together (dQ and dK of 1024
// causal tokens of 128: 2.7e-3 off, 2.3e-3 without it, 1.7e-3 the rounding of the result).  So the dQ kernel adds up its dS in
// binary32 and P K beside dS K: sum dS = delta's error, which it takes off both dQ and delta, before the other kernel reads it.  One
// product more, of operands that are there.
template <class T, int DP, int OT, int BS, int WAVES, int OCCUPANCY, bool KEYS, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, OCCUPANCY) void prompt_backward(PromptArgs a) {
  typedef typename MatrixOf<T>::type M;
  typedef typename M::frag frag;
  typedef TileOf<T, DP> TL;
  typedef Loader<T, DP, BS, WAVES, DIRECT> Load;
  constexpr bool kMend = !KEYS && sizeof(T) == 2, kSecond = KEYS || kMend;
  constexpr int KS = DP / 32, F = DP / 16, TT = BS / 16, kRows = 16 * WAVES * OT, kTile = BS * TL::kRowBytes;
  constexpr bool kKept = keeps_offsets(DP);
  extern __shared__ __attribute__((aligned(1024))) char tiles[];  // [2][first, second], [2][2][BS] row statistics
  float* const stats = reinterpret_cast<float*>(tiles + 4 * kTile);
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const uint32_t heads = (uint32_t)(KEYS ? a.kv_heads : a.heads);
  const int turn = (int)(blockIdx.x % heads);
  const int kv_head = KEYS ? turn : turn % a.kv_heads, head0 = kv_head * a.group + (KEYS ? 0 : turn / a.kv_heads);
  const Packed& own = KEYS ? a.keys : a.queries;
  const PromptTile tile = find_walk(own, KEYS ? a.queries : a.keys, a.by_length, KEYS && a.causal, (int)(blockIdx.x / heads), kRows);
  if (tile.sequence < 0) return;
  const int first = (KEYS ? tile.index : tile.tiles - 1 - tile.index) * kRows;
  const int own_count = tile.length, own0 = tile.start, walk_count = tile.walk_length, walk0 = tile.walk_start;
  const int rows = KEYS ? walk_count : own_count, keys = KEYS ? own_count : walk_count;
  const int shift = keys - rows;  // query i sees key j if j <= i + shift
  const Strided& own1 = KEYS ? a.k : a.q;
  const Strided& own2 = KEYS ? a.v : a.d_o;
  const Strided& walk1 = KEYS ? a.q : a.k;
  const Strided& walk2 = KEYS ? a.d_o : a.v;

  const int mine = first + wave * 16 * OT;
  frag x1[OT][KS], x2[OT][KS];
  float own_lse[OT], own_delta[OT], own_left[OT];
#pragma unroll
  for (int t = 0; t < OT; ++t) {
    const int r = mine + 16 * t + n;
    const bool live = r < own_count;
    const int64_t at = own0 + (live ? r : 0);
    const int head = KEYS ? kv_head : head0;
    own_operand<T, KS>(x1[t], own1, at, head, live, a.dim);
    own_operand<T, KS>(x2[t], own2, at, head, live, a.dim);
    own_lse[t] = own_delta[t] = own_left[t] = 0.0f;
    if constexpr (!KEYS) {
      frag o[KS];
      own_operand<T, KS>(o, a.o, at, head, live, a.dim);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < 8; ++i) own_delta[t] = __builtin_fmaf((float)o[ks][i], (float)x2[t][ks][i], own_delta[t]);
      own_delta[t] = over_groups_sum(own_delta[t]);
      if (live) {
        const int64_t line = (int64_t)head0 * a.queries.rows + at;
        const float l = a.lse[line];
        own_lse[t] = l == -kInfinity ? kInfinity : l * kLog2E;
        if (!kMend && blockIdx.y == 0 && g == 0) a.delta[line] = own_delta[t];
      }
    }
  }
  float4v acc1[OT][F], acc2[kSecond ? OT : 1][kSecond ? F : 1];
#pragma unroll
  for (int t = 0; t < OT; ++t)
#pragma unroll
    for (int f = 0; f < F; ++f) {
      acc1[t][f] = float4v{0, 0, 0, 0};
      if constexpr (kSecond) acc2[t][f] = float4v{0, 0, 0, 0};
    }
  int ds_e = 126;

  // tiles walked over: keys up to the last that a row of ours sees; queries from the first that sees one of ours
  int from = 0, to = walk_count;
  if (a.causal) {
    if (KEYS) from = min(max(first - shift, 0), walk_count) / BS * BS;
    else to = min(max(min(first + kRows, rows) + shift, 0), walk_count);
  }
  const int per_head = to > from ? (to - from + BS - 1) / BS : 0;
  const int all_steps = KEYS ? per_head * a.group : per_head;
  int begin = 0, steps = all_steps;
  if (a.splits > 1) begin = piece_of(all_steps, blockIdx.y, a.splits), steps = piece_of(all_steps, blockIdx.y + 1, a.splits);
  int member = KEYS && begin ? begin / per_head : 0, at = from + (begin - member * per_head) * BS;

  const uint32_t bytes1 = (uint32_t)walk1.row * sizeof(T), bytes2 = (uint32_t)walk2.row * sizeof(T);
  const char* const from1 = (const char*)element<T>(walk1, walk0, KEYS ? head0 : kv_head);
  const char* const from2 = (const char*)element<T>(walk2, walk0, KEYS ? head0 : kv_head);
  Load l1, l2;
  const Lanes<T, DP> lanes;
  l1.begin(bytes1, a.dim);
  l2.begin(bytes2, a.dim);
  float row_stat = 0.0f;
  int next_at = at, next_member = member;  // of the tile that is on its way
  auto issue = [&](int j, auto kept) {
    char* to_tile = tiles + (j & 1) * 2 * kTile;
    l1.issue(from1 + (int64_t)next_at * bytes1 + (KEYS ? (int64_t)next_member * walk1.head * (int64_t)sizeof(T) : 0), to_tile, walk_count - next_at, bytes1, a.dim, kept);
    l2.issue(from2 + (int64_t)next_at * bytes2 + (KEYS ? (int64_t)next_member * walk2.head * (int64_t)sizeof(T) : 0), to_tile + kTile, walk_count - next_at, bytes2, a.dim, kept);
    if (KEYS && threadIdx.x < 2 * BS) {
      const int r = min(next_at + (int)threadIdx.x % BS, walk_count - 1);
      const float* p = (int)threadIdx.x < BS ? a.lse : a.delta;
      row_stat = p[(int64_t)(head0 + next_member) * a.queries.rows + walk0 + r];
    }
  };
  auto land = [&](int j) {
    char* at = tiles + (j & 1) * 2 * kTile;
    l1.land(at);
    l2.land(at + kTile);
    if (KEYS && threadIdx.x < 2 * BS)
      stats[(j & 1) * 2 * BS + threadIdx.x] = (int)threadIdx.x >= BS ? row_stat : row_stat == -kInfinity ? kInfinity : row_stat * kLog2E;
    if (DIRECT) tiles_are_here();
  };
  if (steps > begin) {
    issue(begin, Constant<kKept>{});
    land(begin);
  }
  __syncthreads();
  auto step = [&](int j, int at, auto hidden) {
    constexpr bool kHidden = decltype(hidden)::value;
    const int t1 = (j & 1) * 2 * kTile, t2 = t1 + kTile, rows1 = lanes.row + t1, rows2 = lanes.row + t2;
    // scores (base 2) and dO V^T: rows are the tile's, columns ours
    float4v s[TT][OT], d[TT][OT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
#pragma unroll
      for (int t = 0; t < OT; ++t) s[tt][t] = d[tt][t] = float4v{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const frag y1 = row_operand<T, DP>(tiles, rows1, 16 * tt, ks), y2 = row_operand<T, DP>(tiles, rows2, 16 * tt, ks);
#pragma unroll
        for (int t = 0; t < OT; ++t) {
          s[tt][t] = M::mma(y1, x1[t][ks], s[tt][t]);
          d[tt][t] = M::mma(y2, x2[t][ks], d[tt][t]);
        }
      }
    }
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
          if constexpr (kHidden) {
            const int theirs = at + 16 * tt + 4 * g + i, ours = mine + 16 * t + n;
            const int query = KEYS ? theirs : ours, key = KEYS ? ours : theirs;
            const bool visible = query < rows && key < keys && (!a.causal || key <= query + shift);
            p = visible ? p : 0.0f;
            ds = visible ? ds : 0.0f;
          }
          s[tt][t][i] = p;
          d[tt][t][i] = ds;
          if constexpr (kMend) own_left[t] += ds;
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
        if constexpr (kSecond) p[t] = as_operand<T>(s[2 * kk][t], s[2 * kk + 1][t]);
      }
#pragma unroll
      for (int f = 0; f < F; ++f) {
        const frag y1 = turned_operand<T, DP>(tiles, lanes.turned + t1, 32 * kk, f);
#pragma unroll
        for (int t = 0; t < OT; ++t) acc1[t][f] = M::mma(y1, ds[t], acc1[t][f]);
        if constexpr (kSecond) {
          const frag y2 = kMend ? y1 : turned_operand<T, DP>(tiles, lanes.turned + t2, 32 * kk, f);
#pragma unroll
          for (int t = 0; t < OT; ++t) acc2[t][f] = M::mma(y2, p[t], acc2[t][f]);
        }
      }
    }
    if constexpr (!kHidden && sizeof(T) == 2) interleave<TT * KS * 2, F * (TT / 2) * (KEYS ? 4 : 2), OT, KEYS ? 2 : 1>();
  };
  // Loops of their own for steps with hidden pairs and for those without: together in one, sums move between registers at each step.
  int j = begin;
  auto some_hidden = [&]() {
    const bool end = at + BS > walk_count || mine + 16 * OT > own_count;
    return end || (a.causal && (KEYS ? mine + 16 * OT - 1 > at + shift : at + BS - 1 > mine + shift));
  };
  auto one = [&](auto hidden) {
    next_at = at + BS, next_member = member;
    if (KEYS && next_at >= to) next_at = from, next_member = member + 1;
    if (j + 1 < steps) issue(j + 1, Constant<!decltype(hidden)::value && kKept>{});
    step(j, at, hidden);
    if (j + 1 < steps) land(j + 1);
    __syncthreads();
    at = next_at, member = next_member;
    ++j;
  };
#pragma unroll 1
  while (j < steps) {
#pragma unroll 1
    while (j < steps && !some_hidden()) one(Constant<false>{});
#pragma unroll 1
    while (j < steps && some_hidden()) one(Constant<true>{});
  }
  constexpr float kUnit = __is_same(T, _Float16) ? 1.0f / 128.0f : 1.0f;
#pragma unroll
  for (int t = 0; t < OT; ++t) {
    const int r = mine + 16 * t + n;
    const float left = kMend ? over_groups_sum(own_left[t]) * kUnit : 0.0f;
    if (r >= own_count) continue;
    if constexpr (__is_same(T, _Float16)) {
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc1[t][f][i] = ldexpf(acc1[t][f][i], -ds_e - (int)weight_unit<T>());
    }
    if constexpr (kMend) {
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc1[t][f][i] -= left * (acc2[t][f][i] * kUnit);
      if (g == 0) a.delta[(int64_t)head0 * a.queries.rows + own0 + r] = own_delta[t] + left;
    }
    if constexpr (!kMend) {
      if (a.splits > 1) {
        constexpr int kSums = KEYS ? 2 : 1;
        float* p = a.partial + (((int64_t)blockIdx.y * own.rows + own0 + r) * heads + (KEYS ? kv_head : head0)) * kSums * a.dim + 4 * g;
#pragma unroll
        for (int f = 0; f < F; ++f) {
          if (16 * f + 4 * g >= a.dim) continue;
          *reinterpret_cast<float4v*>(p + 16 * f) = acc1[t][f];
          if constexpr (KEYS) *reinterpret_cast<float4v*>(p + a.dim + 16 * f) = acc2[t][f] * kUnit;
        }
        continue;
      }
    }
    store_column<T, F>(KEYS ? a.dk : a.dq, own0 + r, KEYS ? kv_head : head0, a.dim, acc1[t], a.scale);
    if constexpr (KEYS) store_column<T, F>(a.dv, own0 + r, kv_head, a.dim, acc2[t], kUnit);
  }
}

// Outputs of cut walks, in their order: four elements a thread.
template <class T> __global__ __launch_bounds__(kThreads) void prompt_join_forward(PromptArgs a) {
  const int quads = a.dim / 4;
  const int64_t rows = (int64_t)a.queries.rows * a.heads, at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (at >= rows * quads) return;
  const int64_t line = at / quads, row = line / a.heads;
  const int d = (int)(at - line * quads) * 4, head = (int)(line - row * a.heads);
  float most = -kInfinity;
  for (int i = 0; i < a.splits; ++i) most = fmaxf(most, a.stats[i * rows + line].x);
  const float base = most == -kInfinity ? 0.0f : most;
  float total = 0.0f;
  float4v sum = {0, 0, 0, 0};
  for (int i = 0; i < a.splits; ++i) {
    const float2 st = a.stats[i * rows + line];
    const float w = exp2_fast(st.x - base);
    total += st.y * w;
    sum += *reinterpret_cast<const float4v*>(a.partial + (i * rows + line) * a.dim + d) * w;
  }
  const float by = total == 0.0f ? 0.0f : 1.0f / total;
  struct Four { T v[4]; } o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.v[i] = (T)(sum[i] * by);
  store_any(element<T>(a.o, row, head) + d, o);
  if (a.lse && d == 0)
    a.lse[(int64_t)head * a.queries.rows + row] =
        total == 0.0f ? -kInfinity : (most + __builtin_amdgcn_logf(total * without_unit<T>())) * kLn2;
}

// Sums of cut walks, in their order: four elements a thread.
template <class T, bool KEYS> __global__ __launch_bounds__(kThreads) void prompt_join(PromptArgs a) {
  constexpr int kSums = KEYS ? 2 : 1;
  const int heads = KEYS ? a.kv_heads : a.heads, quads = a.dim / 4;
  const int64_t all = (int64_t)(KEYS ? a.keys.rows : a.queries.rows) * heads * kSums * quads;
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (at >= all) return;
  float4v sum = {0, 0, 0, 0};
  for (int i = 0; i < a.splits; ++i) sum += *reinterpret_cast<const float4v*>(a.partial + (i * all + at) * 4);
  const int64_t line = at / quads, row_head = line / kSums;
  const int d = (int)(at - line * quads) * 4, which = (int)(line - row_head * kSums);
  const int64_t row = row_head / heads;
  struct Four { T v[4]; } o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.v[i] = (T)(which ? sum[i] : sum[i] * a.scale);
  store_any(element<T>(which ? a.dv : KEYS ? a.dk : a.dq, row, (int)(row_head - row * heads)) + d, o);
}

typedef void (*prompt_t)(PromptArgs);
struct PromptKernel {
  prompt_t run;
  int rows;     // of a workgroup
  int walked;   // rows of a tile
  int threads;
  size_t lds;
};

template <class T, int DP, int QT, int BK, int WAVES, int OCCUPANCY> PromptKernel forward_of(bool direct) {
  return {direct ? prompt_forward<T, DP, QT, BK, WAVES, OCCUPANCY, true> : prompt_forward<T, DP, QT, BK, WAVES, OCCUPANCY, false>, 16 * WAVES * QT,
          BK, 64 * WAVES, (size_t)4 * BK * TileOf<T, DP>::kRowBytes + 16};
}
template <class T, int DP, int OT, int BS, int WAVES, int OCCUPANCY, bool KEYS> PromptKernel backward_of(bool direct) {
  return {direct ? prompt_backward<T, DP, OT, BS, WAVES, OCCUPANCY, KEYS, true> : prompt_backward<T, DP, OT, BS, WAVES, OCCUPANCY, KEYS, false>,
          16 * WAVES * OT, BS, 64 * WAVES, (size_t)4 * BS * TileOf<T, DP>::kRowBytes + 16 * BS};
}

// By the head's size; `direct`: what is walked over lies at multiples of 16 bytes; `many`: tiles of 128 rows are
// more than run at once (of queries, whose walks are short, twice that).
PromptKernel prompt_forward_bf16(int dim, bool direct);
PromptKernel prompt_forward_f16(int dim, bool direct);
PromptKernel prompt_forward_f32(int dim, bool direct);
PromptKernel prompt_keys_bf16(int dim, bool direct, bool many);
PromptKernel prompt_keys_f16(int dim, bool direct, bool many);
PromptKernel prompt_keys_f32(int dim, bool direct, bool many);
PromptKernel prompt_queries_bf16(int dim, bool direct, bool many);
PromptKernel prompt_queries_f16(int dim, bool direct, bool many);
PromptKernel prompt_queries_f32(int dim, bool direct, bool many);
prompt_t prompt_join_kernel(int type, bool keys);
prompt_t prompt_join_forward_kernel(int type);

// The loop of hidden steps, with its token-by-token path inlined, keeps registers in memory: 42 to 142 of heads of 192 and 256 (16 bits), 45 and
// 103 of 128 and 256 (binary32), up to 11 of 64 and 128; the other loop none.
template <class T> PromptKernel forward_for(int dim, bool direct) {
  if constexpr (sizeof(T) == 2) {
    if (dim <= 64) return forward_of<T, 64, 2, 64, 4, 3>(direct);  // two waves a SIMD: 8192 tokens, 32 heads: 419 us, 397
    if (dim <= 96) return forward_of<T, 96, 2, 64, 4, 2>(direct);
    if (dim <= 128) return forward_of<T, 128, 2, 64, 4, 2>(direct);
    // 16 rows a wave: 8192 tokens, 16 heads of 192 on 4: 545 us, 488; of 256: 750, 580
    if (dim <= 192) return forward_of<T, 192, 2, 32, 4, 2>(direct);
    return forward_of<T, 256, 2, 32, 4, 2>(direct);
  } else {
    if (dim <= 64) return forward_of<T, 64, 1, 32, 4, 2>(direct);
    if (dim <= 96) return forward_of<T, 96, 1, 32, 4, 2>(direct);
    if (dim <= 128) return forward_of<T, 128, 1, 32, 4, 2>(direct);
    if (dim <= 192) return forward_of<T, 192, 1, 32, 4, 1>(direct);
    return forward_of<T, 256, 1, 32, 4, 1>(direct);
  }
}
template <class T, bool KEYS> PromptKernel backward_for(int dim, bool direct, bool many) {
  if constexpr (sizeof(T) == 2) {
    // 32 rows a wave where that leaves enough workgroups: gradients of 8192 tokens, 32 heads of 64 on 8: 1236 us, 1134 (binary16 1385,
    // 1234); of 96: 1815, 1498 (2049, 1677); of 2048 tokens 127, 145 and 186, 201
    if (dim <= 64 && many) return backward_of<T, 64, 2, 64, 4, 2, KEYS>(direct);
    if (dim <= 64) return backward_of<T, 64, 1, 64, 4, 2, KEYS>(direct);
    if (dim <= 96 && many) return backward_of<T, 96, 2, 32, 4, 2, KEYS>(direct);
    if (dim <= 96) return backward_of<T, 96, 1, 64, 4, 2, KEYS>(direct);
    if (dim <= 128) return backward_of<T, 128, 1, 64, 4, 2, KEYS>(direct);
    // one wave a SIMD: the gradients of 8192 tokens, 16 heads of 192 on 4: 2665 us, 1660; of 256: 2770 (binary16 4055), 2417 (2556)
    if (dim <= 192) return backward_of<T, 192, 1, 32, 4, 2, KEYS>(direct);
    return backward_of<T, 256, 1, 32, 4, 2, KEYS>(direct);
  } else {
    if (dim <= 64) return backward_of<T, 64, 1, 32, 4, 2, KEYS>(direct);
    if (dim <= 96) return backward_of<T, 96, 1, 32, 4, 1, KEYS>(direct);
    if (dim <= 128) return backward_of<T, 128, 1, 32, 4, 1, KEYS>(direct);
    if (dim <= 192) return backward_of<T, 192, 1, 32, 4, 1, KEYS>(direct);
    return backward_of<T, 256, 1, 32, 4, 1, KEYS>(direct);
  }
}

}  // namespace att
}  // namespace squant
