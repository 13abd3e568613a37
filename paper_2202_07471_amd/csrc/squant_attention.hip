// Host side of attention and of the quantised cache: argument checks, how far a sequence is split, launches.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "squant.h"

#include "squant_cache_attention.h"
#include "squant_prompt.h"

namespace {

using namespace squant;
using namespace squant::att;

constexpr int64_t kMost = 0x7fffffffLL, kMostTokens = 1 << 30;  // of a table
// Of a token's keys (512 heads of 256): 2^15 pieces of 8 with its values', whose divisions by multiplication are exact to 2^16.
constexpr int64_t kMostElements = 1 << 17;
// Elements between rows and between heads: a tile's rows are within 32 bits of bytes of each other, a buffer's within 64.
constexpr int64_t kFarRow = (int64_t)1 << 22, kFarHead = (int64_t)1 << 31;

// A scale times log2(e) stays a number: a score of 0 times infinity would be none.
float base2(float scale) { return std::min(scale * kLog2E, FLT_MAX); }

int element_bytes(int type) { return type == SQUANT_W_F32 ? 4 : 2; }
bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }
int check_type(int type) { return type < SQUANT_W_F32 || type > SQUANT_W_BF16 ? SQUANT_ERR_FORMAT : SQUANT_OK; }

// [rows][heads][dim] whose data is there, aligned and without heads or rows of negative or overlapping steps.
int check_heads(const squant_heads_t* h, int64_t rows, int32_t heads, int32_t dim, int type) {
  if (!h || !h->data) return SQUANT_ERR_NULL;
  if (misaligned(h->data, element_bytes(type))) return SQUANT_ERR_FORMAT;
  if ((heads > 1 && (h->head < dim || h->head > kFarHead)) || (rows > 1 && (h->row < dim || h->row > kFarRow))) return SQUANT_ERR_SHAPE;
  return SQUANT_OK;
}
// Whether every head of every row begins at a multiple of 16 bytes.
bool whole_pieces(const squant_heads_t* h, int type) {
  const int e = element_bytes(type);
  return !misaligned(h->data, 16) && h->row * e % 16 == 0 && h->head * e % 16 == 0;
}
// A step that is never taken counts as none.
Strided strided(const squant_heads_t* h, int64_t rows) { return Strided{(char*)h->data, rows > 1 ? h->row : 0, h->head}; }

int check_cache(const squant_cache_t* c) {
  if (!c || !c->key_codes || !c->key_scales || !c->value_codes || !c->value_scales) return SQUANT_ERR_NULL;
  if (c->format != SQUANT_OUT_INT8 && c->format != SQUANT_OUT_INT4) return SQUANT_ERR_FORMAT;
  if (misaligned(c->key_codes, 16) || misaligned(c->value_codes, 16) || misaligned(c->key_scales, 2) || misaligned(c->value_scales, 2))
    return SQUANT_ERR_FORMAT;
  if (c->pages <= 0 || c->page_size <= 0 || c->heads <= 0) return SQUANT_ERR_SHAPE;
  if ((double)c->pages * c->page_size * c->heads > (double)kMost) return SQUANT_ERR_SHAPE;
  const int32_t d = c->head_dim;
  if ((int64_t)c->heads * d > kMostElements) return SQUANT_ERR_SHAPE;
  return d == 32 || d == 64 || d == 96 || d == 128 || d == 192 || d == 256 ? SQUANT_OK : SQUANT_ERR_SHAPE;
}

int check_paged(const squant_paged_t* w, int64_t rows) {
  if (!w) return SQUANT_ERR_NULL;
  if (rows < 0 || rows > kMost || w->sequences < 0 || w->table_width < 0) return SQUANT_ERR_SHAPE;
  if (!w->starts && rows != w->sequences) return SQUANT_ERR_SHAPE;
  if (misaligned(w->table, 4) || misaligned(w->lengths, 4) || misaligned(w->starts, 4)) return SQUANT_ERR_FORMAT;
  return w->sequences && (!w->lengths || (w->table_width && !w->table)) ? SQUANT_ERR_NULL : SQUANT_OK;
}

Cache cache_of(const squant_cache_t& c, const squant_paged_t& w) {
  Cache o{};
  o.codes[0] = (uint8_t*)c.key_codes, o.codes[1] = (uint8_t*)c.value_codes;
  o.scales[0] = (uint16_t*)c.key_scales, o.scales[1] = (uint16_t*)c.value_scales;
  o.pages = c.pages, o.page_size = c.page_size, o.heads = c.heads, o.dim = c.head_dim;
  int l = 0;
  while (((int64_t)1 << l) < c.page_size) ++l;
  o.shift = l - 1;
  o.magic = l ? (uint32_t)((((uint64_t)1 << (31 + l)) / (uint32_t)c.page_size) + 1) : 0;
  o.table = w.table, o.table_width = w.table_width, o.lengths = w.lengths;
  return o;
}
Packed packed_of(const squant_paged_t& w, int64_t rows) { return Packed{w.starts, w.sequences, (int32_t)rows, !w.starts}; }

bool fits(int64_t groups, int64_t gy = 1, int threads = kThreads) { return groups > 0 && groups * threads <= 0xffffffffLL && gy <= 0xffff; }

template <class A> int launch(void (*k)(A), int64_t gx, int64_t gy, size_t lds, hipStream_t st, const A& a, int threads = kThreads) {
  if (!fits(gx, gy, threads)) return SQUANT_ERR_SHAPE;
  // kernels that ask for more LDS than a workgroup gets by default say so: the attribute is the kernel's, not a call's
  if (lds > 64 * 1024 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return SQUANT_ERR_DEVICE;
  }
  hipLaunchKernelGGL(k, dim3((unsigned)gx, (unsigned)gy), dim3((unsigned)threads), (unsigned)lds, st, a);
  return hipGetLastError() == hipSuccess ? SQUANT_OK : SQUANT_ERR_DEVICE;
}

int cache_rows(bool write, const squant_heads_t* k, const squant_heads_t* v, int type, int64_t rows, const squant_cache_t* c,
               const squant_paged_t* w, void* stream) {
  if (int rc = check_type(type)) return rc;
  if (int rc = check_cache(c)) return rc;
  if (int rc = check_paged(w, rows)) return rc;
  if (rows == 0) return SQUANT_OK;
  if (int rc = check_heads(k, rows, c->heads, c->head_dim, type)) return rc;
  if (int rc = check_heads(v, rows, c->heads, c->head_dim, type)) return rc;
  CacheRowsArgs a{};
  a.cache = cache_of(*c, *w);
  a.rows = packed_of(*w, rows);
  a.x[0] = strided(k, rows), a.x[1] = strided(v, rows);
  const int64_t pieces = (int64_t)2 * c->heads * (c->head_dim / 8);
  a.pieces = (int32_t)pieces, a.dim_pieces = c->head_dim / 8;
  a.piece_magic = (uint32_t)((((uint64_t)1 << 32) / (uint64_t)pieces) + 1);
  a.dim_magic = (uint32_t)((((uint64_t)1 << 32) / (uint64_t)a.dim_pieces) + 1);
  // 1024 pieces a workgroup (4 a thread) where that leaves a thousand of them, else 256.  16 and 32 a thread are slower: a cache of 66815 tokens
  // of 8 heads of 128 in 4 bits to bfloat16 106 us, 112 and 125
  const int64_t wanted = rows * pieces >= 1024 * 1024 ? 4 * kThreads : kThreads;
  a.rows_each = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kMostRows, wanted / pieces));
  const int64_t groups = (rows + a.rows_each - 1) / a.rows_each;
  return launch(write ? cache_write_kernel(type, (int)c->format) : cache_read_kernel(type, (int)c->format), groups, 1, 0, (hipStream_t)stream, a);
}

// How attention over a cache is cut: 16 or 32 rows (tokens times grouped heads) a workgroup, and stretches of the sequences,
// whose lengths the host does not know: their capacity counts.
struct CacheSplit {
  int rt;
  int64_t tiles;
  int64_t splits, chunk;
  size_t stats_bytes, bytes;
};
// A workgroup costs as much as a few hundred tokens before its first and behind its last: about as many as run at once, and no more
// than kMostChunk tokens each, so that sequences of different lengths balance.  96 sequences of 1024 to 16384 tokens: 179 us with stretches
// of 6144, 171 with 1536.  Of 32 rows two run on a compute unit, 11 sequences of up to 6007 tokens with five rows each: 48 us with 512
// workgroups, 37 with 768, 38 with 1024; of 16 rows three or more, 13 sequences of up to 3001 tokens with a row each: 23 us with 768, 21 with 1024.
// Pieces' sums take kMostSums bytes at most, whatever a table could hold; those of 8000 workgroups or more, so where it binds there are enough.
// 1024 sequences of up to 1500 tokens, 32 heads of 128 on 8, tables of 131072 tokens: 765 us and 1.5 GB with stretches of 1536, 246 us and
// 119 MB with seven of 18816.
constexpr int64_t kGroups16 = 1024, kGroups32 = 768, kLeastChunk = 512, kMostChunk = 1536, kMostSplits = 1024, kMostSums = 1 << 27;

bool split_cache(int64_t rows, int32_t heads, const squant_cache_t& c, const squant_paged_t& w, CacheSplit& s) {
  const int group = heads / c.heads;
  const int64_t each = w.sequences ? (rows + w.sequences - 1) / w.sequences : 0;
  s.rt = each * group > 16 && c.head_dim <= 128 && c.page_size % 16 == 0 ? 2 : 1;
  const int tile = 16 * s.rt;
  s.tiles = w.starts ? tiles_bound(rows, group, tile, w.sequences) : (int64_t)w.sequences * ((group + tile - 1) / tile);
  const int64_t capacity = (int64_t)w.table_width * c.page_size;
  const int64_t groups = s.tiles * c.heads;
  int64_t chunk = capacity * groups / (s.rt == 2 ? kGroups32 : kGroups16);
  chunk = std::max({kLeastChunk, std::min(kMostChunk, (chunk + 127) / 128 * 128), (capacity / kMostSplits + 127) / 128 * 128});
  const int64_t sums = rows * heads * (4 * (int64_t)c.head_dim + 8), pieces = std::max<int64_t>(1, kMostSums / std::max<int64_t>(1, sums));
  chunk = std::max(chunk, ((capacity + pieces - 1) / pieces + 127) / 128 * 128);
  s.splits = std::max<int64_t>(1, (capacity + chunk - 1) / chunk);
  s.chunk = s.splits == 1 ? std::max<int64_t>(128, (capacity + 127) / 128 * 128) : chunk;
  s.stats_bytes = s.splits > 1 ? (size_t)(s.splits * rows * heads * 8 + 255) / 256 * 256 : 0;
  s.bytes = s.splits > 1 ? s.stats_bytes + (size_t)s.splits * rows * heads * c.head_dim * 4 : 0;
  return fits(groups, s.splits) && fits((rows * heads + kWaves - 1) / kWaves) && s.splits * (double)rows * heads < 4e15;
}

int check_cache_attention(int64_t rows, int32_t heads, const squant_cache_t* c, const squant_paged_t* w) {
  if (int rc = check_cache(c)) return rc;
  if (int rc = check_paged(w, rows)) return rc;
  if ((int64_t)w->table_width * c->page_size > kMostTokens) return SQUANT_ERR_SHAPE;
  return heads <= 0 || heads % c->heads || (double)rows * heads > (double)kMost ? SQUANT_ERR_SHAPE : SQUANT_OK;
}

int check_packed(const squant_packed_t* p) {
  if (!p) return SQUANT_ERR_NULL;
  if (p->q_rows < 0 || p->k_rows < 0 || p->q_rows > kMost || p->k_rows > kMost || p->sequences < 0) return SQUANT_ERR_SHAPE;
  if (p->heads <= 0 || p->kv_heads <= 0 || p->heads % p->kv_heads || p->head_dim <= 0 || p->head_dim > 256 || p->head_dim % 8)
    return SQUANT_ERR_SHAPE;
  if ((double)p->q_rows * p->heads > (double)kMost) return SQUANT_ERR_SHAPE;
  if (!p->q_starts != !p->k_starts) return SQUANT_ERR_NULL;
  if (!p->q_starts && p->sequences != 1) return SQUANT_ERR_SHAPE;
  if (misaligned(p->q_starts, 4) || misaligned(p->k_starts, 4)) return SQUANT_ERR_FORMAT;
  if (!(p->scale >= 0.0f) || !std::isfinite(p->scale) || p->causal < 0 || p->causal > 1) return SQUANT_ERR_MODE;
  return SQUANT_OK;
}

PromptArgs prompt_args(const squant_packed_t& p) {
  PromptArgs a{};
  a.queries = Packed{p.q_starts, p.sequences, (int32_t)p.q_rows, false};
  a.keys = Packed{p.k_starts, p.sequences, (int32_t)p.k_rows, false};
  a.heads = p.heads, a.kv_heads = p.kv_heads, a.group = p.heads / p.kv_heads, a.dim = p.head_dim;
  a.causal = p.causal, a.scale = p.scale;
  a.scale2 = std::max(base2(p.scale), 1.4e-45f);
  return a;
}
int64_t prompt_groups(const Packed& p, const PromptKernel& k, int32_t heads) {
  return tiles_bound(p.rows, 1, k.rows, p.count) * heads;
}

// Where there are few workgroups, walks are cut into at most 8 pieces whose sums a launch more adds up.
// Fewer than run at once: to about 512, at least 2 tiles a piece on average.  Six packed sequences of up to 515 tokens, six heads of 96 on two,
// binary32: dK and dV 199 us, 47 and a join of 5 with eight pieces; dQ 58, 29 and 4 with three.
// Hardly more than that: the longest walk of a causal sequence, twice the average, ends last, so long walks are cut on, to `most`
// workgroups and 12 tiles a piece.  2048 tokens, 32 heads of 128 on 8, bfloat16: all gradients 269 us, 209 with five pieces for dK and dV; 4096
// tokens 675, 570 with two; binary32 1748, 1244.  Pieces of 8 tiles (1024 tokens of 32 heads on 32): 63 us, 77.
int walk_splits(int64_t groups, int64_t walked, const squant_packed_t& p, int heads, int tile, int64_t most) {
  const int64_t tiles = heads * (walked / std::max<int64_t>(1, p.sequences)) / tile, any = std::max<int64_t>(1, groups);
  const int64_t few = std::min<int64_t>(kRunAtOnce / any, tiles / 2), uneven = p.causal ? std::min(most / any, tiles / 12) : 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(8, std::max(few, uneven)));
}
// Forward walks of 16-bit types and of large heads are short against what a piece costs: 2048 tokens, 32 heads of 128: 64 us, 78 with two
// pieces; 4096 of 8 heads 93, 68 with three; binary32, 16 heads of 128: 238, 196 with two, of 256: 440, 472.
constexpr int64_t kMostForward = 1024, kMostPieces = 1536;

struct ForwardPlan {
  PromptKernel run;
  int64_t groups;
  int splits;
  size_t stats, partial;
  bool fit;
  size_t bytes() const { return stats + partial; }
};
ForwardPlan plan_forward(const squant_packed_t& p, int type, bool direct) {
  ForwardPlan f{};
  f.run = (type == SQUANT_W_F32 ? prompt_forward_f32 : type == SQUANT_W_F16 ? prompt_forward_f16 : prompt_forward_bf16)(p.head_dim, direct);
  f.groups = prompt_groups(prompt_args(p).queries, f.run, p.heads);
  f.splits = walk_splits(f.groups, p.k_rows, p, 1, f.run.walked, type == SQUANT_W_F32 && p.head_dim <= 128 ? kMostPieces : kMostForward);
  if (f.splits > 1) {
    f.stats = ((size_t)f.splits * p.q_rows * p.heads * 8 + 255) / 256 * 256;
    f.partial = (size_t)f.splits * p.q_rows * p.heads * p.head_dim * 4;
  }
  f.fit = fits(f.groups, f.splits, f.run.threads);
  return f;
}

// Queries are walked over by dK and dV of all types, keys by dQ of binary32 (16-bit types have three sums to add up there).
struct BackwardPlan {
  PromptKernel queries, keys;
  int64_t q_groups, k_groups;
  int q_splits, k_splits;
  size_t delta, q_partial, k_partial;  // bytes; the partial sums follow delta, one after the other's use
  bool fit;
  size_t bytes() const { return delta + std::max(q_partial, k_partial); }
};
BackwardPlan plan_backward(const squant_packed_t& p, int type, bool queries_direct, bool keys_direct) {
  BackwardPlan b{};
  const PromptArgs a = prompt_args(p);
  const auto many = [](const Packed& own, int32_t heads, int most) { return tiles_bound(own.rows, 1, 128, own.count) * heads > most; };
  b.queries = (type == SQUANT_W_F32 ? prompt_queries_f32 : type == SQUANT_W_F16 ? prompt_queries_f16 : prompt_queries_bf16)(p.head_dim, keys_direct, many(a.queries, p.heads, 2 * kRunAtOnce));
  b.keys = (type == SQUANT_W_F32 ? prompt_keys_f32 : type == SQUANT_W_F16 ? prompt_keys_f16 : prompt_keys_bf16)(p.head_dim, queries_direct, many(a.keys, p.kv_heads, kRunAtOnce));
  b.q_groups = prompt_groups(a.queries, b.queries, p.heads), b.k_groups = prompt_groups(a.keys, b.keys, p.kv_heads);
  b.q_splits = type == SQUANT_W_F32 ? walk_splits(b.q_groups, p.k_rows, p, 1, b.queries.walked, kMostPieces) : 1;
  b.k_splits = walk_splits(b.k_groups, p.q_rows, p, a.group, b.keys.walked, kMostPieces);
  b.delta = ((size_t)p.q_rows * p.heads * 4 + 255) / 256 * 256;
  b.q_partial = b.q_splits > 1 ? (size_t)b.q_splits * p.q_rows * p.heads * p.head_dim * 4 : 0;
  b.k_partial = b.k_splits > 1 ? (size_t)b.k_splits * p.k_rows * p.kv_heads * 2 * p.head_dim * 4 : 0;
  b.fit = (!p.q_rows || fits(b.q_groups, b.q_splits, b.queries.threads)) && (!p.k_rows || fits(b.k_groups, b.k_splits, b.keys.threads));
  return b;
}

}  // namespace

extern "C" {

int squant_cache_write(const squant_heads_t* h_k, const squant_heads_t* h_v, squant_wtype_t type, int64_t rows,
                       const squant_cache_t* h_cache, const squant_paged_t* h_where, void* stream) {
  return cache_rows(true, h_k, h_v, (int)type, rows, h_cache, h_where, stream);
}

int squant_cache_read(const squant_cache_t* h_cache, const squant_paged_t* h_where, squant_wtype_t type, int64_t rows,
                      const squant_heads_t* h_k, const squant_heads_t* h_v, void* stream) {
  return cache_rows(false, h_k, h_v, (int)type, rows, h_cache, h_where, stream);
}

size_t squant_cache_attention_workspace_bytes(int64_t rows, int32_t heads, const squant_cache_t* h_cache, const squant_paged_t* h_where) {
  CacheSplit s;
  if (check_cache_attention(rows, heads, h_cache, h_where) || rows == 0 || !split_cache(rows, heads, *h_cache, *h_where, s)) return 0;
  return s.bytes;
}

int squant_cache_attention(const squant_heads_t* h_q, squant_wtype_t type, int64_t rows, int32_t heads, const squant_cache_t* h_cache,
                           const squant_paged_t* h_where, float scale, const squant_heads_t* h_out, void* d_workspace,
                           size_t workspace_bytes, void* stream) {
  if (int rc = check_type((int)type)) return rc;
  if (int rc = check_cache_attention(rows, heads, h_cache, h_where)) return rc;
  if (!(scale >= 0.0f) || !std::isfinite(scale)) return SQUANT_ERR_MODE;
  if (rows == 0) return SQUANT_OK;
  const squant_cache_t& c = *h_cache;
  if (int rc = check_heads(h_q, rows, heads, c.head_dim, (int)type)) return rc;
  if (int rc = check_heads(h_out, rows, heads, c.head_dim, (int)type)) return rc;
  CacheSplit s;
  if (!split_cache(rows, heads, c, *h_where, s)) return SQUANT_ERR_SHAPE;
  if (workspace_bytes < s.bytes || (s.bytes && (!d_workspace || misaligned(d_workspace, 256)))) return SQUANT_ERR_WORKSPACE;
  CacheAttentionArgs a{};
  a.cache = cache_of(c, *h_where);
  a.rows = packed_of(*h_where, rows);
  a.q = strided(h_q, rows), a.out = strided(h_out, rows);
  a.heads = heads, a.group = heads / c.heads;
  a.splits = (int32_t)s.splits, a.chunk = (int32_t)s.chunk;
  a.scale = base2(scale);
  if (s.splits > 1) a.stats = (float2*)d_workspace, a.partial = (float*)((char*)d_workspace + s.stats_bytes);
  const int ng = c.head_dim / kGroup;
  const auto of = c.format == SQUANT_OUT_INT4
                      ? (type == SQUANT_W_F32 ? cache_attention_int4_f32 : type == SQUANT_W_F16 ? cache_attention_int4_f16 : cache_attention_int4_bf16)
                      : (type == SQUANT_W_F32 ? cache_attention_int8_f32 : type == SQUANT_W_F16 ? cache_attention_int8_f16 : cache_attention_int8_bf16);
  const cache_attention_t k = of(ng, s.rt, c.page_size % 16 == 0);
  hipStream_t st = (hipStream_t)stream;
  if (int rc = launch(k, s.tiles * c.heads, s.splits, cache_attention_lds(ng, s.rt), st, a)) return rc;
  return s.splits > 1 ? launch(join_splits_kernel((int)type), (rows * heads + kWaves - 1) / kWaves, 1, 0, st, a) : SQUANT_OK;
}

size_t squant_attention_workspace_bytes(const squant_packed_t* h_packed, squant_wtype_t type) {
  if (check_type((int)type) || check_packed(h_packed) || !h_packed->q_rows) return 0;
  const ForwardPlan f = plan_forward(*h_packed, (int)type, true);
  return f.fit ? f.bytes() : 0;
}

int squant_attention(const squant_heads_t* h_q, const squant_heads_t* h_k, const squant_heads_t* h_v, squant_wtype_t type,
                     const squant_packed_t* h_packed, const squant_heads_t* h_out, float* d_lse, void* d_workspace, size_t workspace_bytes,
                     void* stream) {
  if (int rc = check_type((int)type)) return rc;
  if (int rc = check_packed(h_packed)) return rc;
  const squant_packed_t& p = *h_packed;
  if (p.q_rows == 0) return SQUANT_OK;
  if (int rc = check_heads(h_q, p.q_rows, p.heads, p.head_dim, (int)type)) return rc;
  if (int rc = check_heads(h_out, p.q_rows, p.heads, p.head_dim, (int)type)) return rc;
  if (p.k_rows) {
    if (int rc = check_heads(h_k, p.k_rows, p.kv_heads, p.head_dim, (int)type)) return rc;
    if (int rc = check_heads(h_v, p.k_rows, p.kv_heads, p.head_dim, (int)type)) return rc;
  }
  if (misaligned(d_lse, 4)) return SQUANT_ERR_FORMAT;
  const bool direct = !p.k_rows || (whole_pieces(h_k, (int)type) && whole_pieces(h_v, (int)type));
  const ForwardPlan f = plan_forward(p, (int)type, direct);
  if (!f.fit) return SQUANT_ERR_SHAPE;
  if (workspace_bytes < f.bytes() || (f.bytes() && (!d_workspace || misaligned(d_workspace, 256)))) return SQUANT_ERR_WORKSPACE;
  PromptArgs a = prompt_args(p);
  a.q = strided(h_q, p.q_rows), a.o = strided(h_out, p.q_rows);
  if (p.k_rows) a.k = strided(h_k, p.k_rows), a.v = strided(h_v, p.k_rows);
  a.lse = d_lse;
  a.by_length = f.groups > kRunAtOnce && p.sequences > 1;
  a.splits = f.splits, a.stats = (float2*)d_workspace, a.partial = (float*)((char*)d_workspace + f.stats);
  hipStream_t st = (hipStream_t)stream;
  if (int rc = launch(f.run.run, f.groups, f.splits, f.run.lds, st, a, f.run.threads)) return rc;
  if (f.splits == 1) return SQUANT_OK;
  return launch(prompt_join_forward_kernel((int)type), (p.q_rows * p.heads * (p.head_dim / 4) + kThreads - 1) / kThreads, 1, 0, st, a);
}

size_t squant_attention_backward_workspace_bytes(const squant_packed_t* h_packed, squant_wtype_t type) {
  if (check_type((int)type) || check_packed(h_packed) || !h_packed->q_rows) return 0;
  const BackwardPlan b = plan_backward(*h_packed, (int)type, true, true);
  return b.fit ? b.bytes() : 0;
}

int squant_attention_backward(const squant_heads_t* h_dout, const squant_heads_t* h_q, const squant_heads_t* h_k, const squant_heads_t* h_v,
                              const squant_heads_t* h_out, const float* d_lse, squant_wtype_t type, const squant_packed_t* h_packed,
                              const squant_heads_t* h_dq, const squant_heads_t* h_dk, const squant_heads_t* h_dv, void* d_workspace,
                              size_t workspace_bytes, void* stream) {
  if (int rc = check_type((int)type)) return rc;
  if (int rc = check_packed(h_packed)) return rc;
  const squant_packed_t& p = *h_packed;
  const int t = (int)type;
  if (p.q_rows) {
    for (const squant_heads_t* h : {h_dout, h_q, h_out, h_dq})
      if (int rc = check_heads(h, p.q_rows, p.heads, p.head_dim, t)) return rc;
    if (!d_lse) return SQUANT_ERR_NULL;
    if (misaligned(d_lse, 4)) return SQUANT_ERR_FORMAT;
  }
  if (p.k_rows)
    for (const squant_heads_t* h : {h_k, h_v, h_dk, h_dv})
      if (int rc = check_heads(h, p.k_rows, p.kv_heads, p.head_dim, t)) return rc;
  const bool keys_direct = !p.k_rows || (whole_pieces(h_k, t) && whole_pieces(h_v, t));
  const bool queries_direct = !p.q_rows || (whole_pieces(h_q, t) && whole_pieces(h_dout, t));
  const BackwardPlan b = plan_backward(p, t, queries_direct, keys_direct);
  if (!b.fit) return SQUANT_ERR_SHAPE;
  const size_t need = p.q_rows ? b.bytes() : 0;
  if (workspace_bytes < need || (need && (!d_workspace || misaligned(d_workspace, 256)))) return SQUANT_ERR_WORKSPACE;
  PromptArgs a = prompt_args(p);
  const int64_t qr = p.q_rows, kr = p.k_rows;
  if (qr) a.q = strided(h_q, qr), a.o = strided(h_out, qr), a.d_o = strided(h_dout, qr), a.dq = strided(h_dq, qr);
  if (kr) a.k = strided(h_k, kr), a.v = strided(h_v, kr), a.dk = strided(h_dk, kr), a.dv = strided(h_dv, kr);
  a.lse = const_cast<float*>(d_lse);
  a.delta = (float*)d_workspace;
  a.partial = (float*)((char*)d_workspace + b.delta);
  hipStream_t st = (hipStream_t)stream;
  const auto join_groups = [&](int64_t elements) { return (elements / 4 + kThreads - 1) / kThreads; };
  if (qr) {
    a.splits = b.q_splits, a.by_length = b.q_groups > kRunAtOnce && p.sequences > 1;
    if (int rc = launch(b.queries.run, b.q_groups, b.q_splits, b.queries.lds, st, a, b.queries.threads)) return rc;
    if (b.q_splits > 1)
      if (int rc = launch(prompt_join_kernel(t, false), join_groups(qr * p.heads * p.head_dim), 1, 0, st, a)) return rc;
  }
  if (!kr) return SQUANT_OK;
  a.splits = qr ? b.k_splits : 1, a.by_length = b.k_groups > kRunAtOnce && p.sequences > 1;
  if (int rc = launch(b.keys.run, b.k_groups, a.splits, b.keys.lds, st, a, b.keys.threads)) return rc;
  return a.splits > 1 ? launch(prompt_join_kernel(t, true), join_groups(kr * p.kv_heads * 2 * p.head_dim), 1, 0, st, a) : SQUANT_OK;
}

}  // extern "C"
