// Host side of the operators that multiply by codes: argument checks, the layout of their workspaces, the choice
// of kernel and of how far a product is split.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "squant.h"

#include "squant_lin_kernels.h"
#include "squant_lin_plan.h"

namespace {

using namespace squant;
using namespace squant::lin;

int element_bytes(int type) { return type == SQUANT_W_F32 ? 4 : 2; }
int planes_of(int type) { return type == SQUANT_W_F32 ? 2 : 1; }

int check_codes(const squant_codes_t* w) {
  if (!w || !w->codes || !w->scales) return SQUANT_ERR_NULL;
  if (w->format != SQUANT_OUT_INT8 && w->format != SQUANT_OUT_INT4) return SQUANT_ERR_FORMAT;
  if (w->cout <= 0 || w->cin <= 0 || w->cout > kMaxSide || w->cin > kMaxSide) return SQUANT_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(w->scales) & 3u) return SQUANT_ERR_FORMAT;
  return SQUANT_OK;
}

int check_rows(int type, int64_t rows) {
  if (type < SQUANT_W_F32 || type > SQUANT_W_BF16) return SQUANT_ERR_FORMAT;
  return rows < 0 || rows > kMaxRows ? SQUANT_ERR_SHAPE : SQUANT_OK;
}

bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

int check_workspace(const void* ws, size_t given, size_t wanted) {
  if (given < wanted || (wanted && (!ws || misaligned(ws, 256)))) return SQUANT_ERR_WORKSPACE;
  return SQUANT_OK;
}

// Cuts a workspace into pieces; without a base it only counts.
struct Cutter {
  char* base;
  size_t used = 0;
  template <class T> T* take(int64_t count) {
    char* p = base ? base + used : nullptr;
    used += ((size_t)count * sizeof(T) + 255) & ~(size_t)255;
    return reinterpret_cast<T*>(p);
  }
};

int64_t code_row(const squant_codes_t& w) { return w.format == SQUANT_OUT_INT8 ? w.cin : ((int64_t)w.cin + 1) / 2; }

// A launch counts its threads in 32 bits.  Every call asks for all of its launches before the first.
bool fits(int64_t groups, int threads) { return groups * threads <= 0xffffffffLL; }
bool fits(const Split& p) { return fits(p.workgroups, p.threads); }

template <class A> int launch(void (*k)(A), int64_t gx, int gy, int threads, size_t lds, hipStream_t st, const A& a) {
  if (!fits(gx, threads)) return SQUANT_ERR_SHAPE;
  hipLaunchKernelGGL(k, dim3((unsigned)gx, (unsigned)gy), dim3((unsigned)threads), (unsigned)lds, st, a);
  return hipGetLastError() == hipSuccess ? SQUANT_OK : SQUANT_ERR_DEVICE;
}

// Kernels that ask for more LDS than a workgroup gets by default say so: the attribute is the kernel's, not a call's.
int launch_product(product_t k, const Split& p, size_t lds, hipStream_t st, const ProductArgs& a) {
  if (lds > 64 * 1024 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return SQUANT_ERR_DEVICE;
  }
  return launch(k, p.workgroups, p.few ? p.tiles_m : p.slices, p.threads, lds, st, a);
}

int launch_layer(int type, const squant_codes_t& w, const Split& p, hipStream_t st, const ProductArgs& a) {
  const int format = (int)w.format;
  if (p.few) {
    const bool words = a.w_row % 4 == 0 && !misaligned(a.w, 4);
    const product_t k = type == SQUANT_W_F32   ? few_f32(format, p.row_frags, p.col_frags_each, words)
                        : type == SQUANT_W_F16 ? few_f16(format, p.row_frags, p.col_frags_each, words)
                                               : few_bf16(format, p.row_frags, p.col_frags_each, words);
    return launch_product(k, p, p.lds, st, a);
  }
  const bool prob = a.f.kind == kProb;
  const product_t k = type == SQUANT_W_F32   ? (prob ? prob_f32 : layer_f32)(format, p.mt)
                      : type == SQUANT_W_F16 ? (prob ? prob_f16 : layer_f16)(format, p.mt)
                                             : (prob ? prob_bf16 : layer_bf16)(format, p.mt);
  return launch_product(k, p, product_lds(p.mt, planes_of(type), format), st, a);
}

int launch_gradient(int type, const squant_codes_t& w, const Split& p, hipStream_t st, const ProductArgs& a) {
  const int format = (int)w.format, planes = planes_of(type);
  const product_t k = planes == 2 ? gradient_2(format, p.mt) : gradient_1(format, p.mt);
  return launch_product(k, p, product_lds(p.mt, planes, format), st, a);
}

float layer_unit(int type, int format) {
  if (format == SQUANT_OUT_INT8) return 1.0f;
  return type == SQUANT_W_BF16 ? CodeUnit<Brain, SQUANT_OUT_INT4>::inverse : CodeUnit<Half, SQUANT_OUT_INT4>::inverse;
}

// The row operand of a layer's product: the caller's rows where the kernels can read them as they are, else a copy.
struct RowOperand {
  const void* p;
  int64_t ld, plane;
  const float* factor;
};

// few_rows reads rows at any alignment and of any length; but each of its workgroups reads them anew, and 16-bit ones that lie
// between 32-bit words at several times the cost.  From 2^16 elements on a copy, a launch of 4 us, is cheaper: bfloat16 rows
// an odd distance apart, 38 x 8000 by 3648 int8 codes 60 us without it, 27 us with; 16 x 4096 by 4096 12 to 16 us without.
bool direct_rows(const void* x, int64_t ldx, int type, int64_t rows, int32_t cin) {
  if (rows <= few_rows_limit(planes_of(type))) {
    const bool between_words = type != SQUANT_W_F32 && rows > 1 && (ldx % 2 != 0 || misaligned(x, 4));
    return !between_words || rows * cin < 1 << 16;
  }
  return type != SQUANT_W_F32 && cin % kBlock == 0 && ldx % 8 == 0 && ldx <= kMaxSide && !misaligned(x, 16);
}

RowOperand lay_out_rows(Cutter& c, const void* x, int64_t ldx, int type, int64_t rows, int32_t cin, RowsArgs& r, bool& copy) {
  copy = !direct_rows(x, ldx, type, rows, cin);
  if (!copy) return RowOperand{x, ldx, 0, nullptr};
  const int planes = planes_of(type);
  const int64_t padded = ((int64_t)cin + kBlock - 1) / kBlock * kBlock;
  uint16_t* out = c.take<uint16_t>(rows * planes * padded);
  float* factor = type == SQUANT_W_F32 ? c.take<float>(rows) : nullptr;
  r.x = x; r.ldx = ldx; r.rows = rows; r.cols = cin; r.out = out; r.padded = (int32_t)padded; r.row_factor = factor;
  return RowOperand{out, planes * padded, padded, factor};
}

// The codes of a product: the caller's where the kernels can read them as they are, else a copy.
struct CodeOperand {
  const uint8_t* p;
  int64_t row;
};
CodeOperand as_they_are(const squant_codes_t& w) { return CodeOperand{(const uint8_t*)w.codes, code_row(w)}; }

// `whole`: rows of whole steps (a layer's product; a gradient reads across rows).
CodeOperand lay_out_codes(Cutter& c, const squant_codes_t& w, bool whole, CodesArgs& k) {
  const int64_t row = code_row(w);
  if (!misaligned(w.codes, 16) && (whole ? w.cin % kBlock == 0 : row % 16 == 0)) return as_they_are(w);
  const int64_t out_row = ((int64_t)w.cin + kBlock - 1) / kBlock * (w.format == SQUANT_OUT_INT8 ? kBlock : kBlock / 2);
  k.codes = (const uint8_t*)w.codes; k.row = row; k.out = c.take<uint8_t>(w.cout * out_row); k.out_row = (int32_t)out_row;
  k.chunks = w.cout * (out_row / 16);
  return CodeOperand{k.out, out_row};
}
int64_t code_blocks(const CodesArgs& k) { return (k.chunks + kRowThreads - 1) / kRowThreads; }

// Rows (`copy`) and codes that are laid out before a product, in one launch of this many workgroups.
int64_t lay_out_groups(RowsArgs& r, bool copy, int type) {
  r.w.first_block = !copy ? 0 : type == SQUANT_W_F32 ? r.rows : (r.rows * (r.padded / 8) + kRowThreads - 1) / kRowThreads;
  return r.w.first_block + code_blocks(r.w);
}
int lay_out(RowsArgs& r, bool copy, int type, hipStream_t st) {
  const int64_t groups = lay_out_groups(r, copy, type);
  if (!groups) return SQUANT_OK;
  return launch(copy && type == SQUANT_W_F32 ? split_rows_kernel() : pad_rows_kernel(), groups, 1, kRowThreads, 0, st, r);
}

void set_product(ProductArgs& a, const RowOperand& x, const CodeOperand& c, const squant_codes_t& w, const Split& p) {
  a.a = x.p; a.lda = x.ld; a.plane = x.plane;
  a.w = c.p; a.w_row = c.row; a.w_rows = w.cout; a.w_cols = w.cin;
  a.w_end = a.w + (int64_t)w.cout * a.w_row;
  a.blocks = p.blocks; a.slices = p.slices; a.tiles_m = p.tiles_m; a.tiles_n = p.tiles_n;
}

int64_t join_groups(const Split& p) {
  constexpr int per = kRowThreads / kLanes;
  return (p.row_frags_all * (p.col_frags_all / 4) + per - 1) / per;
}
int launch_join(bool grad, int type, const Split& p, const float4v* partial, const Finish& f, hipStream_t st) {
  JoinArgs j{};
  j.partial = partial; j.slices = p.slices; j.row_frags = p.row_frags_all; j.col_frags = p.col_frags_all; j.f = f;
  return launch(join_kernel(grad, type), join_groups(p), 1, kRowThreads, 0, st, j);
}

// Workspaces.  Each is laid out by the function that also runs the call, so that the two agree.  `fit`: so do its launches.
struct LinearSpace { RowOperand x; CodeOperand w; RowsArgs rows; bool copy; float4v* partial; Split p; bool fit; };
size_t lay_out_linear(void* ws, const void* x, int64_t ldx, int type, int64_t rows, const squant_codes_t& w, int keep, LinearSpace& s) {
  Cutter c{(char*)ws};
  s.rows = RowsArgs{};
  s.x = lay_out_rows(c, x, ldx, type, rows, w.cin, s.rows, s.copy);
  s.p = split_layer(rows, w.cout, w.cin, planes_of(type), (int)w.format, keep != SQUANT_KEEP_NONE, true);
  s.w = s.p.few ? as_they_are(w) : lay_out_codes(c, w, true, s.rows.w);
  s.partial = s.p.slices > 1 ? c.take<float4v>(s.p.partial_vectors()) : nullptr;
  s.fit = fits(lay_out_groups(s.rows, s.copy, type), kRowThreads) && fits(s.p) && (s.p.slices == 1 || fits(join_groups(s.p), kRowThreads));
  return s.fit ? c.used : 0;
}

int gradient_rows_per_group(int64_t rows) { return (int)std::min<int64_t>(kRowGroup, std::max<int64_t>(1, (rows + 1023) / 1024)); }

struct BackwardSpace {
  CodeOperand w; CodesArgs codes; _Float16* rows; float* factor; float* sums; int64_t partials; int64_t padded; float4v* partial; Split p;
  int64_t groups;  // of gradient_rows, by `shared`; the codes' behind them
  int shared;
  bool fit;
};
size_t lay_out_backward(void* ws, int type, int64_t rows, const squant_codes_t& w, BackwardSpace& s) {
  Cutter c{(char*)ws};
  const int planes = planes_of(type), group = gradient_rows_per_group(rows);
  s.codes = CodesArgs{};
  s.w = lay_out_codes(c, w, false, s.codes);
  s.padded = ((int64_t)w.cout + kBlock - 1) / kBlock * kBlock;
  s.rows = c.take<_Float16>(rows * planes * s.padded);
  s.factor = c.take<float>(rows);
  s.partials = (rows + group - 1) / group * std::max<int64_t>(1, kRowThreads / (s.padded / 8));
  s.sums = c.take<float>(s.partials * w.cout);
  s.p = split_gradient(rows, w.cin, w.cout, planes);
  s.partial = s.p.slices > 1 ? c.take<float4v>(s.p.partial_vectors()) : nullptr;
  const int64_t row_groups = (rows + group - 1) / group, row_threads = (s.padded / 8 + kRowThreads - 1) / kRowThreads;
  // about 512 workgroups, each of which looks for its rows' largest elements anew
  s.shared = (int)std::max<int64_t>(1, std::min(row_threads, 512 / row_groups));
  s.codes.first_block = row_groups;
  s.groups = row_groups + (code_blocks(s.codes) + s.shared - 1) / s.shared;
  s.fit = fits(s.groups, kRowThreads) && fits(s.p) && (s.p.slices == 1 || fits(join_groups(s.p), kRowThreads));
  return s.fit ? c.used : 0;
}

struct LossSpace { RowOperand x; CodeOperand w; RowsArgs rows; bool copy; float2* stats; float* label_logit; Split p; bool fit; };
size_t lay_out_loss(void* ws, const void* h, int64_t ldh, int type, int64_t rows, const squant_codes_t& w, LossSpace& s) {
  Cutter c{(char*)ws};
  s.rows = RowsArgs{};
  s.x = lay_out_rows(c, h, ldh, type, rows, w.cin, s.rows, s.copy);
  s.stats = c.take<float2>(rows * (((int64_t)w.cout + kTile - 1) / kTile));
  s.label_logit = c.take<float>(rows);
  s.p = split_layer(rows, w.cout, w.cin, planes_of(type), (int)w.format, true, false);
  s.w = s.p.few ? as_they_are(w) : lay_out_codes(c, w, true, s.rows.w);
  s.fit = fits(lay_out_groups(s.rows, s.copy, type), kRowThreads) && fits(s.p) && fits(rows, kRowThreads);
  return s.fit ? c.used : 0;
}

struct LossBackwardSpace {
  RowOperand x; CodeOperand w; RowsArgs rows; bool copy; float* unit; _Float16* prob; int64_t piece; int32_t pieces;
  float* label_prob; float* other_sums; int32_t other_tiles; float4v* partial; Split g; bool fit;
};
size_t lay_out_loss_backward(void* ws, const void* h, int64_t ldh, int type, int64_t rows, const squant_codes_t& w, LossBackwardSpace& s) {
  Cutter c{(char*)ws};
  const int planes = planes_of(type);
  s.rows = RowsArgs{};
  s.x = lay_out_rows(c, h, ldh, type, rows, w.cin, s.rows, s.copy);
  s.w = lay_out_codes(c, w, true, s.rows.w);
  s.unit = c.take<float>(1);
  s.piece = vocabulary_piece(rows, w.cout, planes);
  s.pieces = (int32_t)((w.cout + s.piece - 1) / s.piece);
  s.prob = c.take<_Float16>(rows * planes * s.piece);
  const Split first = split_layer(rows, std::min<int64_t>(s.piece, w.cout), w.cin, planes, (int)w.format, true, false);
  const Split last = split_layer(rows, w.cout - (s.pieces - 1) * s.piece, w.cin, planes, (int)w.format, true, false);
  s.other_tiles = first.tiles_n;  // a last piece has fewer
  s.other_sums = c.take<float>(rows * s.other_tiles);
  s.label_prob = c.take<float>(rows);
  s.g = split_gradient(rows, w.cin, s.piece, planes);
  s.partial = c.take<float4v>(s.g.partial_vectors());
  s.fit = fits(lay_out_groups(s.rows, s.copy, type), kRowThreads) && fits(first) && fits(last) && fits(s.g) && fits(join_groups(s.g), kRowThreads);
  return s.fit ? c.used : 0;
}

}  // namespace

extern "C" {

size_t squant_linear_workspace_bytes(const void* d_x, int64_t ldx, squant_wtype_t type, int64_t rows, const squant_codes_t* h_w, squant_keep_t keep) {
  if (check_rows((int)type, rows) || check_codes(h_w) || rows == 0) return 0;
  LinearSpace s;
  return lay_out_linear(nullptr, d_x, ldx, (int)type, rows, *h_w, (int)keep, s);
}

int squant_linear(const void* d_x, int64_t ldx, squant_wtype_t type, int64_t rows, const squant_codes_t* h_w,
                  const void* d_bias, squant_activation_t act, const void* d_residual, int64_t ldr, void* d_y, int64_t ldy,
                  squant_keep_t keep, void* d_kept, float* d_kept_scales, void* d_workspace, size_t workspace_bytes,
                  void* stream) {
  if (int rc = check_rows((int)type, rows)) return rc;
  if (int rc = check_codes(h_w)) return rc;
  if ((int)act < SQUANT_ACT_NONE || act > SQUANT_ACT_SILU || (int)keep < SQUANT_KEEP_NONE || keep > SQUANT_KEEP_FULL)
    return SQUANT_ERR_MODE;
  const squant_codes_t& w = *h_w;
  if (ldx < w.cin || ldy < w.cout || (d_residual && ldr < w.cout)) return SQUANT_ERR_SHAPE;
  if (rows == 0) return SQUANT_OK;
  if (!d_x || !d_y || (keep != SQUANT_KEEP_NONE && !d_kept) || (keep == SQUANT_KEEP_INT8 && !d_kept_scales)) return SQUANT_ERR_NULL;
  const int e = element_bytes((int)type);
  if (misaligned(d_x, e) || misaligned(d_y, e) || misaligned(d_bias, e) || misaligned(d_residual, e) ||
      (keep == SQUANT_KEEP_FULL && misaligned(d_kept, e)) || misaligned(d_kept_scales, 4))
    return SQUANT_ERR_FORMAT;
  LinearSpace s;
  const size_t need = lay_out_linear(d_workspace, d_x, ldx, (int)type, rows, w, (int)keep, s);
  if (!s.fit) return SQUANT_ERR_SHAPE;
  if (int rc = check_workspace(d_workspace, workspace_bytes, need)) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (int rc = lay_out(s.rows, s.copy, (int)type, st)) return rc;
  ProductArgs a{};
  set_product(a, s.x, s.w, w, s.p);
  Finish& f = a.f;
  f.kind = kLinear; f.act = (int)act; f.keep = (int)keep; f.out_type = (int)type;
  f.unit = layer_unit((int)type, (int)w.format);
  f.rows = rows; f.cols = w.cout; f.row_factor = s.x.factor; f.scales = w.scales;
  f.bias = d_bias; f.residual = d_residual; f.ldr = ldr; f.out = d_y; f.ldo = ldy; f.kept = d_kept; f.kept_scales = d_kept_scales;
  const Finish done = f;
  if (s.p.slices > 1) { f.kind = kPartial; f.partial = s.partial; }
  if (int rc = launch_layer((int)type, w, s.p, st, a)) return rc;
  return s.p.slices > 1 ? launch_join(false, (int)type, s.p, s.partial, done, st) : SQUANT_OK;
}

size_t squant_linear_backward_workspace_bytes(squant_wtype_t type, int64_t rows, const squant_codes_t* h_w) {
  if (check_rows((int)type, rows) || check_codes(h_w) || rows == 0) return 0;
  BackwardSpace s;
  return lay_out_backward(nullptr, (int)type, rows, *h_w, s);
}

int squant_linear_backward(const void* d_dy, int64_t lddy, squant_wtype_t type, int64_t rows, const squant_codes_t* h_w,
                           squant_activation_t act, squant_keep_t keep, const void* d_kept, const float* d_kept_scales,
                           void* d_dx, int64_t lddx, void* d_dbias, void* d_workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_rows((int)type, rows)) return rc;
  if (int rc = check_codes(h_w)) return rc;
  if ((int)act < SQUANT_ACT_NONE || act > SQUANT_ACT_SILU || (int)keep < SQUANT_KEEP_NONE || keep > SQUANT_KEEP_FULL ||
      (act == SQUANT_ACT_NONE) != (keep == SQUANT_KEEP_NONE))
    return SQUANT_ERR_MODE;
  const squant_codes_t& w = *h_w;
  if (lddy < w.cout || lddx < w.cin) return SQUANT_ERR_SHAPE;
  const int e = element_bytes((int)type);
  if (misaligned(d_dbias, e)) return SQUANT_ERR_FORMAT;
  hipStream_t st = (hipStream_t)stream;
  ColumnSumArgs sums{nullptr, 0, w.cout, d_dbias, (int)type};
  const int64_t sum_groups = ((int64_t)w.cout + kLanes - 1) / kLanes;
  if (rows == 0) return d_dbias ? launch(column_sums_kernel(), sum_groups, 1, 1024, 0, st, sums) : SQUANT_OK;
  if (!d_dy || !d_dx || (keep != SQUANT_KEEP_NONE && !d_kept) || (keep == SQUANT_KEEP_INT8 && !d_kept_scales)) return SQUANT_ERR_NULL;
  if (misaligned(d_dy, e) || misaligned(d_dx, e) || (keep == SQUANT_KEEP_FULL && misaligned(d_kept, e)) ||
      misaligned(d_kept_scales, 4))
    return SQUANT_ERR_FORMAT;
  BackwardSpace s;
  const size_t need = lay_out_backward(d_workspace, (int)type, rows, w, s);
  if (!s.fit) return SQUANT_ERR_SHAPE;
  if (int rc = check_workspace(d_workspace, workspace_bytes, need)) return rc;
  RowsArgs r{};
  r.x = d_dy; r.ldx = lddy; r.rows = rows; r.cols = w.cout; r.out = s.rows; r.padded = (int32_t)s.padded; r.row_factor = s.factor;
  r.scales = w.scales; r.kept = d_kept; r.kept_scales = d_kept_scales; r.act = (int)act; r.keep = (int)keep;
  r.rows_per_group = gradient_rows_per_group(rows);
  r.column_sums = d_dbias ? s.sums : nullptr;
  r.w = s.codes;
  if (int rc = launch(gradient_rows_kernel((int)type), s.groups, s.shared, kRowThreads, 0, st, r)) return rc;
  if (d_dbias) {
    sums.partial = s.sums; sums.partials = s.partials;
    if (int rc = launch(column_sums_kernel(), sum_groups, 1, 1024, 0, st, sums)) return rc;
  }
  const int planes = planes_of((int)type);
  ProductArgs a{};
  set_product(a, RowOperand{s.rows, planes * s.padded, s.padded, s.factor}, s.w, w, s.p);
  Finish& f = a.f;
  f.kind = kGrad; f.out_type = (int)type; f.unit = kColumnUnitInverse; f.rows = rows; f.cols = w.cin; f.row_factor = s.factor;
  f.out = d_dx; f.ldo = lddx;
  const Finish done = f;
  if (s.p.slices > 1) { f.kind = kPartial; f.partial = s.partial; }
  if (int rc = launch_gradient((int)type, w, s.p, st, a)) return rc;
  return s.p.slices > 1 ? launch_join(true, (int)type, s.p, s.partial, done, st) : SQUANT_OK;
}

size_t squant_cross_entropy_workspace_bytes(const void* d_h, int64_t ldh, squant_wtype_t type, int64_t rows, const squant_codes_t* h_w) {
  if (check_rows((int)type, rows) || check_codes(h_w) || rows == 0) return 0;
  LossSpace s;
  return lay_out_loss(nullptr, d_h, ldh, (int)type, rows, *h_w, s);
}

int squant_cross_entropy(const void* d_h, int64_t ldh, squant_wtype_t type, int64_t rows, const squant_codes_t* h_w,
                         const int64_t* d_labels, int64_t ignore_index, float* d_loss, float* d_lse, void* d_workspace,
                         size_t workspace_bytes, void* stream) {
  if (int rc = check_rows((int)type, rows)) return rc;
  if (int rc = check_codes(h_w)) return rc;
  const squant_codes_t& w = *h_w;
  if (ldh < w.cin) return SQUANT_ERR_SHAPE;
  if (rows == 0) return SQUANT_OK;
  if (!d_h || !d_labels || !d_loss || !d_lse) return SQUANT_ERR_NULL;
  if (misaligned(d_h, element_bytes((int)type)) || misaligned(d_labels, 8) || misaligned(d_loss, 4) || misaligned(d_lse, 4))
    return SQUANT_ERR_FORMAT;
  LossSpace s;
  const size_t need = lay_out_loss(d_workspace, d_h, ldh, (int)type, rows, w, s);
  if (!s.fit) return SQUANT_ERR_SHAPE;
  if (int rc = check_workspace(d_workspace, workspace_bytes, need)) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (int rc = lay_out(s.rows, s.copy, (int)type, st)) return rc;
  ProductArgs a{};
  set_product(a, s.x, s.w, w, s.p);
  Finish& f = a.f;
  f.kind = kStats; f.out_type = (int)type; f.unit = layer_unit((int)type, (int)w.format);
  f.rows = rows; f.cols = w.cout; f.row_factor = s.x.factor; f.scales = w.scales;
  f.labels = d_labels; f.stats = s.stats; f.label_logit = s.label_logit;
  if (int rc = launch_layer((int)type, w, s.p, st, a)) return rc;
  const LossArgs l{s.stats, (w.cout + kTile - 1) / kTile, s.label_logit, d_labels, ignore_index, w.cout, rows, d_loss, d_lse};
  return launch(loss_rows_kernel(), rows, 1, kRowThreads, 0, st, l);
}

size_t squant_cross_entropy_backward_workspace_bytes(const void* d_h, int64_t ldh, squant_wtype_t type, int64_t rows, const squant_codes_t* h_w) {
  if (check_rows((int)type, rows) || check_codes(h_w) || rows == 0) return 0;
  LossBackwardSpace s;
  return lay_out_loss_backward(nullptr, d_h, ldh, (int)type, rows, *h_w, s);
}

int squant_cross_entropy_backward(const void* d_h, int64_t ldh, squant_wtype_t type, int64_t rows, const squant_codes_t* h_w,
                                  const int64_t* d_labels, int64_t ignore_index, const float* d_lse, const float* d_dloss,
                                  void* d_dh, int64_t lddh, void* d_workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_rows((int)type, rows)) return rc;
  if (int rc = check_codes(h_w)) return rc;
  const squant_codes_t& w = *h_w;
  if (ldh < w.cin || lddh < w.cin) return SQUANT_ERR_SHAPE;
  if (rows == 0) return SQUANT_OK;
  if (!d_h || !d_labels || !d_lse || !d_dloss || !d_dh) return SQUANT_ERR_NULL;
  const int e = element_bytes((int)type), planes = planes_of((int)type);
  if (misaligned(d_h, e) || misaligned(d_dh, e) || misaligned(d_labels, 8) || misaligned(d_lse, 4) || misaligned(d_dloss, 4))
    return SQUANT_ERR_FORMAT;
  LossBackwardSpace s;
  const size_t need = lay_out_loss_backward(d_workspace, d_h, ldh, (int)type, rows, w, s);
  if (!s.fit) return SQUANT_ERR_SHAPE;
  if (int rc = check_workspace(d_workspace, workspace_bytes, need)) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (int rc = lay_out(s.rows, s.copy, (int)type, st)) return rc;
  hipLaunchKernelGGL(probability_unit_kernel(), dim3(1), dim3(1024), 0, st, w.scales, w.cout, s.unit);
  if (hipGetLastError() != hipSuccess) return SQUANT_ERR_DEVICE;
  for (int32_t i = 0; i < s.pieces; ++i) {
    const int32_t first = (int32_t)(i * s.piece);
    squant_codes_t piece = w;
    const CodeOperand codes{s.w.p + first * s.w.row, s.w.row};
    piece.cout = (int32_t)std::min<int64_t>(s.piece, w.cout - first);
    const Split p = split_layer(rows, piece.cout, w.cin, planes, (int)w.format, true, false);
    ProductArgs a{};
    set_product(a, s.x, codes, piece, p);
    Finish& f = a.f;
    f.kind = kProb; f.out_type = (int)type; f.unit = layer_unit((int)type, (int)w.format);
    f.rows = rows; f.cols = piece.cout; f.row_factor = s.x.factor; f.scales = w.scales + first;
    f.lse = d_lse; f.prob_unit = s.unit; f.prob = s.prob; f.ld_prob = planes * s.piece; f.prob_plane = s.piece;
    f.labels = d_labels; f.first_col = first; f.label_prob = s.label_prob; f.other_sums = s.other_sums;
    a.accumulate = i > 0;
    if (int rc = launch_layer((int)type, piece, p, st, a)) return rc;
    ProductArgs g{};
    Split split = s.g;
    split.blocks = (int32_t)((piece.cout + kBlock - 1) / kBlock);
    set_product(g, RowOperand{s.prob, planes * s.piece, s.piece, nullptr}, codes, piece, split);
    g.accumulate = i > 0;  // what a long batch needs beside its rows does not grow with the vocabulary
    g.f.kind = kPartial; g.f.rows = rows; g.f.cols = w.cin; g.f.partial = s.partial;
    if (int rc = launch_gradient((int)type, piece, split, st, g)) return rc;
  }
  Finish f{};
  f.kind = kGradLoss; f.out_type = (int)type; f.unit = kColumnUnitInverse; f.rows = rows; f.cols = w.cin; f.scales = w.scales;
  f.out = d_dh; f.ldo = lddh; f.labels = d_labels; f.ignore = ignore_index; f.dloss = d_dloss; f.prob_unit = s.unit;
  f.vocabulary = w.cout; f.label_prob = s.label_prob; f.other_sums = s.other_sums; f.other_tiles = s.other_tiles; f.codes = (const uint8_t*)w.codes; f.code_row = code_row(w); f.format = (int)w.format;
  return launch_join(true, (int)type, s.g, s.partial, f, st);
}

}  // extern "C"
