// C ABI of the operators of models with learned features: checks of the arguments, workspaces, sequences of kernels.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <vector>

#include "ilargi_layers.h"

using namespace ilargi;

namespace {

constexpr int64_t kMost = 2147483647ll;

ilargi_status_t refuse(ilargi_status_t code, const char* fmt, ...) {
  char text[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  return set_error(code, text);
}

ilargi_status_t done(const char* what, hipError_t e) {
  return e == hipSuccess ? ILARGI_OK : refuse(ILARGI_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

bool is_type(int t) { return t == ILARGI_TYPE_F32 || t == ILARGI_TYPE_BF16; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

ilargi_status_t check_workspace(const char* what, const void* ws, size_t have, size_t need) {
  if (need == 0) return ILARGI_OK;
  if (ws == nullptr) return refuse(ILARGI_ERR_NULL, "%s: workspace is NULL", what);
  if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return refuse(ILARGI_ERR_WORKSPACE, "%s: workspace is not 256-byte aligned", what);
  if (have < need) return refuse(ILARGI_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", what, have, need);
  return ILARGI_OK;
}

ilargi_status_t check_rows(const char* what, int64_t n, int64_t rows, int64_t cols, int64_t ld_a, int64_t ld_b, int type_a, int type_b) {
  if (n < 0 || n > kMost || rows < 0 || rows > kMost) return refuse(ILARGI_ERR_SHAPE, "%s: n = %lld, rows = %lld", what, (long long)n, (long long)rows);
  if (cols < 1 || cols > kMost) return refuse(ILARGI_ERR_SHAPE, "%s: cols = %lld", what, (long long)cols);
  if (ld_a < cols || ld_b < cols) return refuse(ILARGI_ERR_SHAPE, "%s: a leading dimension below cols = %lld", what, (long long)cols);
  if (!is_type(type_a) || !is_type(type_b)) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: no such element type", what);
  return ILARGI_OK;
}

ilargi_status_t check_layer(const char* what, const ilargi_layer_t* y) {
  if (y == nullptr) return refuse(ILARGI_ERR_NULL, "%s: layer is NULL", what);
  if (y->n < 0 || y->n > kMost || y->k < 1 || y->k > kMost || y->m < 1 || y->m > kMost)
    return refuse(ILARGI_ERR_SHAPE, "%s: n = %lld, k = %lld, m = %lld", what, (long long)y->n, (long long)y->k, (long long)y->m);
  if (!is_type(y->type)) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: no such element type", what);
  if (y->act < ILARGI_ACT_NONE || y->act > ILARGI_ACT_GELU) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: no such activation", what);
  return ILARGI_OK;
}

size_t shares_bytes(bool h, int64_t M, int64_t N, int64_t K) {
  const size_t f = mm_f32_plan(M, N, K, 1).partial_bytes, m = h ? mm16_plan(M, N, K, 1, kMm16Bf16, 0).partial_bytes : 0;
  return up256(f > m ? f : m);
}

// Products of so many operations are formed on the 16-bit matrix cores also where an operand has to be laid out for them first: a
// launch of about 3 us and a pass over each operand, against 50 to 100 TFLOP/s on the float32 cores.  bfloat16 with odd rows, forward:
// 1003 x 701 x 1001 (1.4e9 operations) 31 us in float32; 2001 x 701 x 603 (1.7e9) 29 laid out; 4001 x 999 x 1001 (8e9) 36 laid out, 98
// in float32.
constexpr double kPackOps = 1.5e9;
bool worth_packing(int64_t n, int64_t k, int64_t m) { return 2.0 * (double)n * (double)k * (double)m >= kPackOps; }
int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }

struct LayerLayout {
  size_t x = 0, w = 0;                          // X and W laid out (bfloat16), in both calls
  size_t forward_shares = 0, forward = 0;       // the forward call's shares of k, and its bytes
  size_t dz = 0, partial = 0, shares = 0, gradient = 0;
};
LayerLayout layer_layout(const ilargi_layer_t& y) {
  LayerLayout l;
  const bool h = y.type == ILARGI_TYPE_BF16, few = mm_rows_takes(y.n, y.k, h);       // (few rows: W is read where it lies)
  size_t copies = 0;
  if (h && worth_packing(y.n, y.k, y.m)) {
    l.w = up256(2 * (size_t)y.n * (size_t)up8(y.k));
    copies = l.w + up256(2 * (size_t)y.k * (size_t)up8(y.m));
  }
  l.forward_shares = few ? 0 : copies;
  l.forward = l.forward_shares + (few ? up256(mm_rows_plan(y.n, y.m, y.k).partial_bytes) : shares_bytes(h, y.n, y.m, y.k));
  l.dz = copies;
  l.partial = l.dz + up256((size_t)y.n * (size_t)up8(y.m) * (h ? 2 : 4));
  l.shares = l.partial + up256(layer_grad_partial_bytes(y.n, y.m));
  const size_t x = shares_bytes(h, y.n, y.k, y.m), w = shares_bytes(h, y.k, y.m, y.n);
  l.gradient = l.shares + (x > w ? x : w);
  return l;
}

// A matrix of the layer as it lies, or laid out in whole 16-byte pieces.
struct Matrix {
  const void* p;
  int64_t ld, rows, cols;
};
bool in_pieces(const Matrix& m) { return reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.ld % 8 == 0 && m.ld < (1 << 22) && m.ld >= up8(m.cols); }

// C = P Q (or with one of them transposed) for two matrices of the layer; `padded` of each: zeros stand behind its rows.
struct Factor {
  Matrix m;
  int k_rows;
  bool padded;
};
hipError_t product(const Factor& P, const Factor& Q, int64_t M, int64_t N, int64_t K, bool h, const Epilogue& epi, float* partial, hipStream_t st) {
  auto ready = [&](const Factor& f) { return in_pieces(f.m) && (f.padded || f.m.cols % 8 == 0); };
  if (h && ready(P) && ready(Q)) {
    Product16 a{};
    auto operand = [&](const Factor& f, int64_t across) { return Operand16{f.m.p, f.m.ld, f.k_rows, 0, 0, f.k_rows ? up8(f.m.cols) : across}; };
    a.P = operand(P, M);
    a.Q = operand(Q, N);
    a.M = M; a.N = N; a.K = K; a.batches = 1;
    a.kind = kMm16Bf16;
    a.epi = epi;
    return launch_mm16(a, mm16_plan(M, N, K, 1, kMm16Bf16, 0), partial, st);
  }
  Product a{};
  a.P = {P.m.p, P.m.ld, P.k_rows, h, 0};
  a.Q = {Q.m.p, Q.m.ld, Q.k_rows, h, 0};
  a.M = M; a.N = N; a.K = K; a.batches = 1;
  a.epi = epi;
  return launch_mm_f32(a, mm_f32_plan(M, N, K, 1), partial, st);
}

// The matrix laid out at `at` if the layer's products are worth it and it does not lie so already.
hipError_t lay_out(const ilargi_layer_t& y, Factor* f, char* at, hipStream_t st) {
  if (y.type != ILARGI_TYPE_BF16 || !worth_packing(y.n, y.k, y.m) || (in_pieces(f->m) && f->m.cols % 8 == 0)) return hipSuccess;
  const hipError_t e = launch_pack16(f->m.p, f->m.ld, f->m.rows, f->m.cols, at, st);
  f->m.p = at;
  f->m.ld = up8(f->m.cols);
  f->padded = true;
  return e;
}

bool is_act(int f) { return f >= ILARGI_ACT_NONE && f <= ILARGI_ACT_GELU; }
bool is_norm(int k) { return k >= ILARGI_NORM_NONE && k <= ILARGI_NORM_CENTRED; }

ilargi_status_t check_norm(const char* what, const ilargi_norm_t* a) {
  if (a == nullptr) return refuse(ILARGI_ERR_NULL, "%s: block is NULL", what);
  if (a->n < 0 || a->n > kMost || a->m < 1 || a->m > kNormMostCols)
    return refuse(ILARGI_ERR_SHAPE, "%s: n = %lld, m = %lld", what, (long long)a->n, (long long)a->m);
  if (!is_type(a->type)) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: no such element type", what);
  if (!is_norm(a->first) || !is_norm(a->second)) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: no such norm", what);
  if (!is_act(a->gate_act)) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: no such activation", what);
  if (a->gate_rows != 0 && a->gate_rows != 1) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: gate_rows = %d", what, a->gate_rows);
  if (a->second == ILARGI_NORM_NONE && (a->gain2 != nullptr || a->bias2 != nullptr))
    return refuse(ILARGI_ERR_UNSUPPORTED, "%s: gain2 or bias2 without a second norm", what);
  if (!(a->eps >= 0.0f)) return refuse(ILARGI_ERR_SHAPE, "%s: eps = %g", what, (double)a->eps);
  if (a->ld_h < a->m || (a->gate != nullptr && a->gate_rows && a->ld_gate < a->m) || (a->x != nullptr && a->ld_x < a->m))
    return refuse(ILARGI_ERR_SHAPE, "%s: a leading dimension below m = %lld", what, (long long)a->m);
  if (a->n > 0 && a->h == nullptr) return refuse(ILARGI_ERR_NULL, "%s: h is NULL", what);
  return ILARGI_OK;
}

ilargi_status_t check_groups(const char* what, const ilargi_groups_t* y) {
  if (y == nullptr) return refuse(ILARGI_ERR_NULL, "%s: layer is NULL", what);
  if (y->groups < 0 || y->groups > 65535 || y->n < 0 || y->n > kMost || y->k < 1 || y->k > kMost || y->m < 1 || y->m > kMost)
    return refuse(ILARGI_ERR_SHAPE, "%s: groups = %lld, n = %lld, k = %lld, m = %lld", what, (long long)y->groups, (long long)y->n, (long long)y->k, (long long)y->m);
  if (!is_type(y->type)) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: no such element type", what);
  if (!is_act(y->act)) return refuse(ILARGI_ERR_UNSUPPORTED, "%s: no such activation", what);
  if (!grouped_blocks_fit(*y)) return refuse(ILARGI_ERR_SHAPE, "%s: too many blocks of results", what);
  return ILARGI_OK;
}
bool apart(const ilargi_groups_t& y, int64_t ld, int64_t stride) { return ld >= y.m && (y.groups <= 1 || stride >= (y.k - 1) * ld + y.m); }

// Where the matrices of a call lie: rows of `row` bytes, `step` bytes apart.
struct Range {
  const char *lo, *hi;
  int64_t rows, row, step;
  bool written;
};
Range range_of(const void* p, const ilargi_tensor_t& t, int64_t ld, bool written) {
  const int64_t size = t.type == ILARGI_TYPE_BF16 ? 2 : 4;
  return {(const char*)p, (const char*)p + ((t.rows - 1) * ld + t.cols) * size, t.rows, t.cols * size, ld * size, written};
}
// Column blocks of one matrix: they interleave and share no byte.  (a begins first.)
bool column_blocks(const Range& a, const Range& b) {
  if (a.rows > 1 && b.rows > 1 && a.step != b.step) return false;
  const int64_t step = a.rows > 1 ? a.step : b.step, at = (b.lo - a.lo) % step;
  return a.row <= at && at + b.row <= step;
}
bool overlapping(const ilargi_tensor_t* t, int64_t count, const float* norm) {
  std::vector<Range> all, open;
  if (norm != nullptr) all.push_back({(const char*)norm, (const char*)(norm + 1), 1, 4, 4, true});
  for (int64_t q = 0; q < count; ++q) {
    if (t[q].rows == 0 || t[q].cols == 0) continue;
    if (t[q].out != t[q].in) all.push_back(range_of(t[q].in, t[q], t[q].ld_in, false));
    if (t[q].out != nullptr) all.push_back(range_of(t[q].out, t[q], t[q].ld_out, true));
  }
  std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
  for (const Range& r : all) {
    size_t kept = 0;
    for (const Range& o : open)
      if (o.hi > r.lo) open[kept++] = o;
    open.resize(kept);
    for (const Range& o : open)
      if ((o.written || r.written) && !column_blocks(o, r)) return true;
    open.push_back(r);
  }
  return false;
}

ilargi_status_t check_tensors(const ilargi_tensor_t* t, int64_t count) {
  if (count < 0 || count > 65535) return refuse(ILARGI_ERR_SHAPE, "clip_norm: count = %lld", (long long)count);
  if (count > 0 && t == nullptr) return refuse(ILARGI_ERR_NULL, "clip_norm: tensors is NULL");
  for (int64_t q = 0; q < count; ++q) {
    if (!is_type(t[q].type)) return refuse(ILARGI_ERR_UNSUPPORTED, "clip_norm: tensor %lld is of no such element type", (long long)q);
    if (t[q].rows < 0 || t[q].rows > kMost || t[q].cols < 0 || t[q].cols > (1ll << 40))
      return refuse(ILARGI_ERR_SHAPE, "clip_norm: tensor %lld is %lld x %lld", (long long)q, (long long)t[q].rows, (long long)t[q].cols);
    const int64_t most = 1ll << 40, ld = std::max(t[q].ld_in, t[q].out != nullptr ? t[q].ld_out : 0);
    if (t[q].rows > 1 && ld > (1ll << 46) / t[q].rows)
      return refuse(ILARGI_ERR_SHAPE, "clip_norm: tensor %lld is %lld x %lld", (long long)q, (long long)t[q].rows, (long long)t[q].cols);
    if (t[q].ld_in < t[q].cols || t[q].ld_in > most || (t[q].out != nullptr && (t[q].ld_out < t[q].cols || t[q].ld_out > most)))
      return refuse(ILARGI_ERR_SHAPE, "clip_norm: a leading dimension of tensor %lld below its columns, or above 2^40", (long long)q);
    if (t[q].rows > 0 && t[q].cols > 0 && t[q].in == nullptr) return refuse(ILARGI_ERR_NULL, "clip_norm: tensor %lld is NULL", (long long)q);
    if (t[q].out == t[q].in && t[q].rows > 1 && t[q].cols > 0 && t[q].ld_out != t[q].ld_in)
      return refuse(ILARGI_ERR_SHAPE, "clip_norm: tensor %lld in place with another leading dimension", (long long)q);
  }
  return ILARGI_OK;
}

}  // namespace

extern "C" {

ilargi_status_t ilargi_embed(const void* table, ilargi_type_t table_type, int64_t rows, int64_t cols, int64_t ld_table, const int32_t* ids,
                             int64_t n, float scale, int accumulate, void* out, ilargi_type_t out_type, int64_t ld_out, void* stream) {
  if (ilargi_status_t e = check_rows("embed", n, rows, cols, ld_table, ld_out, table_type, out_type); e != ILARGI_OK) return e;
  if (n == 0) return ILARGI_OK;
  if (ids == nullptr || out == nullptr || (table == nullptr && rows > 0)) return refuse(ILARGI_ERR_NULL, "embed: table, ids or out is NULL");
  EmbedArgs a{table, rows, cols, ld_table, ids, n, scale, accumulate, out, ld_out, table_type == ILARGI_TYPE_BF16, out_type == ILARGI_TYPE_BF16};
  return done("embed", launch_embed(a, (hipStream_t)stream));
}

ilargi_status_t ilargi_embed_grad_workspace_bytes(int64_t n, int64_t rows, int64_t cols, size_t* bytes) {
  if (bytes == nullptr) return refuse(ILARGI_ERR_NULL, "embed_grad: bytes is NULL");
  if (ilargi_status_t e = check_rows("embed_grad", n, rows, cols, cols, cols, 0, 0); e != ILARGI_OK) return e;
  *bytes = embed_grad_bytes(n, cols);
  return ILARGI_OK;
}

ilargi_status_t ilargi_embed_grad(const void* d_out, ilargi_type_t out_type, int64_t ld_out, const int32_t* ids, int64_t n, float scale,
                                  int accumulate, void* d_table, ilargi_type_t table_type, int64_t rows, int64_t cols, int64_t ld_table,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  if (ilargi_status_t e = check_rows("embed_grad", n, rows, cols, ld_table, ld_out, table_type, out_type); e != ILARGI_OK) return e;
  if (rows == 0) return ILARGI_OK;
  if (d_table == nullptr || (n > 0 && (d_out == nullptr || ids == nullptr))) return refuse(ILARGI_ERR_NULL, "embed_grad: d_out, ids or d_table is NULL");
  if (ilargi_status_t e = check_workspace("embed_grad", workspace, workspace_bytes, embed_grad_bytes(n, cols)); e != ILARGI_OK) return e;
  EmbedGradArgs a{d_out, ld_out, ids, n, rows, cols, scale, accumulate, d_table, ld_table, out_type == ILARGI_TYPE_BF16, table_type == ILARGI_TYPE_BF16};
  return done("embed_grad", launch_embed_grad(a, (char*)workspace, (hipStream_t)stream));
}

ilargi_status_t ilargi_linear_workspace_bytes(const ilargi_layer_t* layer, size_t* forward, size_t* gradient) {
  if (ilargi_status_t e = check_layer("linear", layer); e != ILARGI_OK) return e;
  const LayerLayout l = layer_layout(*layer);
  if (forward != nullptr) *forward = l.forward;
  if (gradient != nullptr) *gradient = l.gradient;
  return ILARGI_OK;
}

ilargi_status_t ilargi_linear(const ilargi_layer_t* layer, const void* X, int64_t ld_x, const void* W, int64_t ld_w, const void* bias,
                              const void* residual, int64_t ld_res, void* out, int64_t ld_out, void* pre, int64_t ld_pre, void* workspace,
                              size_t workspace_bytes, void* stream) {
  if (ilargi_status_t e = check_layer("linear", layer); e != ILARGI_OK) return e;
  const ilargi_layer_t& y = *layer;
  if (ld_x < y.k || ld_w < y.m || ld_out < y.m || (residual != nullptr && ld_res < y.m) || (pre != nullptr && ld_pre < y.m))
    return refuse(ILARGI_ERR_SHAPE, "linear: a leading dimension below the matrix's columns");
  if (y.n == 0) return ILARGI_OK;
  if (X == nullptr || W == nullptr || out == nullptr) return refuse(ILARGI_ERR_NULL, "linear: X, W or out is NULL");
  const LayerLayout l = layer_layout(y);
  if (ilargi_status_t e = check_workspace("linear", workspace, workspace_bytes, l.forward); e != ILARGI_OK) return e;
  const int h = y.type == ILARGI_TYPE_BF16;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  Epilogue epi{};
  epi.mode = kEpiLinear;
  epi.bias = bias; epi.src = residual; epi.ld_src = ld_res; epi.src_bf16 = h;
  epi.pre = pre; epi.ld_pre = ld_pre; epi.act = y.act;
  epi.out = out; epi.ld_out = ld_out; epi.out_bf16 = h;
  if (mm_rows_takes(y.n, y.k, h)) {
    Product p{};
    p.M = y.n; p.N = y.m; p.K = y.k; p.batches = 1;
    p.P = {X, ld_x, 0, h, 0};
    p.Q = {W, ld_w, 1, h, 0};
    p.epi = epi;
    return done("linear", launch_mm_rows(p, mm_rows_plan(y.n, y.m, y.k), (float*)(ws + l.forward_shares), st));
  }
  Factor x{{X, ld_x, y.n, y.k}, 0, false}, w{{W, ld_w, y.k, y.m}, 1, false};
  if (hipError_t e = lay_out(y, &x, ws + l.x, st); e != hipSuccess) return done("linear", e);
  if (hipError_t e = lay_out(y, &w, ws + l.w, st); e != hipSuccess) return done("linear", e);
  return done("linear", product(x, w, y.n, y.m, y.k, h, epi, (float*)(ws + l.forward_shares), st));
}

ilargi_status_t ilargi_linear_grad(const ilargi_layer_t* layer, const void* d_out, int64_t ld_out, const void* pre, int64_t ld_pre,
                                   const void* X, int64_t ld_x, const void* W, int64_t ld_w, void* d_X, int64_t ld_dx, void* d_W,
                                   int64_t ld_dw, void* d_bias, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (ilargi_status_t e = check_layer("linear_grad", layer); e != ILARGI_OK) return e;
  const ilargi_layer_t& y = *layer;
  const bool bent = y.act != ILARGI_ACT_NONE;
  if (ld_out < y.m || (bent && ld_pre < y.m) || (d_W != nullptr && (ld_x < y.k || ld_dw < y.m)) || (d_X != nullptr && (ld_w < y.m || ld_dx < y.k)))
    return refuse(ILARGI_ERR_SHAPE, "linear_grad: a leading dimension below the matrix's columns");
  if (y.n > 0 && (d_out == nullptr || (bent && pre == nullptr) || (d_W != nullptr && X == nullptr) || (d_X != nullptr && W == nullptr)))
    return refuse(ILARGI_ERR_NULL, "linear_grad: d_out, pre, X or W is NULL");
  const LayerLayout l = layer_layout(y);
  if (ilargi_status_t e = check_workspace("linear_grad", workspace, workspace_bytes, l.gradient); e != ILARGI_OK) return e;
  const int h = y.type == ILARGI_TYPE_BF16;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  float* shares = (float*)(ws + l.shares);
  const bool products = d_X != nullptr || d_W != nullptr;
  Factor z{{d_out, ld_out, y.n, y.m}, 0, false};
  // g, where it is not d_out itself, or d_out does not lie in pieces and the products are worth it
  if (products && (bent || (h && worth_packing(y.n, y.k, y.m) && !(in_pieces(z.m) && y.m % 8 == 0)))) {
    z.m.p = ws + l.dz;
    z.m.ld = up8(y.m);
    z.padded = true;
  }
  LayerGradArgs g{y.n, y.m, d_out, ld_out, pre, ld_pre, y.act, h, z.padded ? ws + l.dz : nullptr, up8(y.m), d_bias, accumulate};
  if (hipError_t e = launch_layer_grad(g, (float*)(ws + l.partial), st); e != hipSuccess) return done("linear_grad", e);
  Epilogue epi{};
  epi.mode = kEpiLinear;
  epi.out_bf16 = h;
  if (d_X != nullptr) {
    Factor w{{W, ld_w, y.k, y.m}, 0, false};
    if (hipError_t e = lay_out(y, &w, ws + l.w, st); e != hipSuccess) return done("linear_grad", e);
    epi.out = d_X; epi.ld_out = ld_dx;
    if (hipError_t e = product(z, w, y.n, y.k, y.m, h, epi, shares, st); e != hipSuccess) return done("linear_grad", e);
  }
  if (d_W != nullptr) {
    Factor x{{X, ld_x, y.n, y.k}, 1, false};
    if (hipError_t e = lay_out(y, &x, ws + l.x, st); e != hipSuccess) return done("linear_grad", e);
    z.k_rows = 1;
    epi.out = d_W; epi.ld_out = ld_dw;
    if (accumulate) { epi.src = d_W; epi.ld_src = ld_dw; epi.src_bf16 = h; }
    if (hipError_t e = product(x, z, y.k, y.m, y.n, h, epi, shares, st); e != hipSuccess) return done("linear_grad", e);
  }
  return ILARGI_OK;
}

ilargi_status_t ilargi_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, ilargi_type_t g_type, size_t* bytes) {
  if (bytes == nullptr) return refuse(ILARGI_ERR_NULL, "orthogonalize: bytes is NULL");
  if (batch < 0 || batch > 65535 || rows < 1 || rows > 16384 || cols < 1 || cols > 16384)
    return refuse(ILARGI_ERR_SHAPE, "orthogonalize: batch = %lld, rows = %lld, cols = %lld", (long long)batch, (long long)rows, (long long)cols);
  if (!is_type(g_type)) return refuse(ILARGI_ERR_UNSUPPORTED, "orthogonalize: no such element type");
  *bytes = ortho_bytes(batch, rows, cols);
  return ILARGI_OK;
}

ilargi_status_t ilargi_orthogonalize(const void* G, ilargi_type_t g_type, int64_t batch, int64_t rows, int64_t cols, int64_t ld_g,
                                     int64_t stride_g, int steps, const float* coef, float eps, float alpha, float beta, const void* base,
                                     void* out, ilargi_type_t out_type, int64_t ld_out, int64_t stride_out, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  size_t need = 0;
  if (ilargi_status_t e = ilargi_orthogonalize_workspace_bytes(batch, rows, cols, g_type, &need); e != ILARGI_OK) return e;
  if (!is_type(out_type)) return refuse(ILARGI_ERR_UNSUPPORTED, "orthogonalize: no such element type");
  if (steps < 1 || steps > 100) return refuse(ILARGI_ERR_SHAPE, "orthogonalize: steps = %d outside [1, 100]", steps);
  if (ld_g < cols || ld_out < cols) return refuse(ILARGI_ERR_SHAPE, "orthogonalize: a leading dimension below cols = %lld", (long long)cols);
  if (batch > 1 && (stride_g < (rows - 1) * ld_g + cols || stride_out < (rows - 1) * ld_out + cols))
    return refuse(ILARGI_ERR_SHAPE, "orthogonalize: matrices of the batch overlap");
  if (batch == 0) return ILARGI_OK;
  if (G == nullptr || out == nullptr) return refuse(ILARGI_ERR_NULL, "orthogonalize: G or out is NULL");
  if (beta != 0.0f && base == nullptr) return refuse(ILARGI_ERR_NULL, "orthogonalize: beta is not 0 and base is NULL");
  if (ilargi_status_t e = check_workspace("orthogonalize", workspace, workspace_bytes, need); e != ILARGI_OK) return e;
  OrthoArgs a{};
  a.G = G; a.batch = batch; a.rows = rows; a.cols = cols; a.ld_g = ld_g; a.batch_g = stride_g; a.g_bf16 = g_type == ILARGI_TYPE_BF16;
  a.steps = steps;
  const float usual[3] = {3.4445f, -4.7750f, 2.0315f};
  for (int q = 0; q < 3; ++q) a.coef[q] = coef != nullptr ? coef[q] : usual[q];
  a.eps = eps; a.alpha = alpha; a.beta = beta; a.base = base;
  a.out = out; a.ld_out = ld_out; a.batch_out = stride_out; a.out_bf16 = out_type == ILARGI_TYPE_BF16;
  return done("orthogonalize", launch_ortho(a, (char*)workspace, (hipStream_t)stream));
}

ilargi_status_t ilargi_norm(const ilargi_norm_t* block, void* r, int64_t ld_r, void* y, int64_t ld_y, void* stream) {
  if (ilargi_status_t e = check_norm("norm", block); e != ILARGI_OK) return e;
  if (y != nullptr && block->second == ILARGI_NORM_NONE) return refuse(ILARGI_ERR_UNSUPPORTED, "norm: y without a second norm");
  if ((r != nullptr && ld_r < block->m) || (y != nullptr && ld_y < block->m))
    return refuse(ILARGI_ERR_SHAPE, "norm: a leading dimension below m = %lld", (long long)block->m);
  if (block->n == 0 || (r == nullptr && y == nullptr)) return ILARGI_OK;
  ilargi_norm_t a = *block;
  if (a.gate == nullptr) a.gate_rows = 0;               // (no gate has no rows)
  return done("norm", launch_norm(a, r, ld_r, y, ld_y, (hipStream_t)stream));
}

ilargi_status_t ilargi_norm_grad_workspace_bytes(int64_t n, int64_t m, ilargi_type_t type, size_t* bytes) {
  if (bytes == nullptr) return refuse(ILARGI_ERR_NULL, "norm_grad: bytes is NULL");
  if (n < 0 || n > kMost || m < 1 || m > kNormMostCols) return refuse(ILARGI_ERR_SHAPE, "norm_grad: n = %lld, m = %lld", (long long)n, (long long)m);
  if (!is_type(type)) return refuse(ILARGI_ERR_UNSUPPORTED, "norm_grad: no such element type");
  *bytes = norm_grad_bytes(n, m, type == ILARGI_TYPE_BF16);
  return ILARGI_OK;
}

ilargi_status_t ilargi_norm_grad(const ilargi_norm_t* block, const void* d_r, int64_t ld_dr, const void* d_y, int64_t ld_dy,
                                 const ilargi_norm_grads_t* out, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (ilargi_status_t e = check_norm("norm_grad", block); e != ILARGI_OK) return e;
  if (out == nullptr) return refuse(ILARGI_ERR_NULL, "norm_grad: out is NULL");
  ilargi_norm_t a = *block;
  if (a.gate == nullptr) a.gate_rows = 0;
  const bool second = a.second != ILARGI_NORM_NONE;
  if (!second && (d_y != nullptr || out->d_gain2 != nullptr || out->d_bias2 != nullptr))
    return refuse(ILARGI_ERR_UNSUPPORTED, "norm_grad: d_y, d_gain2 or d_bias2 without a second norm");
  if (out->d_gate != nullptr && a.gate == nullptr) return refuse(ILARGI_ERR_UNSUPPORTED, "norm_grad: d_gate without a gate");
  if ((d_r != nullptr && ld_dr < a.m) || (d_y != nullptr && ld_dy < a.m) || (out->d_h != nullptr && out->ld_h < a.m) ||
      (out->d_x != nullptr && out->ld_x < a.m) || (out->d_gate != nullptr && a.gate_rows && out->ld_gate < a.m))
    return refuse(ILARGI_ERR_SHAPE, "norm_grad: a leading dimension below m = %lld", (long long)a.m);
  if ((out->d_gate != nullptr && !a.gate_rows) || out->d_gain1 != nullptr || out->d_bias1 != nullptr || out->d_gain2 != nullptr || out->d_bias2 != nullptr)
    if (ilargi_status_t e = check_workspace("norm_grad", workspace, workspace_bytes, norm_grad_bytes(a.n, a.m, a.type == ILARGI_TYPE_BF16)); e != ILARGI_OK) return e;
  return done("norm_grad", launch_norm_grad(a, d_r, ld_dr, d_y, ld_dy, *out, accumulate, (float*)workspace, (hipStream_t)stream));
}

ilargi_status_t ilargi_grouped_linear_workspace_bytes(const ilargi_groups_t* layer, size_t* forward, size_t* gradient) {
  if (ilargi_status_t e = check_groups("grouped_linear", layer); e != ILARGI_OK) return e;
  grouped_bytes(*layer, forward, gradient);
  return ILARGI_OK;
}

ilargi_status_t ilargi_grouped_linear(const ilargi_groups_t* layer, const int32_t* offsets, const void* X, int64_t ld_x, const void* W, int64_t ld_w,
                                      int64_t stride_w, const void* bias, int64_t ld_bias, const void* residual, int64_t ld_res, void* out,
                                      int64_t ld_out, void* pre, int64_t ld_pre, void* workspace, size_t workspace_bytes, void* stream) {
  if (ilargi_status_t e = check_groups("grouped_linear", layer); e != ILARGI_OK) return e;
  const ilargi_groups_t& y = *layer;
  if (ld_x < y.k || ld_out < y.m || (bias != nullptr && ld_bias < y.m) || (residual != nullptr && ld_res < y.m) || (pre != nullptr && ld_pre < y.m))
    return refuse(ILARGI_ERR_SHAPE, "grouped_linear: a leading dimension below the matrix's columns");
  if (!apart(y, ld_w, stride_w)) return refuse(ILARGI_ERR_SHAPE, "grouped_linear: matrices of the groups overlap");
  if (y.n == 0 || y.groups == 0) return ILARGI_OK;
  if (offsets == nullptr || X == nullptr || W == nullptr || out == nullptr) return refuse(ILARGI_ERR_NULL, "grouped_linear: offsets, X, W or out is NULL");
  size_t need = 0;
  grouped_bytes(y, &need, nullptr);
  if (ilargi_status_t e = check_workspace("grouped_linear", workspace, workspace_bytes, need); e != ILARGI_OK) return e;
  GroupedArgs a{};
  a.y = y; a.offsets = offsets;
  a.X = X; a.ld_x = ld_x; a.W = W; a.ld_w = ld_w; a.stride_w = y.groups > 1 ? stride_w : 0;
  a.bias = bias; a.ld_bias = ld_bias; a.residual = residual; a.ld_res = ld_res;
  a.out = out; a.ld_out = ld_out; a.pre = pre; a.ld_pre = ld_pre;
  return done("grouped_linear", launch_grouped(a, (char*)workspace, (hipStream_t)stream));
}

ilargi_status_t ilargi_grouped_linear_grad(const ilargi_groups_t* layer, const int32_t* offsets, const void* d_out, int64_t ld_out, const void* pre,
                                           int64_t ld_pre, const void* X, int64_t ld_x, const void* W, int64_t ld_w, int64_t stride_w, void* d_X,
                                           int64_t ld_dx, void* d_W, int64_t ld_dw, int64_t stride_dw, void* d_bias, int64_t ld_dbias, int accumulate,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  if (ilargi_status_t e = check_groups("grouped_linear_grad", layer); e != ILARGI_OK) return e;
  const ilargi_groups_t& y = *layer;
  const bool bent = y.act != ILARGI_ACT_NONE;
  if (ld_out < y.m || (bent && ld_pre < y.m) || (d_W != nullptr && ld_x < y.k) || (d_X != nullptr && ld_dx < y.k) || (d_bias != nullptr && ld_dbias < y.m))
    return refuse(ILARGI_ERR_SHAPE, "grouped_linear_grad: a leading dimension below the matrix's columns");
  if ((d_X != nullptr && !apart(y, ld_w, stride_w)) || (d_W != nullptr && !apart(y, ld_dw, stride_dw)))
    return refuse(ILARGI_ERR_SHAPE, "grouped_linear_grad: matrices of the groups overlap");
  if (y.groups == 0 || (d_X == nullptr && d_W == nullptr && d_bias == nullptr)) return ILARGI_OK;
  if (offsets == nullptr || (y.n > 0 && (d_out == nullptr || (bent && pre == nullptr) || (d_W != nullptr && X == nullptr) || (d_X != nullptr && W == nullptr))))
    return refuse(ILARGI_ERR_NULL, "grouped_linear_grad: offsets, d_out, pre, X or W is NULL");
  size_t need = 0;
  grouped_bytes(y, nullptr, &need);
  if (ilargi_status_t e = check_workspace("grouped_linear_grad", workspace, workspace_bytes, need); e != ILARGI_OK) return e;
  GroupedArgs a{};
  a.y = y; a.offsets = offsets;
  a.d_out = d_out; a.ld_dout = ld_out; a.pre_in = pre;
  a.X = X; a.ld_x = ld_x; a.W = W; a.ld_w = ld_w; a.stride_w = y.groups > 1 ? stride_w : 0;
  a.ld_pre = ld_pre; a.d_X = d_X; a.ld_dx = ld_dx; a.d_W = d_W; a.ld_dw = ld_dw; a.stride_dw = y.groups > 1 ? stride_dw : 0;
  a.d_bias = d_bias; a.ld_dbias = ld_dbias; a.accumulate = accumulate;
  return done("grouped_linear_grad", launch_grouped_grad(a, (char*)workspace, (hipStream_t)stream));
}

ilargi_status_t ilargi_clip_norm_workspace_bytes(const ilargi_tensor_t* tensors, int64_t count, size_t* bytes) {
  if (bytes == nullptr) return refuse(ILARGI_ERR_NULL, "clip_norm: bytes is NULL");
  if (ilargi_status_t e = check_tensors(tensors, count); e != ILARGI_OK) return e;
  *bytes = clip_bytes(tensors, count);
  return ILARGI_OK;
}

ilargi_status_t ilargi_clip_norm(const ilargi_tensor_t* tensors, int64_t count, float max_norm, float* norm, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  if (ilargi_status_t e = check_tensors(tensors, count); e != ILARGI_OK) return e;
  if (!(max_norm >= 0.0f)) return refuse(ILARGI_ERR_SHAPE, "clip_norm: max_norm = %g", (double)max_norm);
  try {
    if (overlapping(tensors, count, norm)) return refuse(ILARGI_ERR_SHAPE, "clip_norm: an output or the norm overlaps another tensor");
  } catch (...) {
    return refuse(ILARGI_ERR_DEVICE, "clip_norm: out of host memory");
  }
  if (ilargi_status_t e = check_workspace("clip_norm", workspace, workspace_bytes, clip_bytes(tensors, count)); e != ILARGI_OK) return e;
  return done("clip_norm", launch_clip(tensors, count, max_norm, norm, (double*)workspace, (hipStream_t)stream));
}

}  // extern "C"
