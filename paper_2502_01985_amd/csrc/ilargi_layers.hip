// C ABI of the operators of models with learned features: checks of the arguments, workspaces, sequences of kernels.
#include <stdarg.h>
#include <stdio.h>

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

struct LayerLayout {
  size_t forward = 0;                                         // bytes of the forward call
  size_t dz = 0, partial = 0, shares = 0, gradient = 0;       // offsets and bytes of the gradient call
};
size_t shares_bytes(bool h, int64_t M, int64_t N, int64_t K) {
  const size_t f = mm_f32_plan(M, N, K, 1).partial_bytes, m = h ? mm16_plan(M, N, K, 1, kMm16Bf16, 0).partial_bytes : 0;
  return up256(f > m ? f : m);
}
LayerLayout layer_layout(const ilargi_layer_t& y) {
  LayerLayout l;
  const bool h = y.type == ILARGI_TYPE_BF16;
  l.forward = mm_rows_takes(y.n, h) ? up256(mm_rows_plan(y.n, y.m, y.k).partial_bytes) : shares_bytes(h, y.n, y.m, y.k);
  l.dz = 0;
  l.partial = up256((size_t)y.n * (size_t)((y.m + 7) / 8 * 8) * (h ? 2 : 4));
  l.shares = l.partial + up256(layer_grad_partial_bytes(y.n, y.m));
  const size_t x = shares_bytes(h, y.n, y.k, y.m), w = shares_bytes(h, y.k, y.m, y.n);
  l.gradient = l.shares + (x > w ? x : w);
  return l;
}

// A product of the layer's matrices: bfloat16 operands that lie in whole 16-byte pieces on the 16-bit matrix cores, others in float32.
hipError_t product(const Product& p, float* partial, hipStream_t st) {
  if (p.P.bf16 && mm16_takes(p.P, p.M, p.K) && mm16_takes(p.Q, p.N, p.K)) {
    Product16 a{};
    a.P = {p.P.p, p.P.ld, p.P.k_rows, 0, 0, p.M};
    a.Q = {p.Q.p, p.Q.ld, p.Q.k_rows, 0, 0, p.N};
    a.M = p.M; a.N = p.N; a.K = p.K; a.batches = 1;
    a.kind = kMm16Bf16;
    a.epi = p.epi;
    return launch_mm16(a, mm16_plan(p.M, p.N, p.K, 1, kMm16Bf16, 0), partial, st);
  }
  return launch_mm_f32(p, mm_f32_plan(p.M, p.N, p.K, 1), partial, st);
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
  if (ilargi_status_t e = check_workspace("linear", workspace, workspace_bytes, layer_layout(y).forward); e != ILARGI_OK) return e;
  const int h = y.type == ILARGI_TYPE_BF16;
  Product p{};
  p.M = y.n; p.N = y.m; p.K = y.k; p.batches = 1;
  p.P = {X, ld_x, 0, h, 0};
  p.Q = {W, ld_w, 1, h, 0};
  p.epi.mode = kEpiLinear;
  p.epi.bias = bias; p.epi.src = residual; p.epi.ld_src = ld_res; p.epi.src_bf16 = h;
  p.epi.pre = pre; p.epi.ld_pre = ld_pre; p.epi.act = y.act;
  p.epi.out = out; p.epi.ld_out = ld_out; p.epi.out_bf16 = h;
  if (mm_rows_takes(y.n, h)) return done("linear", launch_mm_rows(p, mm_rows_plan(y.n, y.m, y.k), (float*)workspace, (hipStream_t)stream));
  return done("linear", product(p, (float*)workspace, (hipStream_t)stream));
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
  const bool products = d_X != nullptr || d_W != nullptr;
  void* dz = bent && products ? ws + l.dz : nullptr;
  LayerGradArgs g{y.n, y.m, d_out, ld_out, pre, ld_pre, y.act, h, dz, y.m, d_bias, accumulate};
  if (hipError_t e = launch_layer_grad(g, (float*)(ws + l.partial), st); e != hipSuccess) return done("linear_grad", e);
  const Operand z = {bent ? dz : d_out, bent ? y.m : ld_out, 0, h, 0};
  Product p{};
  p.batches = 1;
  p.epi.mode = kEpiScale;
  p.epi.s0 = 1.0f; p.epi.out_bf16 = h;
  if (d_X != nullptr) {
    p.M = y.n; p.N = y.k; p.K = y.m;
    p.P = z;
    p.Q = {W, ld_w, 0, h, 0};
    p.epi.out = d_X; p.epi.ld_out = ld_dx;
    if (hipError_t e = product(p, (float*)(ws + l.shares), st); e != hipSuccess) return done("linear_grad", e);
  }
  if (d_W != nullptr) {
    p.M = y.k; p.N = y.m; p.K = y.n;
    p.P = {X, ld_x, 1, h, 0};
    p.Q = z;
    p.Q.k_rows = 1;
    p.epi.out = d_W; p.epi.ld_out = ld_dw;
    if (accumulate) { p.epi.base = d_W; p.epi.s2 = 1.0f; }
    if (hipError_t e = product(p, (float*)(ws + l.shares), st); e != hipSuccess) return done("linear_grad", e);
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

}  // extern "C"
