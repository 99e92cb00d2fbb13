// Orthogonalised updates: X = G / (|G|_F + eps), then steps of X <- a X + (b A + c A^2) X with A = X X^T.
//
// X is held with its short side as rows (G transposed where it is the taller), so A and B = b A + c A^2 are as small as they can be, and
// symmetric: blocks on and above the diagonal are formed and written twice.  A step's small singular directions are multiplied by up
// to a = 3.4, so a rounding of the first step grows 140-fold by the fifth: X, A and B are held as pairs of float16 planes (22 bits)
// and every product is three on the 16-bit matrix cores.  The result is as near to 64 bits as float32 products bring it (2048 x
// 2048: 1.1e-6, those 2.8e-6); single float16 planes are off by 1e-3 to 2e-2, single planes in the last step alone by up to 2e-3,
// which with bfloat16's own 1.7e-3 is too much.  Bound by the matrix cores and, below about 1000, by the chain of launches: 2048 x
// 2048, float32, 786 us (218 TFLOP/s of the formula's operations, those of symmetric products counted once, and three times that in
// products); 1024 x 4096, bfloat16, 401 us.
#include <math.h>

#include "mm_epilogue.h"

namespace ilargi {

namespace {

constexpr int kNormParts = 256, kMostSteps = 100;

// The pairs hold kUnit 2^e X (ortho_exponent) and kUnit A, and B times a power of two that brings it to at most 60000 (float16 ends at
// 65504): their low planes then count in 1.5e-11 of A and of an X of norm 1.  (What A and B lose of a small X is small against the
// identity that a X stands for.)
constexpr float kUnit = 4096.0f;

// Sums of squares of a share of one matrix's rows, in 64 bits: the norm neither overflows nor loses small entries.
template <class T>
__global__ __launch_bounds__(256) void ortho_norm_kernel(OrthoArgs a, double* __restrict__ parts) {
  constexpr int V = ElemOf<T>::kVec;
  __shared__ double wsum[4];
  const T* G = (const T*)a.G + blockIdx.y * a.batch_g;
  const int64_t pieces = (a.cols + V - 1) / V, total = a.rows * pieces;
  double s = 0.0;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += kNormParts * 256) {
    const int64_t r = (uint32_t)at / (uint32_t)pieces, c = (at - r * pieces) * V;     // (at most 2^26 pieces)
    float f[V];
    load_piece<T, V>(G + r * a.ld_g + c, (int)(a.cols - c < V ? a.cols - c : V), f);
#pragma unroll
    for (int q = 0; q < V; ++q) s = fma((double)f[q], (double)f[q], s);
  }
  for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
  if (threadIdx.x % 64 == 0) wsum[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.y * kNormParts + blockIdx.x] = (wsum[0] + wsum[1]) + (wsum[2] + wsum[3]);
}

// X (short side x long side) = G or its transpose over the norm, 32 x 32 tiles through LDS; zeros up to `rows_x` x `ld_x`.
// In pairs of float16 planes, X is held times kUnit 2^e; then `by` receives, for every step and matrix, 2^-2e of X X^T and behind them the
// change of 2^e to the next step, of the last step to 1.
template <class T, bool PAIRS>
__global__ __launch_bounds__(256) void ortho_load_kernel(OrthoArgs a, const double* __restrict__ parts, void* __restrict__ out, int64_t rows_x, int64_t ld_x,
                                                         int tiles_c, float lg_grow, float* __restrict__ by) {
  __shared__ float tile[32][33];
  __shared__ Factor2 scale;
  const int64_t b = blockIdx.y;
  if (threadIdx.x < 64) {
    const double* p = parts + b * kNormParts + threadIdx.x;
    double s = (p[0] + p[64]) + (p[128] + p[192]);
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    const double norm = sqrt(s), one = 1.0 / (norm + (double)a.eps);
    const float lg_norm = PAIRS ? lg_of(norm * one) : 0.0f;
    if (threadIdx.x == 0) scale = factor2(PAIRS ? ldexp(one * (double)kUnit, ortho_exponent(lg_norm, lg_grow, 0)) : one);
    if (PAIRS && blockIdx.x == 0)
      for (int t = threadIdx.x; t < a.steps; t += 64) {
        const int up = ortho_exponent(lg_norm, lg_grow, t), then = t + 1 < a.steps ? ortho_exponent(lg_norm, lg_grow, t + 1) : 0;
        by[(2 * t) * a.batch + b] = ldexpf(1.0f, -2 * up);
        by[(2 * t + 1) * a.batch + b] = ldexpf(1.0f, then - up);
      }
  }
  const T* G = (const T*)a.G + b * a.batch_g;
  const bool flip = a.rows > a.cols;
  const int64_t y0 = (int64_t)(blockIdx.x / tiles_c) * 32, x0 = (int64_t)(blockIdx.x % tiles_c) * 32;     // of X
  const int64_t r0 = flip ? x0 : y0, c0 = flip ? y0 : x0;                                                 // of G
  const int x = threadIdx.x % 32, y = threadIdx.x / 32;
#pragma unroll
  for (int q = 0; q < 32; q += 8) {
    const int64_t r = r0 + y + q, c = c0 + x;
    tile[y + q][x] = r < a.rows && c < a.cols ? (float)G[r * a.ld_g + c] : 0.0f;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 32; q += 8) {
    if (y0 + y + q >= rows_x || x0 + x >= ld_x) continue;
    const int64_t at = (b * rows_x + y0 + y + q) * ld_x + x0 + x;
    const float v = times(flip ? tile[x][y + q] : tile[y + q][x], scale);
    if constexpr (PAIRS) pair_store((_Float16*)out, at, a.batch * rows_x * ld_x, v);
    else ((float*)out)[at] = v;
  }
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Whether the iteration stays where pairs of float16 hold it: some interval [0, R], R <= 2, that holds the first singular values (at
// most 1) is mapped into [-R, R] by p(s) = s (a + b s^2 + c s^4).  Then the entries of X are at most R, of A R^2, and of B |b| R^2 +
// |c| R^4, which gives B's unit (0: it does not stay); and a step multiplies a singular value by at most `grow`.
struct PairRange {
  float unit_b;
  double grow;
};
PairRange pair_range(const float* coef) {
  const double a = coef[0], b = coef[1], c = coef[2];
  auto size = [](double v) { return v < 0 ? -v : v; };
  auto factor = [&](double x) { return a + b * x + c * x * x; };                  // p(s) / s at s^2 = x
  // where p and p / s have their extremes besides the ends: 5 c x^2 + 3 b x + a = 0, 2 c x + b = 0
  const double root = sqrt(9 * b * b - 20 * a * c);
  const double turns[3] = {c != 0 ? (-3 * b + root) / (10 * c) : -a / (3 * b), c != 0 ? (-3 * b - root) / (10 * c) : 0.0, -b / (2 * c)};
  for (int q = 0; q <= 40; ++q) {
    const double R = 1.0 + 0.025 * q;
    double top = size(R * factor(R * R)), grow = size(factor(R * R));
    if (!(grow >= size(a))) grow = size(a);
    for (double x : turns) {
      if (!(x > 0 && x < R * R)) continue;
      const double f = size(factor(x));
      if (sqrt(x) * f > top) top = sqrt(x) * f;
      if (f > grow) grow = f;
    }
    if (!(top <= R)) continue;
    const double most = size(b) * R * R + size(c) * R * R * R * R;
    double unit = 4096.0;
    while (unit > 1.0 && unit * most > 60000.0) unit /= 2.0;
    return {unit * most <= 60000.0 ? (float)unit : 0.0f, grow};
  }
  return {0.0f, 0.0};
}

struct OrthoLayout {
  int64_t s, l, sp, lp;                 // short and long side, and the same up to a multiple of 8
  MmPlan gram, square, apply;
  size_t by, x[2], A, B, partial, most, total;
};
OrthoLayout ortho_layout(int64_t batch, int64_t rows, int64_t cols) {
  OrthoLayout o{};
  o.s = rows < cols ? rows : cols;
  o.l = rows < cols ? cols : rows;
  o.sp = (o.s + 7) / 8 * 8;
  o.lp = (o.l + 7) / 8 * 8;
  o.gram = mm16_plan(o.sp, o.sp, o.lp, batch, kMm16Pairs, 1);
  o.square = mm16_plan(o.sp, o.sp, o.sp, batch, kMm16Pairs, 1);
  o.apply = mm16_plan(o.sp, o.lp, o.sp, batch, kMm16Pairs, 0);
  size_t at = up256((size_t)batch * kNormParts * 8);
  auto take = [&at](size_t bytes) { const size_t p = at; at += up256(bytes); return p; };
  o.by = take(4 * 2 * (size_t)kMostSteps * (size_t)batch);
  o.x[0] = take(4 * (size_t)(batch * o.sp * o.lp));
  o.x[1] = take(4 * (size_t)(batch * o.sp * o.lp));
  o.A = take(4 * (size_t)(batch * o.sp * o.sp));
  o.B = take(4 * (size_t)(batch * o.sp * o.sp));
  o.most = o.gram.partial_bytes;
  if (o.square.partial_bytes > o.most) o.most = o.square.partial_bytes;
  if (o.apply.partial_bytes > o.most) o.most = o.apply.partial_bytes;
  o.partial = take(o.most);
  o.total = at;
  return o;
}

// The last product of the last step writes the result.
void finish(const OrthoArgs& a, float unit, Epilogue* e) {
  e->s0 *= a.alpha / unit;
  e->s1 *= a.alpha / unit;
  e->s2 = a.beta;
  e->base = a.beta != 0.0f ? a.base : nullptr;
  e->out = a.out; e->ld_out = a.ld_out; e->batch_out = a.batch_out; e->out_bf16 = a.out_bf16; e->out_plane = 0;
  e->flip = a.rows > a.cols;
}

hipError_t iterate_pairs(const OrthoArgs& a, const OrthoLayout& o, float unit_b, char* ws, hipStream_t st) {
  float* partial = (float*)(ws + o.partial);
  const int64_t px = a.batch * o.sp * o.lp, pa = a.batch * o.sp * o.sp;
  void *A = ws + o.A, *B = ws + o.B;
  for (int t = 0; t < a.steps; ++t) {
    void *x = ws + o.x[t & 1], *next = ws + o.x[(t & 1) ^ 1];
    Product16 p{};
    p.kind = kMm16Pairs;
    p.batches = a.batch;
    p.M = o.sp; p.N = o.sp; p.K = o.lp; p.symmetric = 1;
    p.P = {x, o.lp, 0, o.sp * o.lp, px, o.sp};
    p.Q = p.P;
    p.epi.mode = kEpiScale;
    p.epi.s0 = 1.0f / kUnit;
    p.epi.by = (const float*)(ws + o.by) + 2 * t * a.batch;
    p.epi.out = A; p.epi.ld_out = o.sp; p.epi.batch_out = o.sp * o.sp; p.epi.out_plane = pa;
    if (hipError_t e = launch_mm16(p, o.gram, partial, st); e != hipSuccess) return e;
    p.K = o.sp;
    p.P = {A, o.sp, 0, o.sp * o.sp, pa, o.sp};
    p.Q = p.P;
    p.epi.s0 = a.coef[2] * unit_b / (kUnit * kUnit); p.epi.s1 = a.coef[1] * unit_b / kUnit;
    p.epi.src = A; p.epi.ld_src = o.sp; p.epi.batch_src = o.sp * o.sp; p.epi.src_plane = pa;
    p.epi.by = nullptr;
    p.epi.out = B;
    if (hipError_t e = launch_mm16(p, o.square, partial, st); e != hipSuccess) return e;
    p.N = o.lp; p.symmetric = 0;
    p.P.p = B;
    p.Q = {x, o.lp, 1, o.sp * o.lp, px, o.lp};
    p.epi.s0 = 1.0f / unit_b; p.epi.s1 = a.coef[0];
    p.epi.src = x; p.epi.ld_src = o.lp; p.epi.batch_src = o.sp * o.lp; p.epi.src_plane = px;
    p.epi.by = (const float*)(ws + o.by) + (2 * t + 1) * a.batch;
    p.epi.out = next; p.epi.ld_out = o.lp; p.epi.batch_out = o.sp * o.lp; p.epi.out_plane = px;
    if (t + 1 == a.steps) {
      finish(a, kUnit, &p.epi);
      p.M = o.s; p.N = o.l;
    }
    if (hipError_t e = launch_mm16(p, o.apply, partial, st); e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t iterate_f32(const OrthoArgs& a, const OrthoLayout& o, char* ws, hipStream_t st) {
  float *A = (float*)(ws + o.A), *B = (float*)(ws + o.B);
  const int64_t s = o.s, l = o.l;
  auto form = [&](const Product& p) {
    MmPlan plan = mm_f32_plan(p.M, p.N, p.K, p.batches);
    if (plan.partial_bytes > o.most) plan = {128, 1, 0};         // (the workspace is as large as the products of pairs have it)
    return launch_mm_f32(p, plan, (float*)(ws + o.partial), st);
  };
  for (int t = 0; t < a.steps; ++t) {
    float *x = (float*)(ws + o.x[t & 1]), *next = (float*)(ws + o.x[(t & 1) ^ 1]);
    Product p{};
    p.M = s; p.N = s; p.K = l; p.batches = a.batch;
    p.P = {x, l, 0, 0, s * l};
    p.Q = p.P;
    p.epi.mode = kEpiScale;
    p.epi.s0 = 1.0f; p.epi.out = A; p.epi.ld_out = s; p.epi.batch_out = s * s;
    if (hipError_t e = form(p); e != hipSuccess) return e;
    p.K = s;
    p.P = {A, s, 0, 0, s * s};
    p.Q = p.P;
    p.epi.s0 = a.coef[2]; p.epi.s1 = a.coef[1];
    p.epi.src = A; p.epi.ld_src = s; p.epi.batch_src = s * s;
    p.epi.out = B;
    if (hipError_t e = form(p); e != hipSuccess) return e;
    p.N = l;
    p.P.p = B;
    p.Q = {x, l, 1, 0, s * l};
    p.epi.s0 = 1.0f; p.epi.s1 = a.coef[0];
    p.epi.src = x; p.epi.ld_src = l; p.epi.batch_src = s * l;
    p.epi.out = next; p.epi.ld_out = l; p.epi.batch_out = s * l;
    if (t + 1 == a.steps) finish(a, 1.0f, &p.epi);
    if (hipError_t e = form(p); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t ortho_typed(const OrthoArgs& a, char* ws, hipStream_t st) {
  const OrthoLayout o = ortho_layout(a.batch, a.rows, a.cols);
  double* parts = (double*)ws;
  const PairRange range = pair_range(a.coef);
  const float lg_grow = range.grow > 1e-38 ? (float)log2(range.grow) : -126.0f;
  // Pairs, where the iteration stays in their range (with eps below 0 the first singular values may be beyond 1), and what they lose of
  // an entry, 2^-37 of the norm in a step, grows to no more than 2^-25 by the last: six steps of the usual coefficients, twenty of a = 1.5.
  // Parts of G that are small against the norm and grow near 1 in more steps keep their bits in float32 products alone (the first
  // steps in float32 and the last six in pairs: a part that is still small at the end is off by 1e-4 of itself).  Seven steps in float32
  // and in pairs: 2048 x 2048 3868 and 1088 us, 1024 x 4096 3367 and 569, four of 220 x 64 299 and 46.
  const bool pairs = range.unit_b > 0.0f && a.eps >= 0.0f && (float)a.steps * lg_grow <= 12.0f;
  if (pairs && ortho_one_takes(a.rows, a.cols)) return launch_ortho_one(a, kUnit, range.unit_b, lg_grow, st);
  const int64_t rows_x = pairs ? o.sp : o.s, ld_x = pairs ? o.lp : o.l;
  const int tc = (int)((ld_x + 31) / 32);
  const dim3 tiles((unsigned)((rows_x + 31) / 32 * tc), (unsigned)a.batch), norms(kNormParts, (unsigned)a.batch);
  ortho_norm_kernel<T><<<norms, 256, 0, st>>>(a, parts);
  if (pairs) ortho_load_kernel<T, true><<<tiles, 256, 0, st>>>(a, parts, ws + o.x[0], rows_x, ld_x, tc, lg_grow, (float*)(ws + o.by));
  else ortho_load_kernel<T, false><<<tiles, 256, 0, st>>>(a, parts, ws + o.x[0], rows_x, ld_x, tc, 0.0f, nullptr);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  return pairs ? iterate_pairs(a, o, range.unit_b, ws, st) : iterate_f32(a, o, ws, st);
}

}  // namespace

size_t ortho_bytes(int64_t batch, int64_t rows, int64_t cols) { return ortho_layout(batch, rows, cols).total; }

hipError_t launch_ortho(const OrthoArgs& a, char* ws, hipStream_t st) {
  if (a.batch == 0) return hipSuccess;
  return a.g_bf16 ? ortho_typed<bf16_t>(a, ws, st) : ortho_typed<float>(a, ws, st);
}

}  // namespace ilargi
