// Orthogonalised updates: X = G / (|G|_F + eps), then steps of X <- a X + (b A + c A^2) X with A = X X^T.
#include "mm_epilogue.h"

namespace ilargi {

namespace {

constexpr int kNormParts = 64;

// Sums of squares of a share of one matrix's rows, in 64 bits: the norm neither overflows nor loses small entries.
template <class T>
__global__ __launch_bounds__(256) void ortho_norm_kernel(OrthoArgs a, double* __restrict__ parts) {
  __shared__ double wsum[4];
  const T* G = (const T*)a.G + blockIdx.y * a.batch_g;
  const int64_t total = a.rows * a.cols;
  double s = 0.0;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += kNormParts * 256) {
    const int64_t r = at / a.cols;
    const double g = (double)(float)G[r * a.ld_g + (at - r * a.cols)];
    s += g * g;
  }
  for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
  if (threadIdx.x % 64 == 0) wsum[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.y * kNormParts + blockIdx.x] = (wsum[0] + wsum[1]) + (wsum[2] + wsum[3]);
}

// X (short side x long side) = G or its transpose over the norm, 32 x 32 tiles through LDS.
template <class T>
__global__ __launch_bounds__(256) void ortho_load_kernel(OrthoArgs a, const double* __restrict__ parts, float* __restrict__ X, int tiles_c) {
  __shared__ float tile[32][33];
  __shared__ float scale;
  const int64_t b = blockIdx.y;
  if (threadIdx.x < 64) {
    double s = parts[b * kNormParts + threadIdx.x];
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if (threadIdx.x == 0) scale = (float)(1.0 / (sqrt(s) + (double)a.eps));
  }
  const T* G = (const T*)a.G + b * a.batch_g;
  const int64_t r0 = (int64_t)(blockIdx.x / tiles_c) * 32, c0 = (int64_t)(blockIdx.x % tiles_c) * 32;
  const int x = threadIdx.x % 32, y = threadIdx.x / 32;
#pragma unroll
  for (int q = 0; q < 32; q += 8)
    if (r0 + y + q < a.rows && c0 + x < a.cols) tile[y + q][x] = (float)G[(r0 + y + q) * a.ld_g + c0 + x];
  __syncthreads();
  X += b * a.rows * a.cols;
  const bool flip = a.rows > a.cols;
#pragma unroll
  for (int q = 0; q < 32; q += 8) {
    if (flip) {
      if (c0 + y + q < a.cols && r0 + x < a.rows) X[(c0 + y + q) * a.rows + r0 + x] = tile[x][y + q] * scale;
    } else {
      if (r0 + y + q < a.rows && c0 + x < a.cols) X[(r0 + y + q) * a.cols + c0 + x] = tile[y + q][x] * scale;
    }
  }
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t ortho_bytes(int64_t batch, int64_t rows, int64_t cols) {
  const size_t s = (size_t)(rows < cols ? rows : cols), l = (size_t)(rows < cols ? cols : rows), n = (size_t)batch;
  return up256(n * kNormParts * 8) + 2 * up256(4 * n * s * l) + 2 * up256(4 * n * s * s);
}

hipError_t launch_ortho(const OrthoArgs& a, char* ws, hipStream_t st) {
  if (a.batch == 0) return hipSuccess;
  const int64_t s = a.rows < a.cols ? a.rows : a.cols, l = a.rows < a.cols ? a.cols : a.rows;
  double* parts = (double*)ws;
  ws += up256((size_t)a.batch * kNormParts * 8);
  float* X[2] = {(float*)ws, (float*)(ws + up256(4 * (size_t)(a.batch * s * l)))};
  ws += 2 * up256(4 * (size_t)(a.batch * s * l));
  float *A = (float*)ws, *B = (float*)(ws + up256(4 * (size_t)(a.batch * s * s)));
  const int tc = (int)((a.cols + 31) / 32);
  const dim3 tiles((unsigned)((a.rows + 31) / 32 * tc), (unsigned)a.batch), norms(kNormParts, (unsigned)a.batch);
  if (a.g_bf16) {
    ortho_norm_kernel<bf16_t><<<norms, 256, 0, st>>>(a, parts);
    ortho_load_kernel<bf16_t><<<tiles, 256, 0, st>>>(a, parts, X[0], tc);
  } else {
    ortho_norm_kernel<float><<<norms, 256, 0, st>>>(a, parts);
    ortho_load_kernel<float><<<tiles, 256, 0, st>>>(a, parts, X[0], tc);
  }
  for (int t = 0; t < a.steps; ++t) {
    const float* x = X[t & 1];
    Product p{};
    p.M = s; p.N = s; p.K = l; p.batches = a.batch;
    p.P = {x, l, 0, 0, s * l};
    p.Q = p.P;
    p.epi.mode = kEpiScale;
    p.epi.s0 = 1.0f; p.epi.out = A; p.epi.ld_out = s; p.epi.batch_out = s * s;
    if (hipError_t e = launch_mm_f32(p, st); e != hipSuccess) return e;
    p.K = s;
    p.P = {A, s, 0, 0, s * s};
    p.Q = p.P;
    p.epi.s0 = a.coef[2]; p.epi.s1 = a.coef[1];
    p.epi.src = A; p.epi.ld_src = s; p.epi.batch_src = s * s;
    p.epi.out = B;
    if (hipError_t e = launch_mm_f32(p, st); e != hipSuccess) return e;
    p.N = l;
    p.P.p = B;
    p.Q = {x, l, 1, 0, s * l};
    p.epi.s0 = 1.0f; p.epi.s1 = a.coef[0];
    p.epi.src = x; p.epi.ld_src = l; p.epi.batch_src = s * l;
    p.epi.out = X[(t & 1) ^ 1]; p.epi.ld_out = l; p.epi.batch_out = s * l;
    if (t + 1 == a.steps) {
      p.epi.s0 = a.alpha; p.epi.s1 = a.alpha * a.coef[0]; p.epi.s2 = a.beta; p.epi.base = a.beta != 0.0f ? a.base : nullptr;
      p.epi.out = a.out; p.epi.ld_out = a.ld_out; p.epi.batch_out = a.batch_out; p.epi.out_bf16 = a.out_bf16;
      p.epi.flip = a.rows > a.cols;
    }
    if (hipError_t e = launch_mm_f32(p, st); e != hipSuccess) return e;
  }
  return hipGetLastError();
}

}  // namespace ilargi
