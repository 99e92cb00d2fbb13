// Orthogonalised updates of small matrices: one workgroup keeps a matrix and its two products in LDS for all steps.
//
// X (up to 64 rows, zeros behind its own) and A, B (64 x 64) are pairs of float16 planes, as in kernels_ortho.hip; sixteen wavefronts
// form blocks of 16 x 16 with three products each, on accumulators of their own that are added at the end: (lo hi + hi lo) + hi hi is
// the same for (i, j) and (j, i), so A and B are symmetric to the bit.  Four of 220 x 64: 36.8 us for five steps, 5.0 of each more;
// seventeen launches of the general kernels 190.  What bounds a step is the LDS reads of X X^T (every block reads both its operands) and
// the chain of four barriers; the other 11.6 us are the launch, two passes over G with one load a lane on its way at a time, and the
// result.
#include <utility>

#include "mm_epilogue.h"

namespace ilargi {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kS = 64, kLdA = kS + 8, kMostLong = 448, kThreads = 1024, kSide = kThreads / 256;     // blocks of a row side by side

struct OneArgs {
  OrthoArgs o;
  float unit, unit_b, lg_grow;
  int lp;              // long side up to a multiple of 32
};

__device__ __forceinline__ f16x8 row_piece(const _Float16* p) { return *reinterpret_cast<const f16x8*>(p); }

// Eight k of one column each, from rows k0 + 8 (lane / 16) .. of a matrix whose rows run over k (ld halves): the transposing LDS read.
__device__ __forceinline__ f16x8 column_piece(const _Float16* m, int ld, int k0, int c0) {
  typedef __attribute__((address_space(3))) s16x4 l4;
  const int lane = threadIdx.x % 64, g = lane >> 4, i = lane & 15;
  const _Float16* p = m + (k0 + 8 * g + (i >> 2)) * ld + c0 + (i & 3) * 4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(p + 4 * ld));
  return __builtin_bit_cast(f16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

struct Three {
  f32x4 lh = {0.f, 0.f, 0.f, 0.f}, hl = lh, hh = lh;
  // first operand: the columns of the result; a lane then holds four neighbours of one row
  __device__ __forceinline__ void add(f16x8 qh, f16x8 ql, f16x8 ph, f16x8 pl) {
    lh = __builtin_amdgcn_mfma_f32_16x16x32_f16(ql, ph, lh, 0, 0, 0);
    hl = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh, pl, hl, 0, 0, 0);
    hh = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh, ph, hh, 0, 0, 0);
  }
  __device__ __forceinline__ f32x4 sum() const { return (lh + hl) + hh; }
};

__device__ __forceinline__ void put_pair(_Float16* hi, _Float16* lo, const f32x4& v) {
  f16x4 h, l;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    h[q] = (_Float16)v[q];
    l[q] = (_Float16)(v[q] - (float)h[q]);
  }
  *reinterpret_cast<f16x4*>(hi) = h;
  *reinterpret_cast<f16x4*>(lo) = l;
}
__device__ __forceinline__ f32x4 get_pair(const _Float16* hi, const _Float16* lo) {
  const f16x4 h = *reinterpret_cast<const f16x4*>(hi), l = *reinterpret_cast<const f16x4*>(lo);
  f32x4 v;
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = (float)h[q] + (float)l[q];
  return v;
}

template <class T>
__global__ __launch_bounds__(kThreads) void ortho_one_kernel(OneArgs a) {
  extern __shared__ __attribute__((aligned(16))) _Float16 lds[];
  __shared__ double wsum[kThreads / 64];
  const OrthoArgs& o = a.o;
  const int ldx = a.lp + 8, t = threadIdx.x, lane = t % 64, wave = t / 64, g4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  _Float16 *xh = lds, *xl = xh + kS * ldx, *ah = xl + kS * ldx, *al = ah + kS * kLdA, *bh = al + kS * kLdA, *bl = bh + kS * kLdA;
  const T* G = (const T*)o.G + blockIdx.x * o.batch_g;
  const int rows = (int)o.rows, cols = (int)o.cols;
  const bool flip = rows > cols;
  double s = 0.0;
  for (int r = wave; r < rows; r += kThreads / 64)
    for (int c = lane; c < cols; c += 64) {
      const double v = (double)(float)G[r * o.ld_g + c];
      s = fma(v, v, s);
    }
  for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
  if (lane == 0) wsum[wave] = s;
  for (int i = t; i < kS * ldx; i += kThreads) reinterpret_cast<uint32_t*>(lds)[i] = 0;       // both planes of X
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < kThreads / 64; ++w) s += wsum[w];
  const double norm = sqrt(s), one = 1.0 / (norm + (double)o.eps);
  const float lg_norm = lg_of(norm * one);
  int up = ortho_exponent(lg_norm, a.lg_grow, 0);             // X is held times unit 2^up
  const Factor2 scale = factor2(ldexp(one * (double)a.unit, up));
  for (int r = wave; r < rows; r += kThreads / 64)
    for (int c = lane; c < cols; c += 64) {
      const float v = times((float)G[r * o.ld_g + c], scale);
      const int at = flip ? c * ldx + r : r * ldx + c;
      const _Float16 h = (_Float16)v;
      xh[at] = h;
      xl[at] = (_Float16)(v - (float)h);
    }
  __syncthreads();
  const int bi = (wave % 4) * 16;                             // this wavefront's rows of A, B and X
  const int blocks = a.lp / 16;                               // it forms blocks wave / 4, + kSide, .. of them
  for (int step = 0; step < o.steps; ++step) {
    // (the places in LDS are worked out anew in every step: kept from one to the next they do not fit the registers)
    int r16 = lane & 15;
    asm volatile("" : "+v"(r16));
    const int then = step + 1 < o.steps ? ortho_exponent(lg_norm, a.lg_grow, step + 1) : 0;
    const float by_a = ldexpf(1.0f / a.unit, -2 * up), by_x = ldexpf(1.0f, then - up);
    up = then;
#pragma unroll
    for (int u = 0; u < 4 / kSide; ++u) {
      const int bj = (wave / 4 + kSide * u) * 16;
      Three f;
      for (int k = 0; k < a.lp; k += 32)
        f.add(row_piece(xh + (bj + r16) * ldx + k + g8), row_piece(xl + (bj + r16) * ldx + k + g8), row_piece(xh + (bi + r16) * ldx + k + g8),
              row_piece(xl + (bi + r16) * ldx + k + g8));
      const int at = (bi + r16) * kLdA + bj + g4;
      put_pair(ah + at, al + at, f.sum() * by_a);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4 / kSide; ++u) {
      const int bj = (wave / 4 + kSide * u) * 16;
      Three f;
#pragma unroll
      for (int k = 0; k < kS; k += 32)
        f.add(row_piece(ah + (bj + r16) * kLdA + k + g8), row_piece(al + (bj + r16) * kLdA + k + g8), row_piece(ah + (bi + r16) * kLdA + k + g8),
              row_piece(al + (bi + r16) * kLdA + k + g8));
      const int at = (bi + r16) * kLdA + bj + g4;
      const f32x4 v = get_pair(ah + at, al + at), w = f.sum();
      f32x4 b;
#pragma unroll
      for (int q = 0; q < 4; ++q) b[q] = fmaf(o.coef[2] * a.unit_b / (a.unit * a.unit), w[q], o.coef[1] * a.unit_b / a.unit * v[q]);
      put_pair(bh + at, bl + at, b);
    }
    __syncthreads();
    f16x8 ph[2], pl[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      ph[k] = row_piece(bh + (bi + r16) * kLdA + 32 * k + g8);
      pl[k] = row_piece(bl + (bi + r16) * kLdA + 32 * k + g8);
    }
    constexpr int kMost = kMostLong / 16 / kSide;
    f32x4 next[kMost];
#pragma unroll
    for (int u = 0; u < kMost; ++u) {
      const int c = (wave / 4 + kSide * u) * 16;
      if (wave / 4 + kSide * u >= blocks) continue;
      Three f;
#pragma unroll
      for (int k = 0; k < 2; ++k) f.add(column_piece(xh, ldx, 32 * k, c), column_piece(xl, ldx, 32 * k, c), ph[k], pl[k]);
      const int at = (bi + r16) * ldx + c + g4;
      const f32x4 v = get_pair(xh + at, xl + at), w = f.sum();
#pragma unroll
      for (int q = 0; q < 4; ++q) next[u][q] = fmaf(1.0f / a.unit_b, w[q], o.coef[0] * v[q]) * by_x;
      __builtin_amdgcn_sched_barrier(0);                      // (all blocks' reads at once do not fit the registers)
    }
    if (step + 1 < o.steps) {
      __syncthreads();                                        // X is read: the next one takes its place
#pragma unroll
      for (int u = 0; u < kMost; ++u) {
        const int c = (wave / 4 + kSide * u) * 16;
        if (wave / 4 + kSide * u >= blocks) continue;
        const int at = (bi + r16) * ldx + c + g4;
        put_pair(xh + at, xl + at, next[u]);
      }
      __syncthreads();
      continue;
    }
    // the result, in float32 where X was, and from there along its rows
    float* last = reinterpret_cast<float*>(lds);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMost; ++u) {
      const int c = (wave / 4 + kSide * u) * 16;
      if (wave / 4 + kSide * u >= blocks) continue;
      *reinterpret_cast<f32x4*>(last + (bi + r16) * ldx + c + g4) = next[u];
    }
  }
  __syncthreads();
  const float* last = reinterpret_cast<const float*>(lds);
  const int S = flip ? cols : rows, L = flip ? rows : cols, quads = (L + 3) / 4;
  Epilogue e{};
  e.mode = kEpiScale;
  e.s0 = o.alpha / a.unit; e.s2 = o.beta; e.base = o.beta != 0.0f ? o.base : nullptr;
  e.out = o.out; e.ld_out = o.ld_out; e.batch_out = o.batch_out; e.out_bf16 = o.out_bf16; e.flip = flip;
  const float none[4] = {0.f, 0.f, 0.f, 0.f};
  for (int q = t; q < kS * quads; q += kThreads) {
    const int i = flip ? q % kS : q / quads, j = (flip ? q / kS : q % quads) * 4;
    if (i >= S) continue;
    const f32x4 w = *reinterpret_cast<const f32x4*>(last + i * ldx + j);
    float v[4] = {w[0], w[1], w[2], w[3]};
    epilogue4(e, 1.0f, blockIdx.x, i, j, L - j < 4 ? L - j : 4, none, SrcQuad{}, v);
  }
}

}  // namespace

// Short side up to 64, long side up to 448: X, A and B take at most 154 of a compute unit's 160 KB.
bool ortho_one_takes(int64_t rows, int64_t cols) {
  const int64_t s = rows < cols ? rows : cols, l = rows < cols ? cols : rows;
  return s <= kS && l <= kMostLong;
}

hipError_t launch_ortho_one(const OrthoArgs& o, float unit, float unit_b, float lg_grow, hipStream_t st) {
  if (!ortho_one_takes(o.rows, o.cols)) return hipErrorInvalidValue;
  const int64_t l = o.rows < o.cols ? o.cols : o.rows;
  const OneArgs a{o, unit, unit_b, lg_grow, (int)((l + 31) / 32 * 32)};
  const size_t bytes = 2 * (2 * (size_t)kS * (size_t)(a.lp + 8) + 4 * (size_t)kS * kLdA);
  const void* kernel = o.g_bf16 ? (const void*)ortho_one_kernel<bf16_t> : (const void*)ortho_one_kernel<float>;
  if (hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); e != hipSuccess) return e;
  if (o.g_bf16) ortho_one_kernel<bf16_t><<<(unsigned)o.batch, kThreads, bytes, st>>>(a);
  else ortho_one_kernel<float><<<(unsigned)o.batch, kThreads, bytes, st>>>(a);
  return hipGetLastError();
}

}  // namespace ilargi
