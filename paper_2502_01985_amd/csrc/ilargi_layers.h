// Internal declarations of the operators of models with learned features: embedding rows, dense layers, orthogonalised
// updates (not installed).
#ifndef ILARGI_LAYERS_H_
#define ILARGI_LAYERS_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ilargi.h"
#include "ilargi_internal.h"

namespace ilargi {

using bf16_t = __bf16;

template <class T> struct ElemOf;
template <> struct ElemOf<float> { static constexpr int kVec = 4; };     // elements of a 16-byte piece
template <> struct ElemOf<bf16_t> { static constexpr int kVec = 8; };

// Sixteen bytes at any address an element may have: the memory system takes dword and halfword addresses.
template <class T, int N> struct __attribute__((packed)) Piece { T v[N]; };

// N consecutive elements as floats, the ones from `valid` on as zeros.
template <class T, int N>
__device__ __forceinline__ void load_piece(const T* __restrict__ p, int valid, float (&f)[N]) {
  if (valid >= N) {
    const Piece<T, N> t = *reinterpret_cast<const Piece<T, N>*>(p);
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = (float)t.v[j];
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = j < valid ? (float)p[j] : 0.0f;
  }
}

template <class T, int N>
__device__ __forceinline__ void store_piece(T* __restrict__ p, int valid, const float (&f)[N]) {
  if (valid >= N) {
    Piece<T, N> t;
#pragma unroll
    for (int j = 0; j < N; ++j) t.v[j] = (T)f[j];
    *reinterpret_cast<Piece<T, N>*>(p) = t;
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < valid) p[j] = (T)f[j];
  }
}

// exp(-|x|) and the reciprocal by the hardware's instructions, each good to a unit of 2^-23; the argument's rounding adds |x| 2^-24.
__device__ __forceinline__ float exp_minus(float x) { return __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(x)); }

// erfc(|z| / sqrt 2) / 2 = the upper tail of the normal distribution, and exp(-z^2 / 2).  With t = 1 / (1 + 0.3 x) the scaled function
// exp(x^2) erfc(x) is a polynomial of t without a constant term, fitted here to 3.4e-8 of itself on [0, 12] (7.4e-8, its largest at
// x = 0.07, with the constants as floats hold them), so the tail keeps its relative accuracy where 1 + erf cancels.  16384 x 2048 x 8192 with gelu, bfloat16: 739 microseconds with the device library's erf
// where this took 661.
__device__ __forceinline__ float normal_tail(float z, float& gauss) {
  const float x = 0.70710678118654752f * fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.3f, x, 1.0f));
  gauss = __builtin_amdgcn_exp2f(-0.72134752044448171f * z * z);
  float p = -0.12925735f;
  p = fmaf(p, t, 0.48432142f);
  p = fmaf(p, t, -0.50981223f);
  p = fmaf(p, t, 0.54501167f);
  p = fmaf(p, t, -0.092856425f);
  p = fmaf(p, t, 0.21419419f);
  p = fmaf(p, t, 0.14851802f);
  p = fmaf(p, t, 0.17069138f);
  p = fmaf(p, t, 0.16918933f);
  return 0.5f * p * t * gauss;
}

// f(z) of a layer in 32 bits.
__device__ __forceinline__ float act_value(float z, int act) {
  switch (act) {
    case ILARGI_ACT_RELU: return z > 0.0f ? z : (z != z ? z : 0.0f);
    case ILARGI_ACT_SIGMOID: {
      const float e = exp_minus(z), q = __builtin_amdgcn_rcpf(1.0f + e);
      return z >= 0.0f ? q : e * q;
    }
    case ILARGI_ACT_SILU: {
      const float e = exp_minus(z), q = __builtin_amdgcn_rcpf(1.0f + e);
      return z == -INFINITY ? 0.0f : z * (z >= 0.0f ? q : e * q);      // (the limit, where infinity times 0 is none)
    }
    case ILARGI_ACT_GELU: {
      float gauss;
      const float h = normal_tail(z, gauss);
      return z == -INFINITY ? 0.0f : z * (z >= 0.0f ? 1.0f - h : h);
    }
    default: return z;
  }
}
// The same of N values, side by side: one chain of branches for all, and their instructions fill each other's latencies.
// (A value at a time: 662 microseconds of that layer where this takes 628.)
template <int N>
__device__ __forceinline__ void act_values(float (&z)[N], int act) {
  auto all = [&](auto which) {
#pragma unroll
    for (int j = 0; j < N; ++j) z[j] = act_value(z[j], decltype(which)::value);
  };
  switch (act) {
    case ILARGI_ACT_RELU: all(std::integral_constant<int, ILARGI_ACT_RELU>()); break;
    case ILARGI_ACT_SIGMOID: all(std::integral_constant<int, ILARGI_ACT_SIGMOID>()); break;
    case ILARGI_ACT_SILU: all(std::integral_constant<int, ILARGI_ACT_SILU>()); break;
    case ILARGI_ACT_GELU: all(std::integral_constant<int, ILARGI_ACT_GELU>()); break;
    default: break;
  }
}
// f'(z)
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case ILARGI_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case ILARGI_ACT_SIGMOID: {
      const float e = exp_minus(z), q = __builtin_amdgcn_rcpf(1.0f + e);
      return e * q * q;
    }
    case ILARGI_ACT_SILU: {
      const float e = exp_minus(z), q = __builtin_amdgcn_rcpf(1.0f + e);        // sigmoid(|z|)
      const float p = z >= 0.0f ? q : e * q, r = z >= 0.0f ? e * q : q;         // sigmoid(z), sigmoid(-z)
      return p + (r == 0.0f || p == 0.0f ? 0.0f : z * p * r);
    }
    case ILARGI_ACT_GELU: {
      float gauss;
      const float h = normal_tail(z, gauss);
      return (z >= 0.0f ? 1.0f - h : h) + (gauss == 0.0f ? 0.0f : 0.39894228040143268f * z * gauss);
    }
    default: return 1.0f;
  }
}

// Outputs of so many bytes are written past the caches: half of the last-level cache.
constexpr int64_t kStreamBytes = 128ll << 20;

// The threads of a launch along an axis are counted in 32 bits: one of 2^32 and more forms the wrong number of workgroups, with no
// error.  So `groups` workgroups of `threads` go in parts: launch(first, count) forms workgroups first .. first + count.
constexpr int64_t kMostThreads = 1ll << 31;
constexpr int64_t kMostAcross = 32768;       // workgroups along the second axis: devices promise 65,535
template <class F>
hipError_t in_parts(int64_t groups, int threads, F launch) {
  const int64_t most = kMostThreads / threads;
  for (int64_t first = 0; first < groups; first += most) launch(first, (unsigned)(groups - first < most ? groups - first : most));
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------- embedding rows
struct EmbedArgs {
  const void* table;
  int64_t rows, cols, ld_table;
  const int32_t* ids;
  int64_t n;
  float scale;
  int accumulate;
  void* out;
  int64_t ld_out;
  int table_bf16, out_bf16;
};
hipError_t launch_embed(const EmbedArgs& a, hipStream_t st);

struct EmbedGradArgs {
  const void* d_out;
  int64_t ld_out;
  const int32_t* ids;
  int64_t n, rows, cols;
  float scale;
  int accumulate;
  void* d_table;
  int64_t ld_table;
  int out_bf16, table_bf16;
};
size_t embed_grad_bytes(int64_t n, int64_t cols);
hipError_t launch_embed_grad(const EmbedGradArgs& a, char* ws, hipStream_t st);

// ------------------------------------------------------------------------------------------------- matrix products
// C(i, j) = sum_k P(i, k) Q(k, j).  An operand is a matrix of rows of `ld` elements; `k_rows` says that its rows run over
// k (then its columns are the i or j of the result), else that its columns do.
struct Operand {
  const void* p;
  int64_t ld;
  int k_rows;
  int bf16;
  int64_t batch;        // elements from one matrix of a batch to the next
};
enum { kEpiLinear = 0, kEpiScale = 1 };
struct Epilogue {
  int mode;
  // kEpiLinear: z = acc + bias[j] kept in `pre`, out = f(z) + src
  // kEpiScale: out = (s0 acc + s1 src) by[b] + s2 base (by: NULL for 1); `flip` writes out(j, i), with `base` laid out as `out`
  float s0, s1, s2;
  const float* by;
  const void* base;
  const void* bias;
  const void* src;
  int64_t ld_src, batch_src;
  int src_bf16;
  int64_t src_plane;      // not 0: src is a pair of float16 planes so far apart
  void* pre;
  int64_t ld_pre;
  int act;
  void* out;
  int64_t ld_out, batch_out;
  int out_bf16;
  int64_t out_plane;      // not 0: out is such a pair
  int flip;
};
struct Product {
  Operand P, Q;
  int64_t M, N, K, batches;
  Epilogue epi;
};
struct MmPlan {
  int tile, splits;         // workgroups form tile x tile sums of a share of k
  size_t partial_bytes;     // sums of the shares, where there are several
};
MmPlan mm_f32_plan(int64_t M, int64_t N, int64_t K, int64_t batches);
hipError_t launch_mm_f32(const Product& a, const MmPlan& plan, float* partial, hipStream_t st);
bool mm_rows_takes(int64_t M, int64_t K, bool bf16);
MmPlan mm_rows_plan(int64_t M, int64_t N, int64_t K);
hipError_t launch_mm_rows(const Product& a, const MmPlan& plan, float* partial, hipStream_t st);
// Adds the shares in their order: `partial` holds splits x batches matrices of M x (N to a multiple of 4).
hipError_t launch_mm_join(int64_t M, int64_t N, int64_t batches, int symmetric, const Epilogue& epi, int splits, const float* partial, hipStream_t st);

// The same for 16-bit operands on the 16-bit matrix cores, with sums in float32.  Operands of pairs are the sum of two planes,
// hi + lo (`plane` elements apart, float16): lo hi + hi lo + hi hi is formed, three products in place of one.
// Rows and columns lie at 16-byte addresses and whole pieces of 8 elements may be read: `across` rows or columns (of i or j), and
// along k up to the next multiple of 8, zeros behind K.
struct Operand16 {
  const void* p;
  int64_t ld;
  int k_rows;
  int64_t batch, plane, across;
};
inline void shift_operand(Operand* o, int64_t by) { o->p = (const char*)o->p + (o->k_rows ? by : by * o->ld) * (o->bf16 ? 2 : 4); }
inline void shift_operand(Operand16* o, int64_t by) {
  o->p = (const char*)o->p + (o->k_rows ? by : by * o->ld) * 2;
  o->across -= by;
}
enum { kMm16Bf16 = 0, kMm16Pairs = 1 };     // bfloat16; pairs of float16 planes
struct Product16 {
  Operand16 P, Q;
  int64_t M, N, K, batches;
  int kind;
  int symmetric;            // C = C^T: blocks above the diagonal are formed, and written twice
  Epilogue epi;
  bool past;                // a layer's outputs are written past the caches
};
MmPlan mm16_plan(int64_t M, int64_t N, int64_t K, int64_t batches, int kind, int symmetric);
// A bfloat16 matrix laid out for launch_mm16: rows of (cols to a multiple of 8) elements.
hipError_t launch_pack16(const void* src, int64_t ld, int64_t rows, int64_t cols, void* dst, hipStream_t st);
hipError_t launch_mm16(const Product16& a, const MmPlan& plan, float* partial, hipStream_t st);

struct LayerGradArgs {
  int64_t n, m;
  const void* d_out;
  int64_t ld_out;
  const void* pre;
  int64_t ld_pre;
  int act, bf16;
  void* dz;             // n x m, ld_dz (NULL: not written)
  int64_t ld_dz;
  void* d_bias;         // may be NULL
  int accumulate;
};
size_t layer_grad_partial_bytes(int64_t n, int64_t m);
hipError_t launch_layer_grad(const LayerGradArgs& a, float* partial, hipStream_t st);

// A product of a layer in blocks of tile_m x tile_n sums, a workgroup of `threads` each: whole, or in parts of whole blocks where they are
// too many for one launch.
template <class P, class F>
hipError_t in_blocks(const P& a, int64_t tile_m, int64_t tile_n, int threads, F launch) {
  const int64_t tm = (a.M + tile_m - 1) / tile_m, tn = (a.N + tile_n - 1) / tile_n, most = kMostThreads / threads;
  if (tm * tn <= most) return launch(a);
  if (a.batches != 1 || a.epi.mode != kEpiLinear) return hipErrorInvalidValue;
  const int64_t across = tn < most ? tn : most, down = most / across;
  for (int64_t ti = 0; ti < tm; ti += down)
    for (int64_t tj = 0; tj < tn; tj += across) {
      const int64_t i = ti * tile_m, j = tj * tile_n;
      P b = a;
      b.M = a.M - i < down * tile_m ? a.M - i : down * tile_m;
      b.N = a.N - j < across * tile_n ? a.N - j : across * tile_n;
      shift_operand(&b.P, i);
      shift_operand(&b.Q, j);
      auto shift = [](const void* p, int64_t by, int bf16) { return p != nullptr ? (const void*)((const char*)p + by * (bf16 ? 2 : 4)) : p; };
      b.epi.bias = shift(a.epi.bias, j, a.epi.out_bf16);
      b.epi.src = shift(a.epi.src, i * a.epi.ld_src + j, a.epi.src_bf16);
      b.epi.pre = (void*)shift(a.epi.pre, i * a.epi.ld_pre + j, a.epi.out_bf16);
      b.epi.out = (void*)shift(a.epi.out, i * a.epi.ld_out + j, a.epi.out_bf16);
      if (hipError_t e = launch(b); e != hipSuccess) return e;
    }
  return hipSuccess;
}

// ------------------------------------------------------------------------------------------------- orthogonal updates
struct OrthoArgs {
  const void* G;
  int64_t batch, rows, cols, ld_g, batch_g;
  int g_bf16;
  int steps;
  float coef[3];
  float eps, alpha, beta;
  const void* base;     // may be NULL; laid out as out
  void* out;
  int64_t ld_out, batch_out;
  int out_bf16;
};
size_t ortho_bytes(int64_t batch, int64_t rows, int64_t cols);
hipError_t launch_ortho(const OrthoArgs& a, char* ws, hipStream_t st);
// x times a factor that may be no float32 number, as the reciprocal of a norm may: a power of two first, then what is left of it.
struct Factor2 {
  float mantissa;
  int exponent;
};
__device__ __forceinline__ Factor2 factor2(double f) {
  int e;
  const double m = frexp(f, &e);
  return {(float)m, e};
}
__device__ __forceinline__ float times(float x, const Factor2& f) { return ldexpf(x, f.exponent) * f.mantissa; }

// Small matrices, whose iteration stays in pairs of float16 times these units.
// X_t of step t is held times 2^e besides, the largest e from 0 to 126 for which grow^t |X_0| 2^e <= 1 (`grow`: most that a step
// multiplies a singular value by): X is as small as |G| / eps where the norm is far below eps.  Logarithms to base 2, of
// |X_0| = norm / (norm + eps) and of grow; 126 where a logarithm is no number.
__device__ __forceinline__ float lg_of(double v) {
  int e;
  const float m = (float)frexp(v, &e);
  return (float)e + __builtin_amdgcn_logf(m);
}
__device__ __forceinline__ int ortho_exponent(float lg_norm, float lg_grow, int t) {
  return (int)fmaxf(0.0f, fminf(126.0f, floorf(-fmaf((float)t, lg_grow, lg_norm))));
}
bool ortho_one_takes(int64_t rows, int64_t cols);
hipError_t launch_ortho_one(const OrthoArgs& a, float unit, float unit_b, float lg_grow, hipStream_t st);

}  // namespace ilargi
#endif
