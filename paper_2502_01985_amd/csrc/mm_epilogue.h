// What happens to the sums of a matrix product before they are stored: four neighbouring columns of one row at a time.
#ifndef ILARGI_MM_EPILOGUE_H_
#define ILARGI_MM_EPILOGUE_H_

#include "ilargi_layers.h"

namespace ilargi {

__device__ __forceinline__ void load4_any(const void* p, int64_t at, int bf16, int valid, float (&f)[4]) {
  if (bf16) load_piece<bf16_t, 4>((const bf16_t*)p + at, valid, f);
  else load_piece<float, 4>((const float*)p + at, valid, f);
}
__device__ __forceinline__ void store4_any(void* p, int64_t at, int bf16, int valid, const float (&f)[4]) {
  if (bf16) store_piece<bf16_t, 4>((bf16_t*)p + at, valid, f);
  else store_piece<float, 4>((float*)p + at, valid, f);
}

// A pair of float16 planes: x = hi + lo, 22 bits of entries that are not small against the largest (lo counts in 2^-24).
__device__ __forceinline__ float pair_value(const _Float16* p, int64_t at, int64_t plane) { return (float)p[at] + (float)p[at + plane]; }
__device__ __forceinline__ void pair_store(_Float16* p, int64_t at, int64_t plane, float x) {
  const _Float16 hi = (_Float16)x;
  p[at] = hi;
  p[at + plane] = (_Float16)(x - (float)hi);
}

// out(i, j) = s0 v + s1 src(i, j) in pairs, columns j .. j + valid.
__device__ __forceinline__ void epilogue4_pairs(const Epilogue& e, int64_t b, int64_t i, int64_t j, int valid, float (&v)[4]) {
  const _Float16* src = (const _Float16*)e.src + b * e.batch_src + i * e.ld_src + j;
  _Float16* out = (_Float16*)e.out + b * e.batch_out + i * e.ld_out + j;
  float t[4] = {0.f, 0.f, 0.f, 0.f}, hi[4], lo[4];
  if (e.src != nullptr) {
    load_piece<_Float16, 4>(src, valid, hi);
    load_piece<_Float16, 4>(src + e.src_plane, valid, lo);
#pragma unroll
    for (int q = 0; q < 4; ++q) t[q] = hi[q] + lo[q];
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float x = fmaf(e.s0, v[q], e.s1 * t[q]);
    hi[q] = (float)(_Float16)x;
    lo[q] = x - hi[q];
  }
  store_piece<_Float16, 4>(out, valid, hi);
  store_piece<_Float16, 4>(out + e.out_plane, valid, lo);
}
// The bias of columns j .. j + valid, zeros where there is none.
__device__ __forceinline__ void epilogue_bias(const Epilogue& e, int64_t j, int valid, float (&bias)[4]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) bias[q] = 0.0f;
  if (e.mode == kEpiLinear && e.bias != nullptr && valid > 0) load4_any(e.bias, j, e.out_bf16, valid, bias);
}

// Columns j .. j + valid of row i of matrix b of the batch.
__device__ __forceinline__ void epilogue4(const Epilogue& e, int64_t b, int64_t i, int64_t j, int valid, const float (&bias)[4], float (&v)[4]) {
  if (e.mode == kEpiLinear) {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += bias[q];
    if (e.pre != nullptr) store4_any(e.pre, i * e.ld_pre + j, e.out_bf16, valid, v);
    if (e.act != ILARGI_ACT_NONE) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = act_value(v[q], e.act);
    }
    if (e.src != nullptr) {
      float t[4];
      load4_any(e.src, i * e.ld_src + j, e.src_bf16, valid, t);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += t[q];
    }
    store4_any(e.out, i * e.ld_out + j, e.out_bf16, valid, v);
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] *= e.s0;
  if (e.src != nullptr) {
    float t[4];
    const int64_t from = b * e.batch_src + i * e.ld_src + j;
    if (e.src_plane != 0) {
#pragma unroll
      for (int q = 0; q < 4; ++q) t[q] = q < valid ? pair_value((const _Float16*)e.src, from + q, e.src_plane) : 0.0f;
    } else {
      load4_any(e.src, from, e.src_bf16, valid, t);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = fmaf(e.s1, t[q], v[q]);
  }
  if (e.flip) {
    for (int q = 0; q < valid && q < 4; ++q) {
      const int64_t at = b * e.batch_out + (j + q) * e.ld_out + i;
      float r = v[q];
      if (e.base != nullptr) r = fmaf(e.s2, e.out_bf16 ? (float)((const bf16_t*)e.base)[at] : ((const float*)e.base)[at], r);
      if (e.out_bf16) ((bf16_t*)e.out)[at] = (bf16_t)r;
      else ((float*)e.out)[at] = r;
    }
    return;
  }
  const int64_t at = b * e.batch_out + i * e.ld_out + j;
  if (e.base != nullptr) {
    float t[4];
    load4_any(e.base, at, e.out_bf16, valid, t);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = fmaf(e.s2, t[q], v[q]);
  }
  store4_any(e.out, at, e.out_bf16, valid, v);
}

}  // namespace ilargi
#endif
