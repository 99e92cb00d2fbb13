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

// The bias of columns j .. j + valid, zeros where there is none.
__device__ __forceinline__ void epilogue_bias(const Epilogue& e, int64_t j, int valid, float (&bias)[4]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) bias[q] = 0.0f;
  if (e.mode == kEpiLinear && e.bias != nullptr && valid > 0) load4_any(e.bias, j, e.out_bf16, valid, bias);
}

// Four columns of `src` as they lie: asked for early, turned into numbers when the sums are finished, so that the loads of many rows
// are on their way together.  (A row at a time, every one waits for its own: 1 us each where another compute unit wrote it.)
struct SrcQuad {
  uint2 a, b;
};
__device__ __forceinline__ SrcQuad epilogue_ask(const Epilogue& e, int64_t b, int64_t i, int64_t j, int valid) {
  SrcQuad r = {make_uint2(0, 0), make_uint2(0, 0)};
  if (e.src == nullptr || valid <= 0) return r;
  const int64_t at = b * e.batch_src + i * e.ld_src + j;
  if (e.src_plane == 0 && !e.src_bf16) {
    const uint32_t* p = (const uint32_t*)e.src + at;
    if (valid >= 4) {
      const Piece<uint32_t, 4> t = *reinterpret_cast<const Piece<uint32_t, 4>*>(p);
      return {make_uint2(t.v[0], t.v[1]), make_uint2(t.v[2], t.v[3])};
    }
    r.a.x = p[0];
    if (valid > 1) r.a.y = p[1];
    if (valid > 2) r.b.x = p[2];
    return r;
  }
  const uint16_t* p = (const uint16_t*)e.src + at;
  auto four = [valid](const uint16_t* q) {
    if (valid >= 4) return __builtin_bit_cast(uint2, *reinterpret_cast<const Piece<uint16_t, 4>*>(q));
    uint2 t = make_uint2(q[0], 0);
    if (valid > 1) t.x |= (uint32_t)q[1] << 16;
    if (valid > 2) t.y = q[2];
    return t;
  };
  r.a = four(p);
  if (e.src_plane != 0) r.b = four(p + e.src_plane);
  return r;
}
__device__ __forceinline__ void epilogue_src(const Epilogue& e, const SrcQuad& r, float (&t)[4]) {
  if (e.src_plane != 0) {
    const Piece<_Float16, 4> hi = __builtin_bit_cast(Piece<_Float16, 4>, r.a), lo = __builtin_bit_cast(Piece<_Float16, 4>, r.b);
#pragma unroll
    for (int q = 0; q < 4; ++q) t[q] = (float)hi.v[q] + (float)lo.v[q];
  } else if (e.src_bf16) {
    t[0] = __uint_as_float(r.a.x << 16); t[1] = __uint_as_float(r.a.x & 0xffff0000u);
    t[2] = __uint_as_float(r.a.y << 16); t[3] = __uint_as_float(r.a.y & 0xffff0000u);
  } else {
    t[0] = __uint_as_float(r.a.x); t[1] = __uint_as_float(r.a.y);
    t[2] = __uint_as_float(r.b.x); t[3] = __uint_as_float(r.b.y);
  }
}

// Columns j .. j + valid of row i of matrix b of the batch: `v` are the sums, `raw` what epilogue_ask gave.
// `by` is by[b], which kernels that have one ask for at their start.  (SRC false: the caller knows that there is no src.)
template <bool SRC = true>
__device__ __forceinline__ void epilogue4(const Epilogue& e, float by, int64_t b, int64_t i, int64_t j, int valid, const float (&bias)[4], const SrcQuad& raw,
                                          float (&v)[4]) {
  float t[4] = {0.f, 0.f, 0.f, 0.f};
  if (SRC && e.src != nullptr) epilogue_src(e, raw, t);
  if (e.mode == kEpiLinear) {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += bias[q];
    if (e.pre != nullptr) store4_any(e.pre, i * e.ld_pre + j, e.out_bf16, valid, v);
    act_values(v, e.act);
    if constexpr (SRC) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += t[q];
    }
    store4_any(e.out, i * e.ld_out + j, e.out_bf16, valid, v);
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = (SRC && e.src != nullptr ? fmaf(e.s1, t[q], e.s0 * v[q]) : e.s0 * v[q]) * by;
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
  if (e.out_plane != 0) {
    float hi[4], lo[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      hi[q] = (float)(_Float16)v[q];
      lo[q] = v[q] - hi[q];
    }
    store_piece<_Float16, 4>((_Float16*)e.out + at, valid, hi);
    store_piece<_Float16, 4>((_Float16*)e.out + at + e.out_plane, valid, lo);
    return;
  }
  if (e.base != nullptr) {
    float o[4];
    load4_any(e.base, at, e.out_bf16, valid, o);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = fmaf(e.s2, o[q], v[q]);
  }
  store4_any(e.out, at, e.out_bf16, valid, v);
}

// Workgroups go to the eight XCDs in turn.  Each XCD takes a run of neighbouring blocks, walked eight rows of blocks at a time,
// so that its L2 keeps the operand tiles they share.
__device__ __forceinline__ void block_of(int id, int tm, int tn, int* ti, int* tj) {
  const int total = tm * tn, q = total / 8, r = total % 8, x = id % 8, l = id / 8;
  id = (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + l;
  constexpr int kGroup = 8;
  const int g = id / (kGroup * tn), first = g * kGroup, rows = tm - first < kGroup ? tm - first : kGroup, in = id % (kGroup * tn);
  *ti = first + in % rows;
  *tj = in / rows;
}

__device__ __forceinline__ int quad_valid(int64_t i, int64_t j, int64_t M, int64_t N) { return i >= M || j >= N ? 0 : N - j < 4 ? (int)(N - j) : 4; }

// U quads of one column block: place(q, &i, &j) says where the q-th lies, sum(q) gives its four sums.
template <int U, class Place, class Sum>
__device__ __forceinline__ void epilogue_quads(const Epilogue& e, float by, int64_t b, int64_t M, int64_t N, const float (&bias)[4], Place place, Sum sum) {
  SrcQuad raw[U];
  int64_t i, j;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    place(u, &i, &j);
    raw[u] = epilogue_ask(e, b, i, j, quad_valid(i, j, M, N));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    place(u, &i, &j);
    const int valid = quad_valid(i, j, M, N);
    if (valid == 0) continue;
    const float4 t = sum(u);
    float v[4] = {t.x, t.y, t.z, t.w};
    epilogue4(e, by, b, i, j, valid, bias, raw[u], v);
  }
}

}  // namespace ilargi
#endif
