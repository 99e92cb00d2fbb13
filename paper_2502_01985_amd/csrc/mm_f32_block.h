// A block of a product in float32 on the matrix cores, for operands of either type, order, stride and alignment (kernels_mm.hip,
// kernels_grouped.hip).
#ifndef ILARGI_MM_F32_BLOCK_H_
#define ILARGI_MM_F32_BLOCK_H_

#include "mm_epilogue.h"

namespace ilargi {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// Eight elements of a TILE x STEP piece of an operand for every thread, as floats; zeros outside the matrix.
template <class T, bool KROWS, int TILE, int STEP>
__device__ __forceinline__ void fetch(const T* __restrict__ p, int64_t ld, int64_t r0, int64_t R, int64_t k0, int64_t K, float (&f)[8]) {
  static_assert(TILE * STEP == 8 * 256, "eight elements a thread");
  const int t = threadIdx.x;
  const int64_t outer = KROWS ? k0 + t / (TILE / 8) : r0 + t / (STEP / 8), inner = KROWS ? r0 + t % (TILE / 8) * 8 : k0 + t % (STEP / 8) * 8;
  const int64_t n_outer = KROWS ? K : R, n_inner = KROWS ? R : K;
  const int64_t left = outer < n_outer ? n_inner - inner : 0;
  const T* at = p + (left > 0 ? outer * ld + inner : 0);
  if (left >= 8) {
    const Piece<T, 8> t = *reinterpret_cast<const Piece<T, 8>*>(at);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (float)t.v[j];
  } else {
    // (places before the end alone are read: the last of them in place of those behind it)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = left > 0 ? (float)at[j < left ? j : 0] : 0.0f;
      f[j] = j < left ? v : 0.0f;
    }
  }
}

template <bool KROWS, int TILE, int STEP>
__device__ __forceinline__ void put(float (*lds)[TILE + 4], const float (&f)[8]) {
  const int t = threadIdx.x;
  if constexpr (KROWS) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<float4*>(&lds[t / (TILE / 8)][t % (TILE / 8) * 8 + 4 * h]) = make_float4(f[4 * h], f[4 * h + 1], f[4 * h + 2], f[4 * h + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) lds[t % (STEP / 8) * 8 + j][t / (STEP / 8)] = f[j];
  }
}

template <int TILE, int STEP>
struct MmF32Lds {
  float p[3][STEP][TILE + 4], q[3][STEP][TILE + 4];
};

// A workgroup forms block (ti, tj) of TILE x TILE sums of matrix b of the batch over share z of k, a wavefront a quarter of them, STEP k
// at a time from LDS while the next are fetched.  The columns of the result are the first operand of the matrix instruction: a lane
// then holds four neighbouring columns.  With `sums_to` the sums go there, a matrix of M x (N to a multiple of 4).
template <class TP, class TQ, bool PK, bool QK, int TILE, int STEP>
__device__ __forceinline__ void mm_f32_block(const Product& a, int ti, int tj, int64_t b, int64_t z, int64_t share, float* __restrict__ sums_to, MmF32Lds<TILE, STEP>& lds) {
  constexpr int F = TILE / 64;        // 32 x 32 pieces of a wavefront, each way
  auto& lp = lds.p;
  auto& lq = lds.q;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t i0 = (int64_t)ti * TILE, j0 = (int64_t)tj * TILE;
  const int64_t first = z * share, K = a.K < first + share ? a.K : first + share;
  const TP* P = (const TP*)a.P.p + b * a.P.batch;
  const TQ* Q = (const TQ*)a.Q.p + b * a.Q.batch;
  const int wi = (wave / 2) * (TILE / 2), wj = (wave % 2) * (TILE / 2), r = lane % 32, h = lane / 32;
  f32x16 acc[F][F];
#pragma unroll
  for (int x = 0; x < F; ++x)
#pragma unroll
    for (int y = 0; y < F; ++y)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[x][y][q] = 0.0f;
  // Three tiles of each operand: at the start of a step its own and the next lie in LDS, and the one behind is fetched, to be put
  // where the last step's was.  So the first fragments of the next step are read before the barrier, and the products go on behind it.
  float fp[8], fq[8];
  auto bring = [&](int64_t k) {
    fetch<TP, PK, TILE, STEP>(P, a.P.ld, i0, a.M, k, K, fp);
    fetch<TQ, QK, TILE, STEP>(Q, a.Q.ld, j0, a.N, k, K, fq);
  };
  auto lay = [&](int to) {
    put<PK, TILE, STEP>(lp[to], fp);
    put<QK, TILE, STEP>(lq[to], fq);
  };
  float p[2][F], q[2][F];
  auto read = [&](int of, int k, int set) {
#pragma unroll
    for (int x = 0; x < F; ++x) p[set][x] = lp[of][k + h][wi + 32 * x + r];
#pragma unroll
    for (int y = 0; y < F; ++y) q[set][y] = lq[of][k + h][wj + 32 * y + r];
  };
  if (first < K) {
    bring(first);
    lay(0);
    if (first + STEP < K) {
      bring(first + STEP);
      lay(1);
    }
  }
  __syncthreads();
  int cur = 0;
  if (first < K) read(0, 0, 0);
  for (int64_t k0 = first; k0 < K; k0 += STEP) {
    const int next = cur == 2 ? 0 : cur + 1, last = cur == 0 ? 2 : cur - 1;
    const bool more = k0 + 2 * STEP < K;
    if (more) bring(k0 + 2 * STEP);
#pragma unroll
    for (int k = 0; k < STEP; k += 2) {
      const int set = k / 2 % 2;
      if (k + 2 < STEP) read(cur, k + 2, set ^ 1);
      else read(next, 0, set ^ 1);                     // (behind the last step: of an old one, for nothing)
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < F; ++x)
#pragma unroll
        for (int y = 0; y < F; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x2f32(q[set][y], p[set][x], acc[x][y], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    static_assert(STEP / 2 % 2 == 0, "the next step begins with the first set");
    if (more) lay(last);
    cur = next;
    __syncthreads();
  }
  // The sums go through LDS, 32 rows of a wavefront at a time, so that stores run along the result's rows.
  constexpr int kPad = 32 * F + 4, kLanes = 8 * F, kRows = 64 / kLanes;      // quads of a row, rows of a turn
  static_assert(4 * 32 * kPad * 4 <= sizeof(lds), "the sums fit where the tiles were");
  float* mine = reinterpret_cast<float*>(&lds) + wave * 32 * kPad;
  const int64_t ldp = (a.N + 3) / 4 * 4;
  const int rr = lane / kLanes, cc = lane % kLanes * 4;
  const int64_t j = j0 + wj + cc;
  float bias[4];
  epilogue_bias(a.epi, j, (int)(a.N - j < 4 ? a.N - j : 4), bias);
#pragma unroll
  for (int x = 0; x < F; ++x) {
#pragma unroll
    for (int y = 0; y < F; ++y)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(mine + r * kPad + 32 * y + 8 * g + 4 * h) =
            make_float4(acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int64_t ri = i0 + wi + 32 * x;
    auto sums = [&](int q) { return *reinterpret_cast<const float4*>(mine + (q * kRows + rr) * kPad + cc); };
    if (sums_to != nullptr) {
#pragma unroll 4
      for (int q = 0; q < 32 / kRows; ++q)
        if (ri + q * kRows + rr < a.M && j < a.N) *reinterpret_cast<float4*>(sums_to + (ri + q * kRows + rr) * ldp + j) = sums(q);
    } else if (!a.epi.flip) {
#pragma unroll 1
      for (int q = 0; q < 32 / kRows; q += 4)
        epilogue_quads<4>(a.epi, 1.0f, b, a.M, a.N, bias, [&](int u, int64_t* i, int64_t* jj) { *i = ri + (q + u) * kRows + rr; *jj = j; }, [&](int u) { return sums(q + u); });
    } else {                                           // written along j's rows, which run over i
#pragma unroll 1
      for (int q = 0; q < 4 * F; q += 4)
        epilogue_quads<4>(a.epi, 1.0f, b, a.M, a.N, bias, [&](int u, int64_t* i, int64_t* jj) { *i = ri + r; *jj = j0 + wj + 8 * (q + u) + 4 * h; },
                          [&](int u) { return *reinterpret_cast<const float4*>(mine + r * kPad + 8 * (q + u) + 4 * h); });
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace

}  // namespace ilargi
#endif
