// Matrix products in float32 on the matrix cores, for operands of either type, order, stride and alignment, and the
// elementwise pass of a layer's gradient.
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

// A workgroup forms TILE x TILE sums over a share of k, a wavefront a quarter of them, STEP k at a time from LDS while the next are
// fetched.  The columns of the result are the first operand of the matrix instruction: a lane then holds four neighbouring columns.
// blockIdx: block, matrix of the batch, share.  With several shares the sums go to `partial`, as in kernels_mm16.hip.
template <class TP, class TQ, bool PK, bool QK, int TILE, int STEP>
__global__ __launch_bounds__(256) void mm_f32_kernel(Product a, int tm, int tn, int64_t share, float* __restrict__ partial) {
  constexpr int F = TILE / 64;        // 32 x 32 pieces of a wavefront, each way
  __shared__ __attribute__((aligned(16))) struct {
    float p[3][STEP][TILE + 4], q[3][STEP][TILE + 4];
  } lds;
  auto& lp = lds.p;
  auto& lq = lds.q;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  int ti, tj;
  block_of(blockIdx.x, tm, tn, &ti, &tj);
  const int64_t i0 = (int64_t)ti * TILE, j0 = (int64_t)tj * TILE, b = blockIdx.y;
  const int64_t first = blockIdx.z * share, K = a.K < first + share ? a.K : first + share;
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
  float* part = partial != nullptr ? partial + ((int64_t)blockIdx.z * a.batches + b) * a.M * ldp : nullptr;
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
    if (part != nullptr) {
#pragma unroll 4
      for (int q = 0; q < 32 / kRows; ++q)
        if (ri + q * kRows + rr < a.M && j < a.N) *reinterpret_cast<float4*>(part + (ri + q * kRows + rr) * ldp + j) = sums(q);
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

template <class TP, class TQ, bool PK, bool QK>
hipError_t mm_f32_order(const Product& a, const MmPlan& plan, float* partial, hipStream_t st) {
  const int64_t tm = (a.M + plan.tile - 1) / plan.tile, tn = (a.N + plan.tile - 1) / plan.tile;
  const dim3 grid((unsigned)(tm * tn), (unsigned)a.batches, (unsigned)plan.splits);
  const int64_t step = plan.tile == 64 ? 32 : 16, steps = (a.K + step - 1) / step, share = (steps + plan.splits - 1) / plan.splits * step;
  float* part = plan.splits > 1 ? partial : nullptr;
  if (plan.tile == 64) mm_f32_kernel<TP, TQ, PK, QK, 64, 32><<<grid, 256, 0, st>>>(a, (int)tm, (int)tn, share, part);
  else mm_f32_kernel<TP, TQ, PK, QK, 128, 16><<<grid, 256, 0, st>>>(a, (int)tm, (int)tn, share, part);
  if (part != nullptr) return launch_mm_join(a.M, a.N, a.batches, 0, a.epi, plan.splits, part, st);
  return hipGetLastError();
}

template <class TP, class TQ>
hipError_t mm_f32_typed(const Product& a, const MmPlan& plan, float* partial, hipStream_t st) {
  if (a.P.k_rows) return a.Q.k_rows ? mm_f32_order<TP, TQ, true, true>(a, plan, partial, st) : hipErrorInvalidValue;
  return a.Q.k_rows ? mm_f32_order<TP, TQ, false, true>(a, plan, partial, st) : mm_f32_order<TP, TQ, false, false>(a, plan, partial, st);
}

}  // namespace

// Blocks of 128 or 64 and the shares of k, by what they cost in microseconds: a step (16 k of a 128-block, 32 of a 64-block) keeps a
// compute unit's matrix cores busy for 0.8 or 0.47 and takes 1.1 or 0.8 alone; shares as in kernels_mm16.hip.  Measured: 8192 x 2048
// x 2048, 128-blocks 570 us (121 TFLOP/s, the library's product 468), 64-blocks 617; 512 x 2048 x 2048 50 (library 36); 1003 x 333 x 517
// 16 (library 18).
MmPlan mm_f32_plan(int64_t M, int64_t N, int64_t K, int64_t batches) {
  MmPlan best{128, 1, 0};
  double least = 1e300;
  for (int tile = 128; tile >= 64; tile /= 2) {
    const int64_t blocks = ((M + tile - 1) / tile) * ((N + tile - 1) / tile) * batches;
    const int64_t step = tile == 64 ? 32 : 16, steps = K > step ? (K + step - 1) / step : 1;
    for (int64_t splits = 1; splits <= 64 && splits <= steps; ++splits) {
      const int64_t share = (steps + splits - 1) / splits, groups = blocks * splits;
      if (splits > 1 && ((steps + share - 1) / share != splits || groups > 2048)) continue;
      const double rounds = (double)((groups + 255) / 256), work = tile == 64 ? 0.47 : 0.8, alone = tile == 64 ? 0.8 : 1.1;
      double cost = (double)share * (rounds * work > alone ? rounds * work : alone);
      const double bytes = (double)groups / (double)blocks * (double)batches * (double)M * (double)((N + 3) / 4 * 4) * 4.0;
      if (splits > 1) cost += 3.0 + 2.0 * bytes / 8e6;
      if (cost < least) {
        least = cost;
        best = {tile, (int)splits, splits > 1 ? (size_t)bytes : 0};
      }
    }
  }
  return best;
}

hipError_t launch_mm_f32(const Product& a, const MmPlan& plan, float* partial, hipStream_t st) {
  if (a.M == 0 || a.N == 0 || a.batches == 0) return hipSuccess;
  if (a.P.bf16 != a.Q.bf16) return hipErrorInvalidValue;
  return in_blocks(a, plan.tile, plan.tile, 256, [&](const Product& b) {
    return b.P.bf16 ? mm_f32_typed<bf16_t, bf16_t>(b, plan, partial, st) : mm_f32_typed<float, float>(b, plan, partial, st);
  });
}

// --------------------------------------------------------------------------------------- elementwise pass of a gradient
namespace {

constexpr int kBiasChunks = 256;

// g = d_out f'(pre), written in the layer's type; column sums of the unrounded g over this workgroup's rows.  bfloat16 layers round g
// for the two products, which read it as they read every operand: d_X and d_W are off by 2.3e-3 of themselves where one rounding is
// 1.7e-3.  Two planes of bfloat16 would keep it and double both products (8192 x 4096 x 4096: 222 us each of the call's 500); on the
// float32 cores the call took 11.8 ms.
// 32 lanes of four columns (`first` workgroups of them in earlier launches), eight rows at a time.  Bound by memory: 8192 x 4096, bfloat16, gelu 51 us for 201 MB (3.9 TB/s).
template <class T>
__global__ __launch_bounds__(256) void layer_grad_kernel(LayerGradArgs a, int64_t first, int64_t rows_per, float* __restrict__ partial) {
  __shared__ float4 part[8][32];
  const int cl = threadIdx.x % 32, rl = threadIdx.x / 32;
  const int64_t j = ((first + blockIdx.x) * 32 + cl) * 4;
  const int64_t r0 = (int64_t)blockIdx.y * rows_per, r1 = r0 + rows_per < a.n ? r0 + rows_per : a.n;
  const int valid = (int)(a.m - j < 0 ? 0 : a.m - j < 4 ? a.m - j : 4);
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (valid > 0 || (a.dz != nullptr && j < a.ld_dz)) {
    for (int64_t i = r0 + rl; i < r1; i += 8) {
      float g[4];
      load_piece<T, 4>((const T*)a.d_out + i * a.ld_out + (valid > 0 ? j : 0), valid, g);
      if (a.act != ILARGI_ACT_NONE) {
        float z[4];
        load_piece<T, 4>((const T*)a.pre + i * a.ld_pre + (valid > 0 ? j : 0), valid, z);
#pragma unroll
        for (int q = 0; q < 4; ++q) g[q] *= act_slope(z[q], a.act);
      }
      // (rows of dz are whole pieces of eight, with zeros behind their end)
      if (a.dz != nullptr) store_piece<T, 4>((T*)a.dz + i * a.ld_dz + j, 4, g);
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] += g[q];
    }
  }
  if (partial == nullptr) return;
  part[rl][cl] = make_float4(s[0], s[1], s[2], s[3]);
  __syncthreads();
  if (rl == 0 && valid > 0) {
    float4 t = part[0][cl];
    for (int q = 1; q < 8; ++q) { t.x += part[q][cl].x; t.y += part[q][cl].y; t.z += part[q][cl].z; t.w += part[q][cl].w; }
    const float f[4] = {t.x, t.y, t.z, t.w};
    store_piece<float, 4>(partial + blockIdx.y * a.m + j, valid, f);
  }
}

// Sixteen threads share a column: each adds every sixteenth chunk, then they are added in order.
template <class T>
__global__ __launch_bounds__(256) void bias_sum_kernel(const float* __restrict__ partial, int chunks, int64_t m, int64_t first, int accumulate, T* __restrict__ out) {
  __shared__ float part[16][17];
  const int c = threadIdx.x % 16, q = threadIdx.x / 16;
  const int64_t j = (first + blockIdx.x) * 16 + c;
  float s = 0.0f;
  if (j < m) {
#pragma unroll
    for (int u = 0; u < kBiasChunks / 16; ++u)
      if (16 * u + q < chunks) s += partial[(16 * u + q) * m + j];
  }
  part[q][c] = s;
  __syncthreads();
  if (q != 0 || j >= m) return;
  for (int u = 1; u < 16; ++u) s += part[u][c];
  out[j] = (T)(accumulate ? (float)out[j] + s : s);
}

int64_t bias_rows(int64_t n) {
  int64_t rows = (n + kBiasChunks - 1) / kBiasChunks;
  return rows < 32 ? 32 : (rows + 7) / 8 * 8;
}

}  // namespace

size_t layer_grad_partial_bytes(int64_t n, int64_t m) {
  const int64_t per = bias_rows(n), chunks = (n + per - 1) / per;
  return (size_t)chunks * (size_t)m * 4;
}

hipError_t launch_layer_grad(const LayerGradArgs& a, float* partial, hipStream_t st) {
  const int64_t per = bias_rows(a.n), chunks = (a.n + per - 1) / per;
  if (a.d_bias == nullptr) partial = nullptr;
  if (chunks > 0 && (a.dz != nullptr || partial != nullptr)) {
    const hipError_t e = in_parts(((a.dz != nullptr ? a.ld_dz : a.m) + 127) / 128, 256, [&](int64_t first, unsigned blocks) {
      const dim3 grid(blocks, (unsigned)chunks);
      if (a.bf16) layer_grad_kernel<bf16_t><<<grid, 256, 0, st>>>(a, first, per, partial);
      else layer_grad_kernel<float><<<grid, 256, 0, st>>>(a, first, per, partial);
    });
    if (e != hipSuccess) return e;
  }
  if (a.d_bias == nullptr) return hipGetLastError();
  return in_parts((a.m + 15) / 16, 256, [&](int64_t first, unsigned blocks) {
    if (a.bf16) bias_sum_kernel<bf16_t><<<blocks, 256, 0, st>>>(partial, (int)chunks, a.m, first, a.accumulate, (bf16_t*)a.d_bias);
    else bias_sum_kernel<float><<<blocks, 256, 0, st>>>(partial, (int)chunks, a.m, first, a.accumulate, (float*)a.d_bias);
  });
}

}  // namespace ilargi
