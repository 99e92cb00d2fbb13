// Matrix products in float32 on the matrix cores, for operands of either type, order, stride and alignment, and the
// elementwise pass of a layer's gradient.
#include "mm_f32_block.h"

namespace ilargi {

namespace {

// blockIdx: block, matrix of the batch, share.  With several shares the sums go to `partial`, as in kernels_mm16.hip.
template <class TP, class TQ, bool PK, bool QK, int TILE, int STEP>
__global__ __launch_bounds__(256) void mm_f32_kernel(Product a, int tm, int tn, int64_t share, float* __restrict__ partial) {
  __shared__ __attribute__((aligned(16))) MmF32Lds<TILE, STEP> lds;
  int ti, tj;
  block_of(blockIdx.x, tm, tn, &ti, &tj);
  mm_f32_block<TP, TQ, PK, QK, TILE, STEP>(a, ti, tj, blockIdx.y, blockIdx.z, share,
                                               partial != nullptr ? partial + ((int64_t)blockIdx.z * a.batches + blockIdx.y) * a.M * ((a.N + 3) / 4 * 4) : nullptr, lds);
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
