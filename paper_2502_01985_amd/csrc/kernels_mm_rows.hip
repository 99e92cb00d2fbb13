// Products of a few rows with a whole matrix: serving.  W is read once, and every element of it multiplies the few rows' values in
// vector registers.
//
// A workgroup takes a line (128 bytes) of every row of W, 128 rows at a time, eight turns of which (four of two rows of bfloat16) are on
// their way at once; its share of k is at most 1024 rows, and a second launch adds the shares, where there are several.  Longer shares in fewer launches are slower where W
// comes from memory: 1 x 4096 x 4096, bfloat16, 15.3 us with shares of 1024 rows and 27.9 with one share; 1 x 8192 x 1000 14.1
// and 45.3.  Blocks on the matrix cores take 17.5 and 13.4 for the same.
// With W in the last-level cache the 4096 x 4096 call takes 13 us.
#include "mm_epilogue.h"

namespace ilargi {

namespace {

constexpr int kThreads = 1024, kLanes = 8, kSubs = kThreads / kLanes;     // lanes of 16 bytes side by side, rows of W at a time
constexpr int kWaves = kThreads / kWave;
constexpr int kMostShare = 1024;                                          // rows of W of a workgroup

// blockIdx: columns kLanes V wide, share of k.  N: rows of X that the registers have room for.
template <class T, int N>
__global__ __launch_bounds__(kThreads) void mm_rows_kernel(Product a, int64_t share, float* __restrict__ partial) {
  constexpr int V = ElemOf<T>::kVec, kCols = kLanes * V, U = N * V > 8 && V == 8 ? 4 : 8;       // (128 registers a lane)
  __shared__ union {
    float x[N][kMostShare];
    float sums[kWaves][N][kCols];
  } lds;
  const int lane = threadIdx.x % kLanes, sub = threadIdx.x / kLanes, wave = threadIdx.x / kWave;
  const int64_t j = (int64_t)blockIdx.x * kCols + lane * V, k0 = blockIdx.y * share, k1 = k0 + share < a.K ? k0 + share : a.K;
  const int n = (int)a.M, rows = (int)(k1 - k0);
  const T* W = (const T*)a.Q.p + k0 * a.Q.ld + j;
  const int valid = (int)(a.N - j < 0 ? 0 : a.N - j < V ? a.N - j : V);
  Piece<T, V> w[U];
  auto ask = [&](int r) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = r + u * kSubs;
      if (q < rows && valid == V) {
        w[u] = *reinterpret_cast<const Piece<T, V>*>(W + q * a.Q.ld);
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) w[u].v[v] = q < rows && v < valid ? W[q * a.Q.ld + v] : (T)0.0f;
      }
    }
  };
  // The rows of X first: what is asked for first arrives first, and goes into LDS while W is on its way.
  static_assert(kMostShare == kThreads, "a k a thread");
  const int k = threadIdx.x;
  T f[N];
#pragma unroll
  for (int x = 0; x < N; ++x) f[x] = x < n && k < rows ? ((const T*)a.P.p)[x * a.P.ld + k0 + k] : (T)0.0f;
  ask(sub);
  float s[N][V];
#pragma unroll
  for (int r = 0; r < N; ++r)
#pragma unroll
    for (int v = 0; v < V; ++v) s[r][v] = 0.0f;
#pragma unroll
  for (int x = 0; x < N; ++x) lds.x[x][k] = (float)f[x];
  __syncthreads();
  for (int r = sub; r < rows; r += U * kSubs) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = r + u * kSubs;
      if (q >= rows) continue;
#pragma unroll
      for (int x = 0; x < N; ++x) {
        const float f = lds.x[x][q];
#pragma unroll
        for (int v = 0; v < V; ++v) s[x][v] = fmaf(f, (float)w[u].v[v], s[x][v]);
      }
    }
    if (r + U * kSubs < rows) ask(r + U * kSubs);
  }
  __syncthreads();
  // the eight rows of W that a wavefront holds side by side, then the wavefronts in order
#pragma unroll
  for (int x = 0; x < N; ++x)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float t = s[x][v];
      t += __shfl_xor(t, 8);
      t += __shfl_xor(t, 16);
      t += __shfl_xor(t, 32);
      if (threadIdx.x % kWave < kLanes) lds.sums[wave][x][lane * V + v] = t;
    }
  __syncthreads();
  const int64_t ldp = (a.N + 3) / 4 * 4;
  const int r = threadIdx.x / (kCols / 4), c = threadIdx.x % (kCols / 4) * 4;
  const int64_t col = (int64_t)blockIdx.x * kCols + c;
  if (r >= n || col >= a.N) return;
  const int left = (int)(a.N - col < 4 ? a.N - col : 4);
  const SrcQuad raw = epilogue_ask(a.epi, 0, r, col, left);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w2 = 0; w2 < kWaves; ++w2)
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += lds.sums[w2][r][c + q];
  if (partial != nullptr) {
    *reinterpret_cast<float4*>(partial + (blockIdx.y * a.M + r) * ldp + col) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
  float bias[4];
  epilogue_bias(a.epi, col, left, bias);
  epilogue4(a.epi, 1.0f, 0, r, col, left, bias, raw, v);
}

template <class T>
hipError_t mm_rows_typed(const Product& a, const MmPlan& plan, float* partial, hipStream_t st) {
  const int64_t cols = kLanes * ElemOf<T>::kVec, share = (a.K + plan.splits - 1) / plan.splits;
  const dim3 grid((unsigned)((a.N + cols - 1) / cols), (unsigned)plan.splits);
  float* part = plan.splits > 1 ? partial : nullptr;
  if (a.M == 1) mm_rows_kernel<T, 1><<<grid, kThreads, 0, st>>>(a, share, part);
  else if (a.M == 2) mm_rows_kernel<T, 2><<<grid, kThreads, 0, st>>>(a, share, part);
  else if constexpr (ElemOf<T>::kVec == 4) mm_rows_kernel<T, 4><<<grid, kThreads, 0, st>>>(a, share, part);
  else return hipErrorInvalidValue;
  if (part != nullptr) return launch_mm_join(a.M, a.N, 1, 0, a.epi, plan.splits, part, st);
  return hipGetLastError();
}

}  // namespace

// Up to two rows of bfloat16, four of float32: with more the vector units take longer than blocks on the matrix cores do (4096 x
// 4096, bfloat16, 4 rows: 30.6 us against 17.7 in blocks; float32, 4 rows: 26.5 against 32, 8 rows: 37.8).
bool mm_rows_takes(int64_t M, int64_t K, bool bf16) { return M <= (bf16 ? 2 : 4) && K <= 65535 * (int64_t)kMostShare; }

MmPlan mm_rows_plan(int64_t M, int64_t N, int64_t K) {
  MmPlan p{0, 1, 0};
  const int64_t splits = (K + kMostShare - 1) / kMostShare, share = (K + splits - 1) / splits;
  p.splits = (int)((K + share - 1) / share);
  if (p.splits > 1) p.partial_bytes = (size_t)p.splits * (size_t)M * (size_t)((N + 3) / 4 * 4) * 4;
  return p;
}

hipError_t launch_mm_rows(const Product& a, const MmPlan& plan, float* partial, hipStream_t st) {
  if (a.M == 0 || a.N == 0) return hipSuccess;
  if (!mm_rows_takes(a.M, a.K, a.P.bf16) || a.P.k_rows || !a.Q.k_rows || a.batches != 1 || a.K < 1 || a.P.bf16 != a.Q.bf16)
    return hipErrorInvalidValue;
  const int64_t cols = kLanes * (a.P.bf16 ? ElemOf<bf16_t>::kVec : ElemOf<float>::kVec);
  return in_blocks(a, a.M, cols, kThreads, [&](const Product& b) {
    return b.P.bf16 ? mm_rows_typed<bf16_t>(b, plan, partial, st) : mm_rows_typed<float>(b, plan, partial, st);
  });
}

}  // namespace ilargi
