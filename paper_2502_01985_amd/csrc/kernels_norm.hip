// Norms around a residual sum, r = x + s f(gate) o N1(h), y = N2(r), and their gradients: a row stays in registers from its loads to
// its stores.
//
// W threads share a row; each holds P pieces of 16 bytes of it, W pieces apart.  A piece that would reach behind the row's end begins
// earlier instead, so that every load is a whole one: the columns that the neighbour holds already count as zeros here and are not
// stored ([lo, hi) is what a piece has of its own).  Bound by memory.
#include "ilargi_layers.h"

namespace ilargi {

namespace {

template <class T, int W, int P>
struct Row {
  static constexpr int V = ElemOf<T>::kVec, E = V * P, NT = W < 256 ? 256 : W, R = NT / W, kWaves = W / kWave;
  using Raw = Piece<T, V>;
  int c[P], lo[P], hi[P], m;

  __device__ __forceinline__ void plan(int64_t cols) {
    m = (int)cols;
    const int t = threadIdx.x % W;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = (t + W * p) * V;
      c[p] = m < V ? 0 : at < m - V ? at : m - V;
      lo[p] = at - c[p] < V ? at - c[p] : V;
      hi[p] = m < V ? m : V;
    }
  }
  __device__ __forceinline__ bool live(int p, int j) const { return j >= lo[p] && j < hi[p]; }
  __device__ __forceinline__ void load(const void* row, Raw (&r)[P]) const {
    const T* at = (const T*)row;
    if (m >= V) {
#pragma unroll
      for (int p = 0; p < P; ++p) r[p] = *reinterpret_cast<const Raw*>(at + c[p]);
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) r[p].v[j] = j < m ? at[j] : (T)0.0f;
    }
  }
  __device__ __forceinline__ void values(const Raw (&r)[P], float (&f)[E]) const {
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j) f[p * V + j] = live(p, j) ? (float)r[p].v[j] : 0.0f;
  }
  __device__ __forceinline__ void store(void* row, const float (&f)[E]) const {
    T* at = (T*)row;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if (lo[p] == 0 && hi[p] == V) {
        Raw r;
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = (T)f[p * V + j];
        *reinterpret_cast<Raw*>(at + c[p]) = r;
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (live(p, j)) at[c[p] + j] = (T)f[p * V + j];
      }
    }
  }
};

// Sums over the threads of a row, the same for all of them.  `turn` alternates between two places in LDS, so one barrier a sum is enough.
template <int W, int R, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*lds)[R * (W < kWave ? 1 : W / kWave)][2], int& turn) {
#pragma unroll
  for (int s = (W < kWave ? W : kWave) / 2; s >= 1; s /= 2)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], s);
  if constexpr (W > kWave) {
    constexpr int kWaves = W / kWave;
    const int wave = threadIdx.x / kWave, first = threadIdx.x / W * kWaves;
    if (threadIdx.x % kWave == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) lds[turn][wave][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = lds[turn][first][k];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v[k] += lds[turn][first + w][k];
    }
    turn ^= 1;
  }
}

// v normalised in place, before gain and bias; returns what it was multiplied by.
template <class L, int W, class Lds>
__device__ __forceinline__ float normalise(const L& row, int kind, float eps, float (&v)[L::E], Lds lds, int& turn) {
  if (kind == ILARGI_NORM_NONE) return 1.0f;
  constexpr int V = L::V, E = L::E;
  const float share = 1.0f / (float)row.m;
  float s[1];
  if (kind == ILARGI_NORM_CENTRED) {
    s[0] = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) s[0] += v[e];
    row_sums<W, L::R>(s, lds, turn);
    const float mean = s[0] * share;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = row.live(e / V, e % V) ? v[e] - mean : 0.0f;
  }
  s[0] = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) s[0] = fmaf(v[e], v[e], s[0]);
  row_sums<W, L::R>(s, lds, turn);
  const float by = 1.0f / sqrtf(fmaf(s[0], share, eps));
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] *= by;
  return by;
}

__device__ __forceinline__ const char* row_at(const void* p, int64_t i, int64_t ld, int size) { return (const char*)p + i * ld * size; }

template <class L, int P>
__device__ __forceinline__ void times_gain(const L& row, const void* is, const typename L::Raw (&gain)[P], float (&v)[L::E]) {
  if (is == nullptr) return;
#pragma unroll
  for (int e = 0; e < L::E; ++e) v[e] *= (float)gain[e / L::V].v[e % L::V];
}
template <class L, int P>
__device__ __forceinline__ void plus_bias(const L& row, const void* is, const typename L::Raw (&bias)[P], float (&v)[L::E]) {
  if (is == nullptr) return;
#pragma unroll
  for (int e = 0; e < L::E; ++e) v[e] += row.live(e / L::V, e % L::V) ? (float)bias[e / L::V].v[e % L::V] : 0.0f;
}

struct NormOut {
  void *r, *y;
  int64_t ld_r, ld_y;
};

template <class T, int W, int P>
__global__ __launch_bounds__(W < 256 ? 256 : W) void norm_kernel(ilargi_norm_t a, NormOut o) {
  using L = Row<T, W, P>;
  constexpr int E = L::E, R = L::R, S = sizeof(T);
  __shared__ float lds[2][R * (W < kWave ? 1 : W / kWave)][2];
  L row;
  row.plan(a.m);
  int turn = 0;
  typename L::Raw g1[P], b1[P], gr[P], g2[P], b2[P];
  if (a.gain1 != nullptr) row.load(a.gain1, g1);
  if (a.bias1 != nullptr) row.load(a.bias1, b1);
  if (a.gate != nullptr && !a.gate_rows) row.load(a.gate, gr);
  if (a.gain2 != nullptr) row.load(a.gain2, g2);
  if (a.bias2 != nullptr) row.load(a.bias2, b2);
  for (int64_t i0 = (int64_t)blockIdx.x * R; i0 < a.n; i0 += (int64_t)gridDim.x * R) {
    const int64_t mine = i0 + threadIdx.x / W, i = mine < a.n ? mine : a.n - 1;
    typename L::Raw h[P], x[P];
    row.load(row_at(a.h, i, a.ld_h, S), h);
    if (a.gate_rows) row.load(row_at(a.gate, i, a.ld_gate, S), gr);
    if (a.x != nullptr) row.load(row_at(a.x, i, a.ld_x, S), x);
    float v[E];
    row.values(h, v);
    normalise<L, W>(row, a.first, a.eps, v, lds, turn);
    times_gain(row, a.gain1, g1, v);
    plus_bias(row, a.bias1, b1, v);
    if (a.gate != nullptr) {
      float f[E];
      row.values(gr, f);
      act_values(f, a.gate_act);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] *= f[e];
    }
    if (a.x != nullptr) {
      float f[E];
      row.values(x, f);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = fmaf(a.scale, v[e], f[e]);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] *= a.scale;
    }
    if (o.r != nullptr && mine < a.n) row.store((char*)o.r + i * o.ld_r * S, v);
    if (a.second == ILARGI_NORM_NONE) continue;
    normalise<L, W>(row, a.second, a.eps, v, lds, turn);
    times_gain(row, a.gain2, g2, v);
    plus_bias(row, a.bias2, b2, v);
    if (o.y != nullptr && mine < a.n) row.store((char*)o.y + i * o.ld_y * S, v);
  }
}

// t becomes the gradient of what was normalised to `unit` by the factor `by`.
template <class L, int W, class Lds>
__device__ __forceinline__ void normalise_back(const L& row, int kind, float by, const float (&unit)[L::E], float (&t)[L::E], Lds lds, int& turn) {
  if (kind == ILARGI_NORM_NONE) return;
  constexpr int E = L::E;
  const float share = 1.0f / (float)row.m;
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    s[0] = fmaf(t[e], unit[e], s[0]);
    s[1] += t[e];
  }
  row_sums<W, L::R>(s, lds, turn);
  const float along = s[0] * share, mean = kind == ILARGI_NORM_CENTRED ? s[1] * share : 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) t[e] = by * (fmaf(-along, unit[e], t[e]) - (row.live(e / L::V, e % L::V) ? mean : 0.0f));
}

struct NormGradIn {
  const void *d_r, *d_y;
  int64_t ld_dr, ld_dy;
};
enum { kSumGain2, kSumBias2, kSumGate, kSumGain1, kSumBias1, kSums };

// The sums over this workgroup's rows go to partial[workgroup][sum][column].
template <class T, int W, int P>
__global__ __launch_bounds__(W < 256 ? 256 : W) void norm_grad_kernel(ilargi_norm_t a, NormGradIn d, ilargi_norm_grads_t o, float* __restrict__ partial) {
  using L = Row<T, W, P>;
  constexpr int E = L::E, R = L::R, V = L::V, S = sizeof(T);
  __shared__ float lds[2][R * (W < kWave ? 1 : W / kWave)][2];
  __shared__ float rows_sums[R > 1 ? R : 1][R > 1 ? W * E : 1];
  L row;
  row.plan(a.m);
  int turn = 0;
  typename L::Raw g1[P], b1[P], gr[P], g2[P];
  if (a.gain1 != nullptr) row.load(a.gain1, g1);
  if (a.bias1 != nullptr) row.load(a.bias1, b1);
  if (a.gate != nullptr && !a.gate_rows) row.load(a.gate, gr);
  if (a.gain2 != nullptr) row.load(a.gain2, g2);
  const bool second = a.second != ILARGI_NORM_NONE, gate_sum = o.d_gate != nullptr && !a.gate_rows;
  float sums[kSums][E];
#pragma unroll
  for (int q = 0; q < kSums; ++q)
#pragma unroll
    for (int e = 0; e < E; ++e) sums[q][e] = 0.0f;
  for (int64_t i0 = (int64_t)blockIdx.x * R; i0 < a.n; i0 += (int64_t)gridDim.x * R) {
    const int64_t mine = i0 + threadIdx.x / W, i = mine < a.n ? mine : a.n - 1;
    const bool is = mine < a.n;
    typename L::Raw h[P], x[P], dr[P], dy[P];
    row.load(row_at(a.h, i, a.ld_h, S), h);
    if (a.gate_rows) row.load(row_at(a.gate, i, a.ld_gate, S), gr);
    if (second && a.x != nullptr) row.load(row_at(a.x, i, a.ld_x, S), x);
    if (d.d_r != nullptr) row.load(row_at(d.d_r, i, d.ld_dr, S), dr);
    if (d.d_y != nullptr) row.load(row_at(d.d_y, i, d.ld_dy, S), dy);
    float unit[E];                                       // h normalised
    row.values(h, unit);
    const float by1 = normalise<L, W>(row, a.first, a.eps, unit, lds, turn);
    float u[E], f[E];
#pragma unroll
    for (int e = 0; e < E; ++e) u[e] = unit[e];
    times_gain(row, a.gain1, g1, u);
    plus_bias(row, a.bias1, b1, u);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = 1.0f;
    if (a.gate != nullptr) {
      row.values(gr, f);
      act_values(f, a.gate_act);
    }
    float t[E];                                          // the gradient on its way back: of r first
    if (d.d_r != nullptr) row.values(dr, t);
    else {
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] = 0.0f;
    }
    if (second && d.d_y != nullptr) {
      float r[E], back[E];
      if (a.x != nullptr) row.values(x, r);
#pragma unroll
      for (int e = 0; e < E; ++e) r[e] = a.x != nullptr ? fmaf(a.scale, f[e] * u[e], r[e]) : a.scale * (f[e] * u[e]);
      const float by2 = normalise<L, W>(row, a.second, a.eps, r, lds, turn);
      row.values(dy, back);
      if (is) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          sums[kSumGain2][e] = fmaf(back[e], r[e], sums[kSumGain2][e]);
          sums[kSumBias2][e] += back[e];
        }
      }
      times_gain(row, a.gain2, g2, back);
      normalise_back<L, W>(row, a.second, by2, r, back, lds, turn);
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] += back[e];
    }
    if (o.d_x != nullptr && is) row.store((char*)o.d_x + i * o.ld_x * S, t);
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] *= a.scale;
    if (o.d_gate != nullptr) {
      float slope[E];
      row.values(gr, slope);
#pragma unroll
      for (int e = 0; e < E; ++e) slope[e] = act_slope(slope[e], a.gate_act) * u[e] * t[e];
      if (gate_sum) {
        if (is) {
#pragma unroll
          for (int e = 0; e < E; ++e) sums[kSumGate][e] += slope[e];
        }
      } else if (is) {
        row.store((char*)o.d_gate + i * o.ld_gate * S, slope);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] *= f[e];
    if (is) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        sums[kSumGain1][e] = fmaf(t[e], unit[e], sums[kSumGain1][e]);
        sums[kSumBias1][e] += t[e];
      }
    }
    if (o.d_h == nullptr) continue;
    times_gain(row, a.gain1, g1, t);
    normalise_back<L, W>(row, a.first, by1, unit, t, lds, turn);
    if (is) row.store((char*)o.d_h + i * o.ld_h * S, t);
  }
  if (partial == nullptr) return;
  float* const to = partial + (int64_t)blockIdx.x * kSums * a.m;
  const void* const wanted[kSums] = {o.d_gain2, o.d_bias2, gate_sum ? o.d_gate : nullptr, o.d_gain1, o.d_bias1};
#pragma unroll
  for (int q = 0; q < kSums; ++q) {
    if (wanted[q] == nullptr) continue;
    if constexpr (R == 1) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (row.live(e / V, e % V)) to[(int64_t)q * a.m + row.c[e / V] + e % V] = sums[q][e];
    } else {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (row.live(e / V, e % V)) rows_sums[threadIdx.x / W][row.c[e / V] + e % V] = sums[q][e];
      __syncthreads();
      for (int j = threadIdx.x; j < a.m; j += L::NT) {
        float s = rows_sums[0][j];
#pragma unroll
        for (int r = 1; r < R; ++r) s += rows_sums[r][j];
        to[(int64_t)q * a.m + j] = s;
      }
    }
  }
}

// Adds the workgroups' sums, in float64: they cancel each other as the rows' parts do.  Sixteen threads share a column, each adds every
// sixteenth workgroup, then they are added in order.
template <class T>
__global__ __launch_bounds__(256) void norm_join_kernel(const float* __restrict__ partial, int groups, int64_t m, ilargi_norm_grads_t o, int gate_sum, int accumulate) {
  __shared__ double part[16][17];
  const int c = threadIdx.x % 16, q = threadIdx.x / 16, which = blockIdx.y;
  T* const out = (T*)(which == kSumGain2 ? o.d_gain2 : which == kSumBias2 ? o.d_bias2 : which == kSumGate ? (gate_sum ? o.d_gate : nullptr) : which == kSumGain1 ? o.d_gain1 : o.d_bias1);
  if (out == nullptr) return;
  const int64_t j = (int64_t)blockIdx.x * 16 + c;
  double s = 0.0;
  if (j < m) {
#pragma unroll 8
    for (int w = q; w < groups; w += 16) s += partial[((int64_t)w * kSums + which) * m + j];
  }
  part[q][c] = s;
  __syncthreads();
  if (q != 0 || j >= m) return;
  for (int u = 1; u < 16; ++u) s += part[u][c];
  out[j] = (T)(float)(accumulate ? (double)(float)out[j] + s : s);
}

// Threads of a row and pieces of a thread: the least that hold it.
template <class T, class F>
hipError_t by_columns(int64_t m, F f) {
  const int64_t pieces = (m + ElemOf<T>::kVec - 1) / ElemOf<T>::kVec;
  auto at = [&](auto w, auto p) { return f(w, p); };
  using std::integral_constant;
  if (pieces <= 16) return at(integral_constant<int, 16>(), integral_constant<int, 1>());
  if (pieces <= 64) return at(integral_constant<int, 64>(), integral_constant<int, 1>());
  if (pieces <= 128) return at(integral_constant<int, 128>(), integral_constant<int, 1>());
  if (pieces <= 256) return at(integral_constant<int, 256>(), integral_constant<int, 1>());
  if (pieces <= 512) return at(integral_constant<int, 512>(), integral_constant<int, 1>());
  if (pieces <= 1024) return at(integral_constant<int, 1024>(), integral_constant<int, 1>());
  if (pieces <= 2048) return at(integral_constant<int, 1024>(), integral_constant<int, 2>());
  if constexpr (ElemOf<T>::kVec == 4)
    if (pieces <= 4096) return at(integral_constant<int, 1024>(), integral_constant<int, 4>());
  return hipErrorInvalidValue;
}

int64_t groups_of(int64_t n, int rows, int64_t most) {
  const int64_t g = (n + rows - 1) / rows;
  return g < most ? g : most;
}

// Workgroups of the gradient: at most two of the larger ones fit a compute unit, and each leaves its sums behind.
template <class T>
int64_t grad_groups(int64_t n, int64_t m) {
  int64_t g = 0;
  const hipError_t e = by_columns<T>(m, [&](auto w, auto p) {
    using L = Row<T, decltype(w)::value, decltype(p)::value>;
    g = groups_of(n, L::R, L::NT == 256 ? 1024 : 512);
    return hipSuccess;
  });
  return e == hipSuccess ? g : 0;
}

template <class T>
hipError_t norm_typed(const ilargi_norm_t& a, const NormOut& o, hipStream_t st) {
  return by_columns<T>(a.m, [&](auto w, auto p) {
    constexpr int W = decltype(w)::value, P = decltype(p)::value;
    using L = Row<T, W, P>;
    norm_kernel<T, W, P><<<(unsigned)groups_of(a.n, L::R, 256 * (2048 / L::NT)), L::NT, 0, st>>>(a, o);
    return hipGetLastError();
  });
}

template <class T>
hipError_t norm_grad_typed(const ilargi_norm_t& a, const NormGradIn& d, const ilargi_norm_grads_t& o, int accumulate, float* partial, hipStream_t st) {
  const bool gate_sum = o.d_gate != nullptr && !a.gate_rows;
  const bool sums = gate_sum || o.d_gain1 != nullptr || o.d_bias1 != nullptr || o.d_gain2 != nullptr || o.d_bias2 != nullptr;
  if (!sums) partial = nullptr;
  const int64_t groups = grad_groups<T>(a.n, a.m);
  if (groups > 0) {
    const hipError_t e = by_columns<T>(a.m, [&](auto w, auto p) {
      constexpr int W = decltype(w)::value, P = decltype(p)::value;
      norm_grad_kernel<T, W, P><<<(unsigned)groups, Row<T, W, P>::NT, 0, st>>>(a, d, o, partial);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (sums) norm_join_kernel<T><<<dim3((unsigned)((a.m + 15) / 16), kSums), 256, 0, st>>>(partial, (int)groups, a.m, o, gate_sum, accumulate);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const ilargi_norm_t& a, void* r, int64_t ld_r, void* y, int64_t ld_y, hipStream_t st) {
  const NormOut o{r, y, ld_r, ld_y};
  return a.type == ILARGI_TYPE_BF16 ? norm_typed<bf16_t>(a, o, st) : norm_typed<float>(a, o, st);
}

size_t norm_grad_bytes(int64_t n, int64_t m, bool bf16) { return (size_t)(bf16 ? grad_groups<bf16_t>(n, m) : grad_groups<float>(n, m)) * kSums * (size_t)m * 4; }

hipError_t launch_norm_grad(const ilargi_norm_t& a, const void* d_r, int64_t ld_dr, const void* d_y, int64_t ld_dy, const ilargi_norm_grads_t& out,
                            int accumulate, float* partial, hipStream_t st) {
  const NormGradIn d{d_r, d_y, ld_dr, ld_dy};
  return a.type == ILARGI_TYPE_BF16 ? norm_grad_typed<bf16_t>(a, d, out, accumulate, partial, st) : norm_grad_typed<float>(a, d, out, accumulate, partial, st);
}

}  // namespace ilargi
