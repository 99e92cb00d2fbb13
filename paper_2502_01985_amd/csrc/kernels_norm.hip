// Norms around a residual sum, r = x + s f(gate) o N1(h), y = N2(r), and their gradients: a row stays in registers from its loads to
// its stores.
//
// W threads share a row; each holds P pieces of 16 bytes of it, W pieces apart.  A piece that would reach behind the row's end begins
// earlier instead, so that every load is a whole one: the columns that the neighbour holds already count as zeros here and are not
// stored ([lo, hi) is what a piece has of its own).  Rows of whole pieces have only pieces of their own and others.
//
// Bound by memory: 16384 x 4096, bfloat16, rms on both sides 95 us for 537 MB (5.7 TB/s; two workgroups a compute unit, with three 108); the
// gradient of 8192 x 4096 with gates 121 for 537 MB (4.4) and of 100,000 x 220, float32, 103 for 528 MB (5.1), with 6 for the sums over rows.  By the
// vector units where all sums are wanted of narrower bfloat16 rows (30,000 x 768, centred on both sides: 103 us for 276 MB).  Gradients of float32 rows of 4097
// columns and more, and of bfloat16 rows of 8193 and more, do not fit the registers, nor do norms of more than 8192: what spills grows from 20 of a
// thread's registers to 660 (1800 x 16384, float32, centred on both sides with all sums: 975 us for 708 MB; the norm alone, rms on both sides, 112 for 472).
#include "ilargi_layers.h"

namespace ilargi {

namespace {

enum { kFull, kWhole, kRagged, kShort };       // rows that fill their threads; of whole pieces; of any length; shorter than a piece

template <class T, int W, int P, int SHAPE>
struct Row {
  static constexpr int kW = W, kP = P, V = ElemOf<T>::kVec, E = V * P, NT = W < 256 ? 256 : W, R = NT / W;
  static constexpr int kShape = SHAPE;
  // which of the R rows side by side: the same for a whole wavefront, where it can be
  static __device__ __forceinline__ int slot() {
    if constexpr (R == 1) return 0;
    else if constexpr (W >= kWave) return __builtin_amdgcn_readfirstlane(threadIdx.x / W);
    else return threadIdx.x / W;
  }
  using Raw = Piece<T, V>;
  int c[P], lo[P], hi[P], m;
  uint32_t keep[SHAPE >= kRagged ? P : 1][4];      // the bits of a piece that are the thread's own

  __device__ __forceinline__ void plan(int64_t cols) {
    m = (int)cols;
    const int t = threadIdx.x % W;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int at = (t + W * p) * V;
      c[p] = SHAPE == kShort ? 0 : at < m - V ? at : m - V;
      lo[p] = at - c[p] < V ? at - c[p] : V;
      hi[p] = SHAPE == kShort ? m : V;
      if constexpr (SHAPE >= kRagged) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          keep[p][w] = V == 4 ? (live(p, w) ? ~0u : 0u) : (live(p, 2 * w) ? 0xffffu : 0u) | (live(p, 2 * w + 1) ? 0xffff0000u : 0u);
          asm volatile("" : "+v"(keep[p][w]));     // (held: worked out again at each use they cost more than the products)
        }
      }
    }
  }
  __device__ __forceinline__ void own(Raw& r, int p) const {
    if constexpr (SHAPE >= kRagged) {
      uint4 w = __builtin_bit_cast(uint4, r);
      w.x &= keep[p][0]; w.y &= keep[p][1]; w.z &= keep[p][2]; w.w &= keep[p][3];
      r = __builtin_bit_cast(Raw, w);
    }
  }
  // v, or 0 for a column that is another thread's or none
  __device__ __forceinline__ float own(float v, int e) const {
    if constexpr (SHAPE == kFull) return v;
    if constexpr (SHAPE == kWhole) return lo[e / V] == 0 ? v : 0.0f;
    const int p = e / V, j = e % V;
    const uint32_t bits = V == 4 ? keep[p][j] : (uint32_t)(j % 2 != 0 ? (int)keep[p][j / 2] >> 16 : (int)(keep[p][j / 2] << 16) >> 16);
    return __uint_as_float(__float_as_uint(v) & bits);
  }
  __device__ __forceinline__ bool live(int p, int j) const { return SHAPE == kFull || (SHAPE == kWhole ? lo[p] == 0 : SHAPE == kRagged ? j >= lo[p] : lo[p] == 0 && j < hi[p]); }
  __device__ __forceinline__ void load(const void* row, Raw (&r)[P]) const {
    const T* at = (const T*)row;
    if constexpr (SHAPE != kShort) {
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
    for (int p = 0; p < P; ++p) {
      Raw mine = r[p];
      own(mine, p);
#pragma unroll
      for (int j = 0; j < V; ++j) f[p * V + j] = SHAPE != kWhole || lo[p] == 0 ? (float)mine.v[j] : 0.0f;
    }
  }
  // a gain or a bias, for good: zeros in others' columns, where a number that is not finite would spoil the sums
  __device__ __forceinline__ void load_vector(const void* at, Raw (&r)[P]) const {
    if (at == nullptr) return;
    load(at, r);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      own(r[p], p);
      if constexpr (SHAPE == kWhole)
        if (lo[p] != 0) r[p] = __builtin_bit_cast(Raw, make_uint4(0, 0, 0, 0));
    }
  }
  __device__ __forceinline__ void store(void* row, const float (&f)[E], bool past) const {
    T* at = (T*)row;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if (SHAPE == kFull || (SHAPE != kShort && lo[p] == 0)) {
        Raw r;
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = (T)f[p * V + j];
        if (past) {
          typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
          __builtin_nontemporal_store(__builtin_bit_cast(words, r), reinterpret_cast<words*>(at + c[p]));
        } else {
          *reinterpret_cast<Raw*>(at + c[p]) = r;
        }
      } else if (SHAPE >= kRagged) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (live(p, j)) at[c[p] + j] = (T)f[p * V + j];
      }
    }
  }
};

template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// Sums over the threads of a row (4 at least), the same for all of them: over sixteen lanes by lane permutations of the vector units (through LDS,
// each of the six steps of a wavefront would wait a hundred cycles), then wavefronts through LDS.  `turn` alternates between two
// places there, so one barrier a sum is enough.
template <int W, int R>
struct RowLds {
  static constexpr int kWaves = W < kWave ? 1 : W / kWave;
  float v[2][2][R * kWaves];
  double wide[2][R * kWaves];
};
template <int W, int R, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], RowLds<W, R>& lds, int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] += from_lane<0xB1>(v[k]);       // lanes 1 away
    v[k] += from_lane<0x4E>(v[k]);       // 2 away
    if constexpr (W >= 8) v[k] += from_lane<0x141>(v[k]);       // mirrored in eight
    if constexpr (W >= 16) v[k] += from_lane<0x140>(v[k]);      // mirrored in sixteen
    if constexpr (W >= kWave) v[k] = (lane_value(v[k], 0) + lane_value(v[k], 16)) + (lane_value(v[k], 32) + lane_value(v[k], 48));
  }
  if constexpr (W > kWave) {
    constexpr int kWaves = W / kWave;
    const int wave = threadIdx.x / kWave, first = threadIdx.x / W * kWaves;
    if (threadIdx.x % kWave == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) lds.v[turn][k][wave] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = lds.v[turn][k][first];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v[k] += lds.v[turn][k][first + w];
    }
    turn ^= 1;
  }
}

template <int CTRL>
__device__ __forceinline__ double from_lane(double v) {
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, true), __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
// The same for one sum in float64.
template <int W, int R>
__device__ __forceinline__ double row_sum(double v, RowLds<W, R>& lds, int& turn) {
  v += from_lane<0xB1>(v);
  v += from_lane<0x4E>(v);
  if constexpr (W >= 8) v += from_lane<0x141>(v);
  if constexpr (W >= 16) v += from_lane<0x140>(v);
  if constexpr (W >= kWave) v = (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
  if constexpr (W > kWave) {
    constexpr int kWaves = W / kWave;
    const int first = threadIdx.x / W * kWaves;
    if (threadIdx.x % kWave == 0) lds.wide[turn][threadIdx.x / kWave] = v;
    __syncthreads();
    v = lds.wide[turn][first];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += lds.wide[turn][first + w];
    turn ^= 1;
  }
  return v;
}

// v normalised in place, before gain and bias; returns what it was multiplied by.
//
// A mean in float32 is off by roundings of its own size, which is far more than the deviations in a row that is near a constant (one of 1000 came
// out at 0.06, with eps 1e-6).  So it is summed in float64 and taken away in two parts: the deviations keep float32's accuracy for their own size.  (bfloat16, centred on both sides: 30,000 x 768 44 us where float32 sums
// took 40, its gradient 102 and 95; 16384 x 4096 104 and 96.  Correcting a float32 mean by the sum of the deviations, with a third sum where
// that cancels: 47, 107 and 102.)
template <class L, int W>
__device__ __forceinline__ float normalise(const L& row, int kind, float eps, float (&v)[L::E], RowLds<W, L::R>& lds, int& turn) {
  if (kind == ILARGI_NORM_NONE) return 1.0f;
  constexpr int E = L::E;
  const float share = 1.0f / (float)row.m;
  if (kind == ILARGI_NORM_CENTRED) {
    double even = 0.0, odd = 0.0;
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      even += (double)v[e];
      odd += (double)v[e + 1];
    }
    const double mean = row_sum<W, L::R>(even + odd, lds, turn) * (1.0 / (double)row.m);
    const float most = (float)mean, rest = (float)(mean - (double)most);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = row.own(v[e] - most - rest, e);
  }
  float s[1];
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

// Keeps the compiler from holding a vector's values in 32 bits, in twice the registers, from row to row.
template <class Raw, int P>
__device__ __forceinline__ void as_they_are(Raw (&r)[P]) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    uint4 w = __builtin_bit_cast(uint4, r[p]);
    asm volatile("" : "+v"(w.x), "+v"(w.y), "+v"(w.z), "+v"(w.w));
    r[p] = __builtin_bit_cast(Raw, w);
  }
}

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
  for (int e = 0; e < L::E; ++e) v[e] += (float)bias[e / L::V].v[e % L::V];
}

struct NormOut {
  void *r, *y;
  int64_t ld_r, ld_y;
};

template <class T, int W, int P, int SHAPE>
__global__ __launch_bounds__(W < 256 ? 256 : W) void norm_kernel(ilargi_norm_t a, NormOut o, bool past) {
  using L = Row<T, W, P, SHAPE>;
  constexpr int E = L::E, R = L::R, S = sizeof(T);
  __shared__ __attribute__((aligned(16))) RowLds<W, R> lds;
  L row;
  row.plan(a.m);
  int turn = 0;
  typename L::Raw g1[P], b1[P], gr[P], g2[P], b2[P];
  row.load_vector(a.gain1, g1);
  row.load_vector(a.bias1, b1);
  if (!a.gate_rows) row.load_vector(a.gate, gr);
  row.load_vector(a.gain2, g2);
  row.load_vector(a.bias2, b2);
  for (int64_t i0 = (int64_t)blockIdx.x * R; i0 < a.n; i0 += (int64_t)gridDim.x * R) {
    const int64_t mine = i0 + L::slot(), i = mine < a.n ? mine : a.n - 1;
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
    if (o.r != nullptr && mine < a.n) row.store((char*)o.r + i * o.ld_r * S, v, past);
    if (a.second == ILARGI_NORM_NONE || o.y == nullptr) continue;
    normalise<L, W>(row, a.second, a.eps, v, lds, turn);
    times_gain(row, a.gain2, g2, v);
    plus_bias(row, a.bias2, b2, v);
    if (mine < a.n) row.store((char*)o.y + i * o.ld_y * S, v, past);
  }
}

// t becomes the gradient of what was normalised to `unit` by the factor `by`.
template <class L, int W>
__device__ __forceinline__ void normalise_back(const L& row, int kind, float by, const float (&unit)[L::E], float (&t)[L::E], RowLds<W, L::R>& lds, int& turn) {
  if (kind == ILARGI_NORM_NONE) return;
  constexpr int E = L::E;
  const float share = 1.0f / (float)row.m;
  if (kind == ILARGI_NORM_CENTRED) {
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      s[0] = fmaf(t[e], unit[e], s[0]);
      s[1] += t[e];
    }
    row_sums<W, L::R>(s, lds, turn);
    const float along = s[0] * share, mean = s[1] * share;
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = by * row.own(fmaf(-along, unit[e], t[e]) - mean, e);
  } else {
    float s[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < E; ++e) s[0] = fmaf(t[e], unit[e], s[0]);
    row_sums<W, L::R>(s, lds, turn);
    const float along = s[0] * share;
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = by * fmaf(-along, unit[e], t[e]);
  }
}

// f(z) in place of z, and f'(z): one exponential for both.
template <int N>
__device__ __forceinline__ void act_both(float (&z)[N], float (&slope)[N], int act) {
  switch (act) {
    case ILARGI_ACT_SIGMOID:
    case ILARGI_ACT_SILU:
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float e = exp_minus(z[j]), q = __builtin_amdgcn_rcpf(1.0f + e), far = e * q;        // sigmoid(|z|), sigmoid(-|z|)
        const float p = z[j] >= 0.0f ? q : far, both = far * q;
        if (act == ILARGI_ACT_SIGMOID) {
          slope[j] = both;
          z[j] = p;
        } else {                                         // (beyond 200 both factors are 0 or 1 already: no infinity meets a 0)
          slope[j] = fmaf(fminf(fmaxf(z[j], -200.0f), 200.0f), both, p);
          z[j] = fmaxf(z[j], -200.0f) * p;
        }
      }
      break;
    case ILARGI_ACT_NONE:
#pragma unroll
      for (int j = 0; j < N; ++j) slope[j] = 1.0f;
      break;
    default:
#pragma unroll
      for (int j = 0; j < N; ++j) {
        slope[j] = act_slope(z[j], act);
        z[j] = act_value(z[j], act);
      }
  }
}

struct NormGradIn {
  const void *d_r, *d_y;
  int64_t ld_dr, ld_dy;
};
constexpr int kGradWaves = 2;        // of a SIMD, at least: with 128 registers (four) a thread's values did not fit, 173 us for 132 at 8192 x 4096
enum { kSumGate, kSumGain1, kSumGain2, kSumBias1, kSumBias2, kSums };
// Whether all five sums of such rows are held in LDS (those of more than 8192 columns do not fit), and the bytes of it.
template <class L>
constexpr bool kSumsInLds = (L::kW == 512 && L::E == 16) || (L::V == 8 && L::NT == 256);
template <class L>
constexpr size_t kSumsLds = kSumsInLds<L> ? sizeof(float) * (kSums - 1) * L::E * L::NT : 0;

// Sums over a workgroup's rows, of the columns that a thread holds: in registers, or where all five of many columns are wanted all but the
// gate's in LDS, each thread's in places of its own: of 16 columns a thread (80 registers of 256; 3600 x 8192, bfloat16, centred: 284 us in
// registers that spill, 111 so), and of eight in workgroups of 256, three of which then fit a compute unit (centred on both sides, a gate row: 18,976 x
// 1544 164 and 132, 30,000 x 768 134 and 103).
template <class L, int HELD, bool IN_LDS>
struct RowSums {
  static constexpr int E = L::E;
  float held[IN_LDS ? 1 : HELD][E];
  float4* mine;              // [sum][four columns][thread]
  __device__ __forceinline__ explicit RowSums(float4* lds) : mine(lds + threadIdx.x) {
#pragma unroll
    for (int q = 0; q < (IN_LDS ? 1 : HELD); ++q)
#pragma unroll
      for (int e = 0; e < E; ++e) held[q][e] = 0.0f;
    if constexpr (IN_LDS)
#pragma unroll
      for (int q = 0; q < (HELD - 1) * E / 4; ++q) mine[q * L::NT] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  static __device__ __forceinline__ constexpr bool registers(int q) { return !IN_LDS || q == 0; }
  __device__ __forceinline__ float4& place(int q, int e) const { return mine[((q - 1) * (E / 4) + e / 4) * L::NT]; }
  // a o b, or a
  template <int Q>
  __device__ __forceinline__ void add(const float (&a)[E], const float (&b)[E]) {
    if constexpr (registers(Q)) {
#pragma unroll
      for (int e = 0; e < E; ++e) held[Q][e] = fmaf(a[e], b[e], held[Q][e]);
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        float4& p = place(Q, e);
        const float4 v = p;
        p = make_float4(fmaf(a[e], b[e], v.x), fmaf(a[e + 1], b[e + 1], v.y), fmaf(a[e + 2], b[e + 2], v.z), fmaf(a[e + 3], b[e + 3], v.w));
      }
    }
  }
  template <int Q>
  __device__ __forceinline__ void add(const float (&a)[E]) {
    if constexpr (registers(Q)) {
#pragma unroll
      for (int e = 0; e < E; ++e) held[Q][e] += a[e];
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        float4& p = place(Q, e);
        const float4 v = p;
        p = make_float4(a[e] + v.x, a[e + 1] + v.y, a[e + 2] + v.z, a[e + 3] + v.w);
      }
    }
  }
  template <int Q>
  __device__ __forceinline__ void take(float (&f)[E]) const {
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      if constexpr (registers(Q)) {
#pragma unroll
        for (int u = 0; u < 4; ++u) f[e + u] = held[Q][e + u];
      } else {
        const float4 v = place(Q, e);
        f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w;
      }
    }
  }
};

// The sums over this workgroup's rows go to partial[workgroup][sum][column].  FEW: there is no bias1, and those
// of the gains alone are wanted.  A row's data are
// asked for as soon as those of the row before have been taken out of their registers
// (8192 columns of bfloat16, two pieces a thread, means in float32: 106 us for 3600 rows; asked for when the row begins, 148).
template <class T, int W, int P, int SHAPE, bool FEW>
__global__ __launch_bounds__(W < 256 ? 256 : W, kGradWaves) void norm_grad_kernel(ilargi_norm_t a, NormGradIn d, ilargi_norm_grads_t o, float* __restrict__ partial, bool past) {
  using L = Row<T, W, P, SHAPE>;
  constexpr int E = L::E, R = L::R, V = L::V, S = sizeof(T), kHeld = FEW ? 3 : kSums;
  __shared__ __attribute__((aligned(16))) RowLds<W, R> lds;
  __shared__ float rows_sums[R > 1 ? R : 1][R > 1 ? W * E : 1];
  L row;
  row.plan(a.m);
  int turn = 0;
  const bool second = a.second != ILARGI_NORM_NONE && d.d_y != nullptr, with_x = second && a.x != nullptr, gate_sum = o.d_gate != nullptr && !a.gate_rows;
  typename L::Raw g1[P], b1[P], gr[P], g2[P], h[P], x[P], dr[P], dy[P];
  const int64_t first = (int64_t)blockIdx.x * R + L::slot(), step = (int64_t)gridDim.x * R;
  auto at = [&](int64_t i) { return i < a.n ? i : a.n - 1; };
  auto load_row = [&](int64_t i) {
    row.load(row_at(a.h, i, a.ld_h, S), h);
    if (a.gate_rows) row.load(row_at(a.gate, i, a.ld_gate, S), gr);
    if (with_x) row.load(row_at(a.x, i, a.ld_x, S), x);
    if (second) row.load(row_at(d.d_y, i, d.ld_dy, S), dy);
    if (d.d_r != nullptr) row.load(row_at(d.d_r, i, d.ld_dr, S), dr);
  };
  load_row(at(first));
  row.load_vector(a.gain1, g1);
  if constexpr (!FEW) row.load_vector(a.bias1, b1);
  if (!a.gate_rows) row.load_vector(a.gate, gr);
  row.load_vector(a.gain2, g2);
  extern __shared__ __attribute__((aligned(16))) float4 sums_lds[];
  RowSums<L, kHeld, !FEW && kSumsInLds<L>> sums(sums_lds);
  for (int64_t i0 = (int64_t)blockIdx.x * R; i0 < a.n; i0 += step) {
    const int64_t mine = i0 + L::slot(), i = at(mine), next = at(mine + step);
    const bool is = mine < a.n;
    if constexpr (V == 8) {
      as_they_are(g1);
      if constexpr (!FEW) as_they_are(b1);
      as_they_are(gr);
      as_they_are(g2);
    }
    float unit[E];                                       // h normalised
    row.values(h, unit);
    row.load(row_at(a.h, next, a.ld_h, S), h);
    const float by1 = normalise<L, W>(row, a.first, a.eps, unit, lds, turn);
    float f[E], slope[E];
    if (a.gate != nullptr) {
      row.values(gr, f);
      if (a.gate_rows) row.load(row_at(a.gate, next, a.ld_gate, S), gr);
      act_both(f, slope, a.gate_act);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = 1.0f;
    }
    float t[E];                                          // the gradient on its way back: of r first
    if (second) {
      float r[E], back[E];
#pragma unroll
      for (int e = 0; e < E; ++e) r[e] = unit[e];
      times_gain(row, a.gain1, g1, r);
      if constexpr (!FEW) plus_bias(row, a.bias1, b1, r);
      if (with_x) {
        row.values(x, back);
        row.load(row_at(a.x, next, a.ld_x, S), x);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) r[e] = with_x ? fmaf(a.scale, f[e] * r[e], back[e]) : a.scale * (f[e] * r[e]);
      const float by2 = normalise<L, W>(row, a.second, a.eps, r, lds, turn);
      row.values(dy, back);
      row.load(row_at(d.d_y, next, d.ld_dy, S), dy);
      if (is) {
        sums.template add<kSumGain2>(back, r);
        if constexpr (!FEW) sums.template add<kSumBias2>(back);
      }
      times_gain(row, a.gain2, g2, back);
      normalise_back<L, W>(row, a.second, by2, r, back, lds, turn);
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] = back[e];
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] = 0.0f;
    }
    if (d.d_r != nullptr) {
      float v[E];
      row.values(dr, v);
      row.load(row_at(d.d_r, next, d.ld_dr, S), dr);
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] += v[e];
    }
    if (o.d_x != nullptr && is) row.store((char*)o.d_x + i * o.ld_x * S, t, past);
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] *= a.scale;
    if (o.d_gate != nullptr) {
      float u[E];
#pragma unroll
      for (int e = 0; e < E; ++e) u[e] = unit[e];
      times_gain(row, a.gain1, g1, u);
      if constexpr (!FEW) plus_bias(row, a.bias1, b1, u);
#pragma unroll
      for (int e = 0; e < E; ++e) u[e] *= slope[e] * t[e];
      if (!is) {
      } else if (a.gate_rows) {
        row.store((char*)o.d_gate + i * o.ld_gate * S, u, past);
      } else if constexpr (!FEW) {
        sums.template add<kSumGate>(u);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] *= f[e];
    if (is) {
      sums.template add<kSumGain1>(t, unit);
      if constexpr (!FEW) sums.template add<kSumBias1>(t);
    }
    if (o.d_h == nullptr) continue;
    times_gain(row, a.gain1, g1, t);
    normalise_back<L, W>(row, a.first, by1, unit, t, lds, turn);
    if (is) row.store((char*)o.d_h + i * o.ld_h * S, t, past);
  }
  if (partial == nullptr) return;
  float* const to = partial + (int64_t)blockIdx.x * kSums * a.m;
  auto leave = [&](auto which, const void* wanted) {
    constexpr int Q = decltype(which)::value;
    if (wanted == nullptr) return;
    float f[E];
    sums.template take<Q>(f);
    if constexpr (R == 1) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (row.live(e / V, e % V)) to[(int64_t)Q * a.m + row.c[e / V] + e % V] = f[e];
    } else {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (row.live(e / V, e % V)) rows_sums[threadIdx.x / W][row.c[e / V] + e % V] = f[e];
      __syncthreads();
      for (int j = threadIdx.x; j < a.m; j += L::NT) {
        float s = rows_sums[0][j];
#pragma unroll
        for (int r = 1; r < R; ++r) s += rows_sums[r][j];
        to[(int64_t)Q * a.m + j] = s;
      }
    }
  };
  leave(std::integral_constant<int, kSumGain1>(), o.d_gain1);
  leave(std::integral_constant<int, kSumGain2>(), o.d_gain2);
  if constexpr (!FEW) {
    leave(std::integral_constant<int, kSumGate>(), gate_sum ? o.d_gate : nullptr);
    leave(std::integral_constant<int, kSumBias1>(), o.d_bias1);
    leave(std::integral_constant<int, kSumBias2>(), o.d_bias2);
  }
}

// Adds the workgroups' sums, in float64: they cancel each other as the rows' parts do.  Sixteen threads share a column, each adds every
// sixteenth workgroup, then they are added in order.
template <class T>
__global__ __launch_bounds__(256) void norm_join_kernel(const float* __restrict__ partial, int groups, int64_t m, ilargi_norm_grads_t o, int gate_sum, int accumulate) {
  __shared__ double part[16][17];
  const int c = threadIdx.x % 16, q = threadIdx.x / 16, which = blockIdx.y;
  T* const out = (T*)(which == kSumGain1 ? o.d_gain1 : which == kSumGain2 ? o.d_gain2 : which == kSumGate ? (gate_sum ? o.d_gate : nullptr) : which == kSumBias1 ? o.d_bias1 : o.d_bias2);
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

// f(row): threads of a row and pieces of a thread, the least that hold it.  WIDE: 512 threads, which have twice the registers of 1024, for
// rows of up to 32 KB too.  (Gradients with 512 threads and with 1024.  bfloat16, 3600 x 8192: rms on both sides and gates 92 and 157 us, centred on both
// sides with all five sums 113 and 464.  float32, the same two: 126 and 159, 122 and 267 at 1800 x 8192; 158 and 188, 257 and 329 at 2115 x 5441.)
template <class T, bool WIDE, class F>
hipError_t by_columns(int64_t m, F f) {
  constexpr int V = ElemOf<T>::kVec;
  const int64_t pieces = (m + V - 1) / V;
  auto with = [&](auto w, auto p) {
    constexpr int W = decltype(w)::value, P = decltype(p)::value;
    if constexpr (W == 4)
      if (m < V) return f(Row<T, W, P, kShort>());
    return m % V != 0 ? f(Row<T, W, P, kRagged>()) : m == W * P * V ? f(Row<T, W, P, kFull>()) : f(Row<T, W, P, kWhole>());
  };
  using std::integral_constant;
  constexpr integral_constant<int, 1> one;
  if (pieces <= 4) return with(integral_constant<int, 4>(), one);
  if (pieces <= 8) return with(integral_constant<int, 8>(), one);
  if (pieces <= 16) return with(integral_constant<int, 16>(), one);
  if (pieces <= 64) return with(integral_constant<int, 64>(), one);
  if (pieces <= 128) return with(integral_constant<int, 128>(), one);
  if (pieces <= 256) return with(integral_constant<int, 256>(), one);
  if (pieces <= 512) return with(integral_constant<int, 512>(), one);
  if constexpr (WIDE && V == 8) {
    if (pieces <= 1024) return with(integral_constant<int, 512>(), integral_constant<int, 2>());
  } else {
    if (pieces <= 1024) return with(integral_constant<int, 1024>(), one);
  }
  if constexpr (WIDE && V == 4) {
    if (pieces <= 2048) return with(integral_constant<int, 512>(), integral_constant<int, 4>());
  } else {
    if (pieces <= 2048) return with(integral_constant<int, 1024>(), integral_constant<int, 2>());
  }
  if constexpr (V == 4)
    if (pieces <= 4096) return with(integral_constant<int, 1024>(), integral_constant<int, 4>());
  return hipErrorInvalidValue;
}

int64_t groups_of(int64_t n, int rows, int64_t most) {
  const int64_t g = (n + rows - 1) / rows;
  return g < most ? g : most;
}

// Workgroups of the gradient: as many as are on the card at once, three of 256 threads or one larger on a compute unit, as each leaves its
// sums behind.  (8192 x 4096, bfloat16: 256 of them 125 us, 512 129, 1024 140; 100,000 x 220: 768 109, 1024 113, 2048 118.)
template <class T>
int64_t grad_groups(int64_t n, int64_t m) {
  int64_t g = 0;
  const hipError_t e = by_columns<T, false>(m, [&](auto row) {
    using L = decltype(row);
    g = groups_of(n, L::R, L::NT == 256 ? 768 : 256);
    return hipSuccess;
  });
  return e == hipSuccess ? g : 0;
}

template <class T>
hipError_t norm_typed(const ilargi_norm_t& a, const NormOut& o, hipStream_t st) {
  const bool past = (int64_t)sizeof(T) * a.n * a.m * ((o.r != nullptr) + (o.y != nullptr)) >= kStreamBytes;
  return by_columns<T, false>(a.m, [&](auto row) {
    using L = decltype(row);
    norm_kernel<T, L::kW, L::kP, L::kShape><<<(unsigned)groups_of(a.n, L::R, 256 * (2048 / L::NT)), L::NT, 0, st>>>(a, o, past);
    return hipGetLastError();
  });
}

template <class T>
hipError_t norm_grad_typed(const ilargi_norm_t& a, const NormGradIn& d, const ilargi_norm_grads_t& o, int accumulate, float* partial, hipStream_t st) {
  const bool gate_sum = o.d_gate != nullptr && !a.gate_rows;
  const bool sums = gate_sum || o.d_gain1 != nullptr || o.d_bias1 != nullptr || o.d_gain2 != nullptr || o.d_bias2 != nullptr;
  const bool past = (int64_t)sizeof(T) * a.n * a.m * ((o.d_h != nullptr) + (o.d_x != nullptr) + (o.d_gate != nullptr && a.gate_rows)) >= kStreamBytes;
  const bool few = !gate_sum && a.bias1 == nullptr && o.d_bias1 == nullptr && o.d_bias2 == nullptr;
  if (!sums) partial = nullptr;
  const int64_t groups = grad_groups<T>(a.n, a.m);
  if (groups > 0) {
    auto launch = [&](auto row, auto which) {
      using L = decltype(row);
      constexpr bool FEW = decltype(which)::value;
      const auto kernel = norm_grad_kernel<T, L::kW, L::kP, L::kShape, FEW>;
      const size_t bytes = FEW ? 0 : kSumsLds<L>;
      if (bytes > 0)
        if (hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); e != hipSuccess) return e;
      kernel<<<(unsigned)groups, L::NT, bytes, st>>>(a, d, o, partial, past);
      return hipGetLastError();
    };
    const hipError_t e = few ? by_columns<T, true>(a.m, [&](auto row) { return launch(row, std::true_type()); })
                             : by_columns<T, true>(a.m, [&](auto row) { return launch(row, std::false_type()); });
    if (e != hipSuccess) return e;
  }
  if (sums) norm_join_kernel<T><<<dim3((unsigned)((a.m + 15) / 16), few ? 3 : kSums), 256, 0, st>>>(partial, (int)groups, a.m, o, gate_sum, accumulate);
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
