// The norm over many tensors and the tensors scaled by it: every workgroup leaves the sum of the squares of its part, in float64; the
// workgroups of the second pass add those sums up themselves, all in the same order, and where they are many a workgroup does it for all.
//
// Tensors go sixty-four to a launch, in the launch's arguments (sixteen, where there are no more: 4 KB of arguments cost the host 2 us a
// launch): nothing is copied to the device before.  A workgroup takes a run of one
// tensor's pieces of 16 bytes; a tensor whose rows follow each other counts as one row.  The second pass goes through the parts from
// the last to the first, whose data the caches still hold.  Bound by memory: 60 tensors of 630 MB 113 us for the squares (5.6 TB/s), 5 for their
// sum, 225 for the scaled copies (5.6 TB/s read and written); in one round of 2055 parts, 7 of them in a second, the squares took 176.
#include "ilargi_layers.h"

namespace ilargi {

namespace {

constexpr int kMostTensors = 64, kFewTensors = 16, kMostSums = 1024, kLoads = 4;
// Pieces of a part: at least what a workgroup asks for at once (12 tensors, 250 KB: 9.6 us, 11.8 with twice and 11.5 with half of it).
constexpr int64_t kLeastPart = 256 * kLoads, kMostPart = 8192;

struct Part {
  const char* in;
  char* out;
  int64_t row_pieces, pieces;       // of a row, of all
  int64_t cols, ld_in, ld_out;
};
template <int MOST>
struct Parts {
  Part t[MOST];
  int first[MOST + 1];      // its first workgroup
  int count;
  uint64_t bf16;                    // a bit a tensor
  int64_t part;                     // pieces of a workgroup
};

// The tensor of a workgroup.
template <int MOST>
__device__ __forceinline__ int tensor_of(const Parts<MOST>& a, int group) {
  const int lane = threadIdx.x % kWave;
  const bool before = lane < a.count && a.first[lane < MOST ? lane : 0] <= group;
  return __popcll(__ballot(before)) - 1;
}

// use(piece, valid elements, offset in `out`) for the pieces of this workgroup's part; kLoads of them are asked for together.
template <class T, class Use>
__device__ __forceinline__ void pieces_of(const Part& t, int64_t first, int64_t last, Use use) {
  constexpr int V = ElemOf<T>::kVec;
  for (int64_t at = first + threadIdx.x; at < last; at += 256 * kLoads) {
    int64_t in[kLoads], out[kLoads];
    int valid[kLoads];
    Piece<T, V> v[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int64_t p = at + 256 * u;
      int64_t row = 0, c = p;
      if (t.row_pieces != t.pieces) {
        row = t.pieces < (1ll << 31) ? (int64_t)((uint32_t)p / (uint32_t)t.row_pieces) : p / t.row_pieces;
        c = p - row * t.row_pieces;
      }
      const int64_t left = t.cols - c * V;
      valid[u] = p >= last ? 0 : left < V ? (int)left : V;
      in[u] = row * t.ld_in + c * V;
      out[u] = row * t.ld_out + c * V;
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      if (valid[u] == V) {
        v[u] = *reinterpret_cast<const Piece<T, V>*>((const T*)t.in + in[u]);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[u].v[j] = j < valid[u] ? ((const T*)t.in)[in[u] + j] : (T)0.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) use(v[u], valid[u], out[u]);
  }
}

__device__ __forceinline__ double workgroup_sum(double s, double (&lds)[4]) {
#pragma unroll
  for (int q = kWave / 2; q >= 1; q /= 2) s += __shfl_xor(s, q);
  if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = s;
  __syncthreads();
  return lds[0] + lds[1] + lds[2] + lds[3];
}

template <int MOST>
__global__ __launch_bounds__(256) void squares_kernel(Parts<MOST> a, double* __restrict__ partial) {
  __shared__ double lds[4];
  const int q = tensor_of(a, blockIdx.x);
  const Part& t = a.t[q];
  const int64_t first = (int64_t)(blockIdx.x - a.first[q]) * a.part, last = first + a.part < t.pieces ? first + a.part : t.pieces;
  double s = 0.0;
  auto add = [&](auto piece) {
#pragma unroll
    for (auto x : piece.v) s = fma((double)(float)x, (double)(float)x, s);
  };
  if (a.bf16 >> q & 1) pieces_of<bf16_t>(t, first, last, [&](const Piece<bf16_t, 8>& v, int, int64_t) { add(v); });
  else pieces_of<float>(t, first, last, [&](const Piece<float, 4>& v, int, int64_t) { add(v); });
  s = workgroup_sum(s, lds);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ double add_sums(const double* __restrict__ partial, int sums, double (&lds)[4]) {
  double s = 0.0;
#pragma unroll 8
  for (int w = threadIdx.x; w < sums; w += 256) s += partial[w];
  return workgroup_sum(s, lds);
}

__global__ __launch_bounds__(256) void add_sums_kernel(const double* __restrict__ partial, int sums, double* __restrict__ to) {
  __shared__ double lds[4];
  const double s = add_sums(partial, sums, lds);
  if (threadIdx.x == 0) *to = s;
}

// blockIdx: the part of a tensor, each tensor's from its last on; without tensors one workgroup that stores the norm.  `past`: what is written is larger
// than the caches.
template <int MOST>
__global__ __launch_bounds__(256) void clip_kernel(Parts<MOST> a, const double* __restrict__ partial, int sums, float max_norm, float* __restrict__ norm, bool past) {
  __shared__ double lds[4];
  const double total = sqrt(add_sums(partial, sums, lds));
  if (norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
  if (a.count == 0) return;
  const bool scaled = total > (double)max_norm && total <= 1.7976931348623157e308;      // (no for NaN and infinity)
  const Factor2 factor = factor2(scaled ? (double)max_norm / total : 1.0);      // (a factor below 2^-126 keeps its bits)
  const int q = tensor_of(a, blockIdx.x);
  const Part& t = a.t[q];
  if (!scaled && t.in == t.out) return;
  const int64_t first = (int64_t)(a.first[q + 1] - 1 - (int)blockIdx.x) * a.part, last = first + a.part < t.pieces ? first + a.part : t.pieces;
  auto put = [&](auto v, int valid, int64_t at) {
    using P = decltype(v);
    using T = std::remove_reference_t<decltype(v.v[0])>;
    constexpr int V = sizeof(P) / sizeof(T);
    if (scaled) {
#pragma unroll
      for (int j = 0; j < V; ++j) v.v[j] = (T)times((float)v.v[j], factor);
    }
    T* const to = (T*)t.out + at;
    if (valid == V && past) {
      typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
      __builtin_nontemporal_store(__builtin_bit_cast(words, v), reinterpret_cast<words*>(to));
    } else if (valid == V) {
      *reinterpret_cast<P*>(to) = v;
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < valid) to[j] = v.v[j];
    }
  };
  if (a.bf16 >> q & 1) pieces_of<bf16_t>(t, first, last, put);
  else pieces_of<float>(t, first, last, put);
}

int64_t vec_of(const ilargi_tensor_t& t) { return t.type == ILARGI_TYPE_BF16 ? ElemOf<bf16_t>::kVec : ElemOf<float>::kVec; }
// How a pass cuts a tensor into pieces and parts.  The first goes by the inputs alone (WRITTEN false): what is written, and where to, does not
// change the order of its sums.
template <bool WRITTEN>
bool in_one_row(const ilargi_tensor_t& t) { return t.rows <= 1 || (t.ld_in == t.cols && (!WRITTEN || t.ld_out == t.cols)); }
template <bool WRITTEN>
int64_t row_pieces(const ilargi_tensor_t& t) { return ((in_one_row<WRITTEN>(t) ? t.rows * t.cols : t.cols) + vec_of(t) - 1) / vec_of(t); }
template <bool WRITTEN>
int64_t pieces_in(const ilargi_tensor_t& t) {
  return t.rows == 0 || t.cols == 0 || (WRITTEN && t.out == nullptr) ? 0 : row_pieces<WRITTEN>(t) * (in_one_row<WRITTEN>(t) ? 1 : t.rows);
}

struct ClipPlan {
  int64_t part, groups;      // pieces of a workgroup, workgroups
};
template <bool WRITTEN>
ClipPlan clip_plan(const ilargi_tensor_t* t, int64_t count) {
  int64_t all = 0;
  for (int64_t q = 0; q < count; ++q) all += pieces_in<WRITTEN>(t[q]);
  ClipPlan p{all / kMostSums, 0};
  p.part = p.part < kLeastPart ? kLeastPart : p.part > kMostPart ? kMostPart : (p.part + 255) / 256 * 256;
  for (int64_t q = 0; q < count; ++q) p.groups += (pieces_in<WRITTEN>(t[q]) + p.part - 1) / p.part;
  return p;
}

}  // namespace

size_t clip_bytes(const ilargi_tensor_t* t, int64_t count) { return (size_t)(clip_plan<false>(t, count).groups + 1) * 8; }

namespace {

template <int MOST>
hipError_t clip_in(const ilargi_tensor_t* t, int64_t count, float max_norm, float* norm, double* partial, hipStream_t st) {
  const ClipPlan read = clip_plan<false>(t, count), write = clip_plan<true>(t, count);
  if (read.groups > 2147483647ll || write.groups > 2147483647ll) return hipErrorInvalidValue;
  int64_t written = 0;
  for (int64_t q = 0; q < count; ++q)
    if (t[q].out != t[q].in) written += pieces_in<true>(t[q]) * 16;
  const bool past = written >= kStreamBytes;
  auto next = [&](int64_t& q, int step, auto which) {                  // tensors from q on, until a launch is full
    constexpr bool WRITTEN = decltype(which)::value;
    const int64_t part = WRITTEN ? write.part : read.part;
    Parts<MOST> a{};
    a.part = part;
    for (; q >= 0 && q < count && a.count < MOST; q += step) {
      const int64_t pieces = pieces_in<WRITTEN>(t[q]);
      if (pieces == 0) continue;
      const bool one = in_one_row<WRITTEN>(t[q]);
      a.t[a.count] = {(const char*)t[q].in, (char*)t[q].out, row_pieces<WRITTEN>(t[q]), pieces, one ? t[q].rows * t[q].cols : t[q].cols, t[q].ld_in, t[q].ld_out};
      a.bf16 |= (uint64_t)(t[q].type == ILARGI_TYPE_BF16) << a.count;
      a.first[a.count + 1] = a.first[a.count] + (int)((pieces + part - 1) / part);
      ++a.count;
    }
    return a;
  };
  int64_t done = 0;
  for (int64_t q = 0; q < count;) {
    const Parts<MOST> a = next(q, 1, std::false_type());
    if (a.count == 0) break;
    squares_kernel<<<(unsigned)a.first[a.count], 256, 0, st>>>(a, partial + done);
    done += a.first[a.count];
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  int sums = (int)read.groups;
  const double* from = partial;
  if (sums > kMostSums) {
    add_sums_kernel<<<1, 256, 0, st>>>(partial, sums, partial + sums);
    from = partial + sums;
    sums = 1;
  }
  bool stored = norm == nullptr;
  for (int64_t q = count - 1; q >= 0;) {
    const Parts<MOST> a = next(q, -1, std::true_type());
    if (a.count == 0) break;
    clip_kernel<<<(unsigned)a.first[a.count], 256, 0, st>>>(a, from, sums, max_norm, stored ? nullptr : norm, past);
    stored = true;
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (!stored) clip_kernel<<<1, 256, 0, st>>>(Parts<MOST>{}, from, sums, max_norm, norm, false);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_clip(const ilargi_tensor_t* t, int64_t count, float max_norm, float* norm, double* partial, hipStream_t st) {
  return count <= kFewTensors ? clip_in<kFewTensors>(t, count, max_norm, norm, partial, st) : clip_in<kMostTensors>(t, count, max_norm, norm, partial, st);
}

}  // namespace ilargi
