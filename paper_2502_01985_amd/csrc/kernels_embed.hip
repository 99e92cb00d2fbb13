// Rows of a learned table picked by keys, and the gradient of that table: rows of the output's gradient summed by key.
#include "ilargi_layers.h"

namespace ilargi {

namespace {

// A group of 2^sh lanes shares a row; every lane takes 16-byte pieces of it.
template <class TI, class TO, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_kernel(EmbedArgs a, int sh) {
  constexpr int V = ElemOf<TI>::kVec < ElemOf<TO>::kVec ? ElemOf<TI>::kVec : ElemOf<TO>::kVec;
  const int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh;
  if (i >= a.n) return;
  const int lane = threadIdx.x & ((1 << sh) - 1);
  const int64_t id = a.ids[i];
  const bool live = id >= 0 && id < a.rows;
  if (ADD && !live) return;
  const TI* src = (const TI*)a.table + (live ? id : 0) * a.ld_table;
  TO* dst = (TO*)a.out + i * a.ld_out;
  for (int64_t c = (int64_t)lane * V; c < a.cols; c += (int64_t)V << sh) {
    const int valid = (int)(a.cols - c < V ? a.cols - c : V);
    float f[V];
    if (live) load_piece<TI, V>(src + c, valid, f);
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = live ? f[j] * a.scale : 0.0f;
    if constexpr (ADD) {
      float o[V];
      load_piece<TO, V>(dst + c, valid, o);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] += o[j];
    }
    store_piece<TO, V>(dst + c, valid, f);
  }
}

template <class TI, class TO>
hipError_t embed_typed(const EmbedArgs& a, hipStream_t st) {
  constexpr int V = ElemOf<TI>::kVec < ElemOf<TO>::kVec ? ElemOf<TI>::kVec : ElemOf<TO>::kVec;
  int sh = ilog2_ceil((a.cols + V - 1) / V);
  if (sh > 6) sh = 6;
  const int64_t blocks = ((a.n << sh) + kBlock - 1) / kBlock;
  if (a.accumulate) embed_kernel<TI, TO, true><<<(unsigned)blocks, kBlock, 0, st>>>(a, sh);
  else embed_kernel<TI, TO, false><<<(unsigned)blocks, kBlock, 0, st>>>(a, sh);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  if (a.table_bf16) return a.out_bf16 ? embed_typed<bf16_t, bf16_t>(a, st) : embed_typed<bf16_t, float>(a, st);
  return a.out_bf16 ? embed_typed<float, bf16_t>(a, st) : embed_typed<float, float>(a, st);
}

// ------------------------------------------------------------------------------------------------------- gradient
//
// The ids are sorted stably (radix, least digit first), with those that name no row behind all others.  Then groups of lanes
// walk runs of equal length of the sorted ids and sum the rows of d_out that they stand for: a row of the table whose ids all lie
// in one run is written there, and the sums of the others are carried to a second pass.  So one row that holds a large part of the
// ids is spread over as many groups as it has runs, and every sum has a fixed order.
namespace {

constexpr int kBits = 9, kBins = 1 << kBits;      // two passes for tables of up to 262,143 rows
constexpr int kChunk = 4096;                      // ids a workgroup sorts by one digit
constexpr int kOneSort = 16384;                   // ids that one workgroup sorts in LDS by itself

__device__ __forceinline__ uint32_t id_key(int32_t id, uint32_t rows) { return id >= 0 && (uint32_t)id < rows ? (uint32_t)id : rows; }

// The lanes whose digit equals this lane's, among the live ones.
template <int BITS>
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool live) {
  uint64_t match = __ballot(live);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const uint64_t vote = __ballot(live && ((d >> b) & 1));
    match &= ((d >> b) & 1) ? vote : ~vote;
  }
  return match;
}

template <bool FIRST>
__global__ __launch_bounds__(kBlock) void id_hist_kernel(const int32_t* __restrict__ keys, int64_t n, uint32_t rows, int shift, int chunks,
                                                         int32_t* __restrict__ hist) {
  __shared__ int32_t h[kBins];
  for (int i = threadIdx.x; i < kBins; i += kBlock) h[i] = 0;
  __syncthreads();
  const int64_t at = (int64_t)blockIdx.x * kChunk + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kChunk / kBlock; ++u) {
    const int64_t i = at + u * kBlock;
    if (i < n) atomicAdd(&h[((FIRST ? id_key(keys[i], rows) : (uint32_t)keys[i]) >> shift) & (kBins - 1)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kBlock) hist[(int64_t)i * chunks + blockIdx.x] = h[i];
}

// Exclusive sums over the chunks of one digit, and the digit's total.
__global__ __launch_bounds__(kBlock) void id_scan_kernel(int32_t* __restrict__ hist, int chunks, int32_t* __restrict__ totals) {
  __shared__ int32_t wsum[kBlock / kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int32_t* row = hist + (int64_t)blockIdx.x * chunks;
  int32_t carry = 0;
  for (int base = 0; base < chunks; base += kBlock) {
    const int i = base + threadIdx.x;
    const int32_t v = i < chunks ? row[i] : 0;
    int32_t inc = v;
    for (int d = 1; d < kWave; d <<= 1) {
      const int32_t t = __shfl_up(inc, d);
      if (lane >= d) inc += t;
    }
    if (lane == kWave - 1) wsum[wave] = inc;
    __syncthreads();
    int32_t before = carry, all = carry;
    for (int w = 0; w < kBlock / kWave; ++w) {
      if (w < wave) before += wsum[w];
      all += wsum[w];
    }
    if (i < chunks) row[i] = before + inc - v;
    carry = all;
    __syncthreads();
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

// Every wavefront walks a quarter of the chunk 64 ids at a time; an id's place is its digit's first place, plus the equal digits of the
// chunks, wavefronts and steps before, plus its rank among those of its step.
template <bool FIRST>
__global__ __launch_bounds__(kBlock) void id_scatter_kernel(const int32_t* __restrict__ keys_in, const int32_t* __restrict__ vals_in, int64_t n, uint32_t rows,
                                                            int shift, int chunks, const int32_t* __restrict__ hist, const int32_t* __restrict__ totals,
                                                            int32_t* __restrict__ keys_out, int32_t* __restrict__ vals_out) {
  constexpr int kWaves = kBlock / kWave, kSteps = kChunk / kBlock;
  static_assert(kBins == 2 * kBlock, "two digits a thread");
  __shared__ int32_t off[kWaves][kBins];
  __shared__ int32_t wsum[kWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) { off[w][threadIdx.x] = 0; off[w][threadIdx.x + kBlock] = 0; }
  const int64_t first = (int64_t)blockIdx.x * kChunk + (int64_t)wave * kSteps * kWave + lane;
  uint32_t k[kSteps];
  int32_t v[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int64_t i = first + u * kWave;
    k[u] = 0; v[u] = 0;
    if (i < n) {
      k[u] = FIRST ? id_key(keys_in[i], rows) : (uint32_t)keys_in[i];
      v[u] = FIRST ? (int32_t)i : vals_in[i];
    }
  }
  // first places of the digits: thread t has 2 t and 2 t + 1
  const int32_t a0 = totals[2 * threadIdx.x], a1 = totals[2 * threadIdx.x + 1];
  int32_t inc = a0 + a1;
  for (int d = 1; d < kWave; d <<= 1) {
    const int32_t t = __shfl_up(inc, d);
    if (lane >= d) inc += t;
  }
  if (lane == kWave - 1) wsum[wave] = inc;
  __syncthreads();
  int32_t start = inc - a0 - a1;
  for (int w = 0; w < wave; ++w) start += wsum[w];
#pragma unroll
  for (int u = 0; u < kSteps; ++u)
    if (first + u * kWave < n) atomicAdd(&off[wave][(k[u] >> shift) & (kBins - 1)], 1);
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int d = 2 * threadIdx.x + h;
    int32_t at = start + (h ? a0 : 0) + hist[(int64_t)d * chunks + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int32_t c = off[w][d];
      off[w][d] = at;
      at += c;
    }
  }
  __syncthreads();
  const uint64_t below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const bool live = first + u * kWave < n;
    const uint32_t d = (k[u] >> shift) & (kBins - 1);
    const uint64_t match = same_digit<kBits>(d, live);
    int32_t dst = 0;
    if (live) dst = off[wave][d] + __popcll(match & below);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");                 // (a wavefront's own offsets: no barrier)
    __builtin_amdgcn_wave_barrier();
    if (live && (match >> lane) <= 1ull) off[wave][d] += __popcll(match);  // the highest lane of its digit
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (live) {
      keys_out[dst] = (int32_t)k[u];
      vals_out[dst] = v[u];
    }
  }
}

// The whole sort of up to kOneSort ids by one workgroup: 16 ids a thread in registers, which change places through LDS after every
// digit of eight bits.  9001 ids of 13 bits: one launch in place of six.
__global__ __launch_bounds__(1024) void id_sort_one_kernel(const int32_t* __restrict__ ids, int n, uint32_t rows, int passes, int32_t* __restrict__ keys_out,
                                                           int32_t* __restrict__ vals_out) {
  constexpr int kSteps = kOneSort / 1024, kD = 256;
  __shared__ uint32_t lk[kOneSort];
  __shared__ uint16_t lv[kOneSort];
  __shared__ int32_t off[16][kD];
  __shared__ int32_t wsum[4];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int steps = (n + 1023) / 1024, first = wave * steps * kWave + lane;        // a wavefront's ids lie together
  uint32_t k[kSteps], v[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int i = first + u * kWave;
    k[u] = u < steps && i < n ? id_key(ids[i], rows) : 0;
    v[u] = (uint32_t)i;
  }
  const uint64_t below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
  for (int p = 0; p < passes; ++p) {
    const int shift = 8 * p;
    for (int i = threadIdx.x; i < 16 * kD; i += 1024) off[i / kD][i % kD] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSteps; ++u)
      if (u < steps && first + u * kWave < n) atomicAdd(&off[wave][(k[u] >> shift) & (kD - 1)], 1);
    __syncthreads();
    int32_t total = 0, inc = 0;
    if (threadIdx.x < kD) {
      for (int w = 0; w < 16; ++w) total += off[w][threadIdx.x];
      inc = total;
      for (int d = 1; d < kWave; d <<= 1) {
        const int32_t t = __shfl_up(inc, d);
        if (lane >= d) inc += t;
      }
      if (lane == kWave - 1) wsum[wave] = inc;
    }
    __syncthreads();
    if (threadIdx.x < kD) {
      int32_t at = inc - total;
      for (int w = 0; w < wave; ++w) at += wsum[w];
      for (int w = 0; w < 16; ++w) {
        const int32_t c = off[w][threadIdx.x];
        off[w][threadIdx.x] = at;
        at += c;
      }
    }
    __syncthreads();
    int32_t dst[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      if (u >= steps) continue;
      const bool live = first + u * kWave < n;
      const uint32_t d = (k[u] >> shift) & (kD - 1);
      const uint64_t match = same_digit<8>(d, live);
      dst[u] = live ? off[wave][d] + __popcll(match & below) : 0;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (live && (match >> lane) <= 1ull) off[wave][d] += __popcll(match);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u)
      if (u < steps && first + u * kWave < n) {
        if (p + 1 == passes) {
          keys_out[dst[u]] = (int32_t)k[u];
          vals_out[dst[u]] = (int32_t)v[u];
        } else {
          lk[dst[u]] = k[u];
          lv[dst[u]] = (uint16_t)v[u];
        }
      }
    if (p + 1 == passes) return;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int i = first + u * kWave;
      if (u < steps && i < n) {
        k[u] = lk[i];
        v[u] = lv[i];
      }
    }
    __syncthreads();
  }
}

struct RunArgs {
  EmbedGradArgs g;
  const int32_t *perm, *sorted;
  float* carry;            // 2 rows of cols floats for every run: sums of the segments that reach into it, and out of it
  int64_t runs;
  int run;                 // sorted ids of a run, a multiple of 8
};

template <class TO, int V, bool ADD>
__device__ __forceinline__ void write_row(const EmbedGradArgs& g, int64_t v, int64_t c, int valid, const float (&f)[V]) {
  TO* dst = (TO*)g.d_table + v * g.ld_table + c;
  float r[V];
#pragma unroll
  for (int j = 0; j < V; ++j) r[j] = f[j] * g.scale;
  if constexpr (ADD) {
    float o[V];
    load_piece<TO, V>(dst, valid, o);
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] += o[j];
  }
  store_piece<TO, V>(dst, valid, r);
}

// A group of 2^sh lanes walks a run over columns [blockIdx.y V 2^sh, ...), eight rows of d_out on their way at a time.
template <class TI, class TO, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_runs_kernel(RunArgs a, int sh) {
  constexpr int V = ElemOf<TI>::kVec;
  const int64_t run = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh;
  const int lane = threadIdx.x & ((1 << sh) - 1);
  const int64_t c = ((int64_t)blockIdx.y << sh) * V + (int64_t)lane * V;
  if (run >= a.runs || c >= a.g.cols) return;
  const int valid = (int)(a.g.cols - c < V ? a.g.cols - c : V);
  const int64_t n = a.g.n, p0 = run * a.run, p1 = p0 + a.run < n ? p0 + a.run : n;
  const int32_t none = (int32_t)a.g.rows;              // the key of ids that name no row: behind all others
  float s[V];
#pragma unroll
  for (int j = 0; j < V; ++j) s[j] = 0.0f;
  int32_t key = a.sorted[p0];
  bool open = p0 > 0 && a.sorted[p0 - 1] == key;       // the segment began in an earlier run
  for (int64_t p = p0; p < p1 && key != none; p += 8) {
    int32_t from[8], next[8];
    float f[8][V];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t q = p + u < p1 ? p + u : p1 - 1;
      from[u] = a.perm[q];
      next[u] = q + 1 < n ? a.sorted[q + 1] : -1;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) load_piece<TI, V>((const TI*)a.g.d_out + (int64_t)from[u] * a.g.ld_out + c, valid, f[u]);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (p + u >= p1 || key == none) break;
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] += f[u][j];
      if (next[u] != key || p + u + 1 == p1) {
        // slot 0: a segment from before (through the whole run, perhaps); slot 1: one that begins here and goes on
        if (open || next[u] == key) store_piece<float, V>(a.carry + (2 * run + (open ? 0 : 1)) * a.g.cols + c, valid, s);
        else write_row<TO, V, ADD>(a.g, key, c, valid, s);
        open = false;
        key = next[u];
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = 0.0f;
      }
    }
  }
}

// First place of the sorted ids whose key is at least `key`.
__device__ __forceinline__ int64_t lower_place(const int32_t* __restrict__ sorted, int64_t lo, int64_t hi, int32_t key) {
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (sorted[mid] < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

constexpr int kClearRows = 64;

// Workgroup r < runs: if a segment begins in run r and goes on behind it, its carries are added, by 2^(8 - sh) groups of lanes that take
// every so manieth of them and are then added in order.  The other workgroups zero the rows without ids (unless the caller
// accumulates), kClearRows of them each.
template <class TO, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_join_kernel(RunArgs a, int sh) {
  constexpr int V = 4;
  const int64_t n = a.g.n;
  if ((int64_t)blockIdx.x >= a.runs) {
    __shared__ uint8_t empty[kClearRows];
    const int64_t v0 = ((int64_t)blockIdx.x - a.runs) * kClearRows;
    if (threadIdx.x < kClearRows) {
      const int64_t v = v0 + threadIdx.x;
      uint8_t e = 0;
      if (v < a.g.rows) {
        const int64_t at = lower_place(a.sorted, 0, n, (int32_t)v);
        e = at == n || a.sorted[at] != (int32_t)v;
      }
      empty[threadIdx.x] = e;
    }
    __syncthreads();
    const float zero[V] = {0.f, 0.f, 0.f, 0.f};
    const int lane = threadIdx.x & ((1 << sh) - 1);
    for (int r = threadIdx.x >> sh; r < kClearRows; r += kBlock >> sh) {
      if (!empty[r]) continue;
      for (int64_t c = (int64_t)lane * V; c < a.g.cols; c += (int64_t)V << sh)
        store_piece<TO, V>((TO*)a.g.d_table + (v0 + r) * a.g.ld_table + c, (int)(a.g.cols - c < V ? a.g.cols - c : V), zero);
    }
    return;
  }
  __shared__ float4 part[kBlock];
  const int64_t run = blockIdx.x, p0 = run * a.run, p1 = p0 + a.run;
  if (p1 >= n) return;
  const int32_t key = a.sorted[p1 - 1];
  if (key == (int32_t)a.g.rows || a.sorted[p1] != key) return;
  if (p0 > 0 && a.sorted[p0 - 1] == key) return;       // it began before
  const int64_t last = (lower_place(a.sorted, p1, n, key + 1) - 1) / a.run;       // the run that the segment ends in
  const int lane = threadIdx.x & ((1 << sh) - 1), group = threadIdx.x >> sh, groups = kBlock >> sh;
  const int64_t wide = (((a.g.cols + V - 1) / V + (1 << sh) - 1) >> sh << sh) * V;       // every lane makes the same number of turns
  for (int64_t c = (int64_t)lane * V; c < wide; c += (int64_t)V << sh) {
    const int valid = c < a.g.cols ? (int)(a.g.cols - c < V ? a.g.cols - c : V) : 0;
    float s[V] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t r = run + group; r <= last; r += 8 * groups) {
      float f[8][V];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int64_t q = r + u * groups;
        load_piece<float, V>(a.carry + (2 * (q <= last ? q : run) + (q == run ? 1 : 0)) * a.g.cols + (valid > 0 ? c : 0), q <= last ? valid : 0, f[u]);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] += f[u][j];
    }
    __syncthreads();
    part[threadIdx.x] = make_float4(s[0], s[1], s[2], s[3]);
    __syncthreads();
    if (group == 0 && valid > 0) {
      for (int q = 1; q < groups; ++q) {
        const float4 t = part[(q << sh) + lane];
        s[0] += t.x; s[1] += t.y; s[2] += t.z; s[3] += t.w;
      }
      write_row<TO, V, ADD>(a.g, key, c, valid, s);
    }
  }
}

struct GradLayout {
  size_t keys_a, vals_a, keys_b, vals_b, hist, totals, carry, total;
  int64_t runs;
  int run;
};
size_t up256(size_t v) { return (v + 255) / 256 * 256; }
GradLayout grad_layout(int64_t n, int64_t cols) {
  GradLayout l{};
  // Long runs leave fewer carries, short ones more groups: enough groups of lanes to fill the chip eight times over come first.
  // 1,000,000 ids, 128 columns: runs of 64 / 128 / 256; 9001 ids, 75 columns: runs of 8 / 16 / 64.
  const int64_t lanes = (cols + 7) / 8;
  l.run = 256;
  while (l.run > 16 && n / l.run * lanes < 64 * 1024) l.run /= 2;
  l.runs = (n + l.run - 1) / l.run;
  size_t at = 0;
  auto take = [&at](size_t bytes) { const size_t o = at; at += up256(bytes); return o; };
  l.keys_a = take(4 * (size_t)n);
  l.vals_a = take(4 * (size_t)n);
  if (n > kOneSort) {
    l.keys_b = take(4 * (size_t)n);
    l.vals_b = take(4 * (size_t)n);
    l.hist = take(4 * (size_t)kBins * (size_t)((n + kChunk - 1) / kChunk));
    l.totals = take(4 * (size_t)kBins);
  }
  l.carry = take(4 * 2 * (size_t)l.runs * (size_t)cols);
  l.total = at;
  return l;
}

int lane_shift(int64_t cols, int vec) {
  const int sh = ilog2_ceil((cols + vec - 1) / vec);
  return sh > 6 ? 6 : sh;
}

template <class TI, class TO, bool ADD>
hipError_t grad_launch(const RunArgs& r, hipStream_t st) {
  constexpr int V = ElemOf<TI>::kVec;
  if (r.runs > 0) {
    const int sh = lane_shift(r.g.cols, V);
    const unsigned slabs = (unsigned)((r.g.cols + ((int64_t)V << sh) - 1) / ((int64_t)V << sh));
    embed_runs_kernel<TI, TO, ADD><<<dim3((unsigned)(((r.runs << sh) + kBlock - 1) / kBlock), slabs), kBlock, 0, st>>>(r, sh);
  }
  const int64_t clear = ADD ? 0 : (r.g.rows + kClearRows - 1) / kClearRows;
  if (r.runs + clear > 0) embed_join_kernel<TO, ADD><<<(unsigned)(r.runs + clear), kBlock, 0, st>>>(r, lane_shift(r.g.cols, 4));
  return hipGetLastError();
}

template <class TI, class TO>
hipError_t grad_typed(const RunArgs& r, hipStream_t st) {
  return r.g.accumulate ? grad_launch<TI, TO, true>(r, st) : grad_launch<TI, TO, false>(r, st);
}

}  // namespace

size_t embed_grad_bytes(int64_t n, int64_t cols) { return grad_layout(n, cols).total; }

hipError_t launch_embed_grad(const EmbedGradArgs& a, char* ws, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const GradLayout l = grad_layout(a.n, a.cols);
  const int32_t *keys = (int32_t*)(ws + l.keys_a), *vals = (int32_t*)(ws + l.vals_a);
  const uint32_t rows = (uint32_t)a.rows;
  int bits = ilog2_ceil(a.rows + 1);                   // keys 0 .. rows
  if (bits < 1) bits = 1;
  if (a.n > 0 && a.n <= kOneSort) {
    id_sort_one_kernel<<<1, 1024, 0, st>>>(a.ids, (int)a.n, rows, (bits + 7) / 8, (int32_t*)keys, (int32_t*)vals);
  } else if (a.n > 0) {
    const int chunks = (int)((a.n + kChunk - 1) / kChunk), passes = (bits + kBits - 1) / kBits;
    int32_t *hist = (int32_t*)(ws + l.hist), *totals = (int32_t*)(ws + l.totals);
    const int32_t *kin = a.ids, *vin = nullptr;
    for (int p = 0; p < passes; ++p) {
      int32_t *kout = (int32_t*)(ws + (p % 2 == 0 ? l.keys_a : l.keys_b)), *vout = (int32_t*)(ws + (p % 2 == 0 ? l.vals_a : l.vals_b));
      if (p == 0) id_hist_kernel<true><<<chunks, kBlock, 0, st>>>(kin, a.n, rows, kBits * p, chunks, hist);
      else id_hist_kernel<false><<<chunks, kBlock, 0, st>>>(kin, a.n, rows, kBits * p, chunks, hist);
      id_scan_kernel<<<kBins, kBlock, 0, st>>>(hist, chunks, totals);
      if (p == 0) id_scatter_kernel<true><<<chunks, kBlock, 0, st>>>(kin, vin, a.n, rows, kBits * p, chunks, hist, totals, kout, vout);
      else id_scatter_kernel<false><<<chunks, kBlock, 0, st>>>(kin, vin, a.n, rows, kBits * p, chunks, hist, totals, kout, vout);
      kin = kout;
      vin = vout;
    }
    keys = kin;
    vals = vin;
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const RunArgs r{a, vals, keys, (float*)(ws + l.carry), l.runs, l.run};
  if (a.out_bf16) return a.table_bf16 ? grad_typed<bf16_t, bf16_t>(r, st) : grad_typed<bf16_t, float>(r, st);
  return a.table_bf16 ? grad_typed<float, bf16_t>(r, st) : grad_typed<float, float>(r, st);
}

}  // namespace ilargi
