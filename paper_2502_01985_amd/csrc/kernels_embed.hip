// Rows of a learned table picked by keys, and the gradient of that table: rows of the output's gradient summed by key.
#include "ilargi_layers.h"

namespace ilargi {

namespace {

// Sixteen aligned bytes written past the caches.
template <class TO, int V>
__device__ __forceinline__ void store_streaming(TO* p, const float (&f)[V]) {
  typedef uint32_t words __attribute__((ext_vector_type(V * sizeof(TO) / 4)));
  Piece<TO, V> t;
#pragma unroll
  for (int j = 0; j < V; ++j) t.v[j] = (TO)f[j];
  __builtin_nontemporal_store(__builtin_bit_cast(words, t), reinterpret_cast<words*>(p));
}

// out[i, :] = scale table[ids[i], :] (+ out[i, :]): bound by the bytes of the output and of the table's distinct rows.  A group of 2^sh
// lanes shares a row; every lane takes 16-byte pieces of it.  STREAM: the output is larger than the caches and in aligned pieces, and
// is written past them, which leaves them to the table: 1,000,000 rows of 256 from 100,000, bfloat16, skewed keys, 93 us = 6.1 TB/s
// of its 563 MB, and 176 us through the caches; outputs of 15 to 102 MB take the same either way.
template <class TI, class TO, bool ADD, bool STREAM>
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
    if constexpr (STREAM) store_streaming<TO, V>(dst + c, f);
    else store_piece<TO, V>(dst + c, valid, f);
  }
}

template <class TI, class TO>
hipError_t embed_typed(const EmbedArgs& a, hipStream_t st) {
  constexpr int V = ElemOf<TI>::kVec < ElemOf<TO>::kVec ? ElemOf<TI>::kVec : ElemOf<TO>::kVec;
  int sh = ilog2_ceil((a.cols + V - 1) / V);
  if (sh > 6) sh = 6;
  const bool whole = a.cols % V == 0 && a.ld_out * sizeof(TO) % 16 == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && V * sizeof(TO) >= 8;
  const bool past = whole && a.n * a.cols * (int64_t)sizeof(TO) >= kStreamBytes;
  return in_parts(((a.n << sh) + kBlock - 1) / kBlock, kBlock, [&](int64_t first, unsigned blocks) {
    const int64_t row = first * (kBlock >> sh), rows = (int64_t)blocks * (kBlock >> sh);
    EmbedArgs b = a;
    b.ids += row;
    b.out = (TO*)a.out + row * a.ld_out;
    b.n = a.n - row < rows ? a.n - row : rows;
    if (a.accumulate) embed_kernel<TI, TO, true, false><<<blocks, kBlock, 0, st>>>(b, sh);
    else if (past) embed_kernel<TI, TO, false, true><<<blocks, kBlock, 0, st>>>(b, sh);
    else embed_kernel<TI, TO, false, false><<<blocks, kBlock, 0, st>>>(b, sh);
  });
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
//
// Bound by the rows of d_out, gathered 256 bytes at a time, and the launches of the sort.  1,000,000 ids of 100,000 x 128, bfloat16,
// skewed: 158 us, of which the sort 50, the runs 70 (256 MB: 3.7 TB/s), the carries and rows without ids 31; one row holds 13 % of
// the ids.  9001 ids of 6040 x 75, float32: 40 us, of which the sort 22.
namespace {

constexpr int kBits = 9, kBins = 1 << kBits;      // two passes for tables of up to 262,143 rows
constexpr int kChunk = 4096, kSort = 512;         // ids a workgroup sorts by one digit, and its threads
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
__global__ __launch_bounds__(kSort) void id_hist_kernel(const int32_t* __restrict__ keys, int64_t n, uint32_t rows, int shift, int chunks,
                                                        int32_t* __restrict__ hist) {
  __shared__ int32_t h[kBins];
  static_assert(kBins == kSort, "a digit a thread");
  h[threadIdx.x] = 0;
  const int64_t at = (int64_t)blockIdx.x * kChunk + threadIdx.x;
  uint32_t k[kChunk / kSort];
#pragma unroll
  for (int u = 0; u < kChunk / kSort; ++u) k[u] = at + u * kSort < n ? (FIRST ? id_key(keys[at + u * kSort], rows) : (uint32_t)keys[at + u * kSort]) : 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kChunk / kSort; ++u)
    if (at + u * kSort < n) atomicAdd(&h[(k[u] >> shift) & (kBins - 1)], 1);
  __syncthreads();
  hist[(int64_t)threadIdx.x * chunks + blockIdx.x] = h[threadIdx.x];
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

// The place of this lane's id among the equal digits of its wavefront so far: `seen` counts them, and the highest lane of a digit
// adds this step's.  (A wavefront's own counters: no barrier, and no atomics, which would queue on a digit that many ids share.)
template <int BITS>
__device__ __forceinline__ int32_t rank_in_wave(uint32_t d, bool live, int32_t* seen) {
  const int lane = threadIdx.x % kWave;
  const uint64_t match = same_digit<BITS>(d, live), below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
  const int32_t before = live ? seen[d] : 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (live && (match >> lane) <= 1ull) seen[d] = before + __popcll(match);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  return before + __popcll(match & below);
}

// Every wavefront walks its part of the chunk 64 ids at a time; an id's place is its digit's first place, plus the equal digits of the
// chunks and wavefronts before, plus its rank in its wavefront.
template <bool FIRST>
__global__ __launch_bounds__(kSort) void id_scatter_kernel(const int32_t* __restrict__ keys_in, const int32_t* __restrict__ vals_in, int64_t n, uint32_t rows,
                                                           int shift, int chunks, const int32_t* __restrict__ hist, const int32_t* __restrict__ totals,
                                                           int32_t* __restrict__ keys_out, int32_t* __restrict__ vals_out) {
  constexpr int kWaves = kSort / kWave, kSteps = kChunk / kSort;
  static_assert(kBins == kSort, "a digit a thread");
  __shared__ int32_t off[kWaves][kBins];
  __shared__ int32_t wsum[kWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, t = threadIdx.x;
  const int64_t first = (int64_t)blockIdx.x * kChunk + (int64_t)wave * kSteps * kWave + lane;
  uint32_t k[kSteps];
  int32_t v[kSteps], rank[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int64_t i = first + u * kWave;
    k[u] = 0; v[u] = 0;
    if (i < n) {
      k[u] = FIRST ? id_key(keys_in[i], rows) : (uint32_t)keys_in[i];
      v[u] = FIRST ? (int32_t)i : vals_in[i];
    }
  }
  const int32_t total = totals[t], mine = hist[(int64_t)t * chunks + blockIdx.x];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) off[w][t] = 0;
  int32_t inc = total;
  for (int d = 1; d < kWave; d <<= 1) {
    const int32_t x = __shfl_up(inc, d);
    if (lane >= d) inc += x;
  }
  if (lane == kWave - 1) wsum[wave] = inc;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kSteps; ++u) rank[u] = rank_in_wave<kBits>((k[u] >> shift) & (kBins - 1), first + u * kWave < n, off[wave]);
  int32_t at = inc - total + mine;
  for (int w = 0; w < wave; ++w) at += wsum[w];
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int32_t c = off[w][t];
    off[w][t] = at;
    at += c;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kSteps; ++u)
    if (first + u * kWave < n) {
      const int32_t dst = off[wave][(k[u] >> shift) & (kBins - 1)] + rank[u];
      keys_out[dst] = (int32_t)k[u];
      vals_out[dst] = v[u];
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
  for (int p = 0; p < passes; ++p) {
    const int shift = 8 * p;
    for (int i = threadIdx.x; i < 16 * kD; i += 1024) off[i / kD][i % kD] = 0;
    __syncthreads();
    int32_t rank[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u)
      if (u < steps) rank[u] = rank_in_wave<8>((k[u] >> shift) & (kD - 1), first + u * kWave < n, off[wave]);
    __syncthreads();
    int32_t c[16], total = 0, inc = 0;
    if (threadIdx.x < kD) {
#pragma unroll
      for (int w = 0; w < 16; ++w) { c[w] = off[w][threadIdx.x]; total += c[w]; }
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
#pragma unroll
      for (int w = 0; w < 16; ++w) { off[w][threadIdx.x] = at; at += c[w]; }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSteps; ++u)
      if (u < steps && first + u * kWave < n) {
        const int32_t dst = off[wave][(k[u] >> shift) & (kD - 1)] + rank[u];
        if (p + 1 == passes) {
          keys_out[dst] = (int32_t)k[u];
          vals_out[dst] = (int32_t)v[u];
        } else {
          lk[dst] = k[u];
          lv[dst] = (uint16_t)v[u];
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

// A group of 2^sh lanes walks a run over columns [(slab + blockIdx.y) V 2^sh, ...), eight rows of d_out on their way at a time.
template <class TI, class TO, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_runs_kernel(RunArgs a, int sh, int64_t slab) {
  constexpr int V = ElemOf<TI>::kVec;
  const int64_t run = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh;
  const int lane = threadIdx.x & ((1 << sh) - 1);
  const int64_t c = ((slab + blockIdx.y) << sh) * V + (int64_t)lane * V;
  if (run >= a.runs || c >= a.g.cols) return;
  const int valid = (int)(a.g.cols - c < V ? a.g.cols - c : V);
  const int64_t n = a.g.n, p0 = run * a.run, p1 = p0 + a.run < n ? p0 + a.run : n;
  const int32_t none = (int32_t)a.g.rows;              // the key of ids that name no row: behind all others
  float s[V];
#pragma unroll
  for (int j = 0; j < V; ++j) s[j] = 0.0f;
  int32_t from[8], next[8];
  auto ask = [&](int64_t p) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t q = p + u < p1 ? p + u : p1 - 1;
      from[u] = a.perm[q];
      next[u] = q + 1 < n ? a.sorted[q + 1] : -1;
    }
  };
  ask(p0);
  int32_t key = a.sorted[p0];
  bool open = p0 > 0 && a.sorted[p0 - 1] == key;       // the segment began in an earlier run
  for (int64_t p = p0; p < p1 && key != none; p += 8) {
    float f[8][V];
    int32_t then[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      load_piece<TI, V>((const TI*)a.g.d_out + (int64_t)from[u] * a.g.ld_out + c, valid, f[u]);
      then[u] = next[u];
    }
    if (p + 8 < p1) ask(p + 8);                         // the next places, while the rows are on their way
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (p + u >= p1 || key == none) break;
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] += f[u][j];
      if (then[u] != key || p + u + 1 == p1) {
        // slot 0: a segment from before (through the whole run, perhaps); slot 1: one that begins here and goes on
        if (open || then[u] == key) store_piece<float, V>(a.carry + (2 * run + (open ? 0 : 1)) * a.g.cols + c, valid, s);
        else write_row<TO, V, ADD>(a.g, key, c, valid, s);
        open = false;
        key = then[u];
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = 0.0f;
      }
    }
  }
}

// A load that depends on the one before costs most of a microsecond here (the sorted ids were written by other compute units), so a
// whole wavefront looks at 64 places at a time.
// First place of the sorted ids whose key is at least `key`.
__device__ __forceinline__ int64_t wave_lower(const int32_t* __restrict__ sorted, int64_t n, int64_t key) {
  const int lane = threadIdx.x % kWave;
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
    const int less = __popcll(__ballot(at < hi && sorted[at] < key));       // the keys rise: the first lanes
    if (less == 0) return lo;
    const int64_t end = lo + less * step;
    lo = end - step + 1;
    if (end < hi) hi = end;
    if (step == 1) return lo;
  }
  return lo;
}
// Runs that the segment of `key` reaches which goes on behind run `run`: those that follow and begin with its key.
__device__ __forceinline__ int32_t wave_span(const RunArgs& a, int64_t run, int32_t key) {
  const int lane = threadIdx.x % kWave;
  auto begins = [&](int64_t r) { return r < a.runs && a.sorted[r * a.run] == key; };
  int64_t in = run + 1;                                 // run `in` begins with the key; so many runs of 64 of them behind it
  int more = __popcll(__ballot(begins(in + 1 + lane)));
  if (more < kWave) return (int32_t)(in + more - run + 1);
  for (int64_t step = kWave * kWave; step >= 1; step /= kWave) {
    do {
      more = __popcll(__ballot(begins(in + (lane + 1) * step)));
      in += more * step;
    } while (more == kWave);
  }
  return (int32_t)(in - run + 1);
}

constexpr int kClearRows = 256, kJoin = 1024, kJoinRuns = 64, kShortSpan = 16;

// Carries of runs from, from + by, .. last of a segment that begins in run `begin`, added to s, eight on their way at a time.
template <int V>
__device__ __forceinline__ void add_carries(const RunArgs& a, int64_t begin, int64_t from, int64_t by, int64_t last, int64_t c, int valid, float (&s)[V]) {
  for (int64_t r = from; r <= last; r += 8 * by) {
    float f[8][V];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t q = r + u * by;
      load_piece<float, V>(a.carry + (2 * (q <= last ? q : begin) + (q == begin ? 1 : 0)) * a.g.cols + (valid > 0 ? c : 0), q <= last ? valid : 0, f[u]);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] += f[u][j];
  }
}

// The first workgroups look at kJoinRuns runs each: a segment that begins in one of them and goes on behind it is the sum of its
// carries.  Up to kShortSpan of them are added by a group of 2^sh lanes, longer ones by all groups, each every so manieth, which are
// then added in order.  The other workgroups zero the rows without ids (unless the caller accumulates), kClearRows of them each.
// `first`: workgroups of this call in earlier launches.
template <class TO, bool ADD>
__global__ __launch_bounds__(kJoin) void embed_join_kernel(RunArgs a, int sh, int64_t joins, int64_t first) {
  constexpr int V = 4;
  const int64_t id = first + blockIdx.x;
  const int64_t n = a.g.n;
  const int lane = threadIdx.x & ((1 << sh) - 1), group = threadIdx.x >> sh, groups = kJoin >> sh;
  if (id >= joins) {
    __shared__ uint8_t full[kClearRows];
    __shared__ int64_t ends[2];
    const int64_t v0 = (id - joins) * kClearRows, v1 = v0 + kClearRows < a.g.rows ? v0 + kClearRows : a.g.rows;
    if (threadIdx.x < kClearRows) full[threadIdx.x] = v0 + threadIdx.x >= v1;
    if (threadIdx.x < 2 * kWave) {
      const int64_t at = wave_lower(a.sorted, n, threadIdx.x < kWave ? v0 : v1);
      if (threadIdx.x % kWave == 0) ends[threadIdx.x / kWave] = at;
    }
    __syncthreads();
    const int64_t b = ends[0], e = ends[1];
    if (e - b <= 16 * kJoin) {
#pragma unroll 4
      for (int64_t p = b + threadIdx.x; p < e; p += kJoin) full[a.sorted[p] - v0] = 1;
    } else if (threadIdx.x < kClearRows && v0 + threadIdx.x < v1) {      // a row with many ids is among them: look for each
      const int32_t v = (int32_t)(v0 + threadIdx.x);
      int64_t lo = b, hi = e;
      while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (a.sorted[mid] < v) lo = mid + 1;
        else hi = mid;
      }
      full[threadIdx.x] = lo < e && a.sorted[lo] == v;
    }
    __syncthreads();
    const float zero[V] = {0.f, 0.f, 0.f, 0.f};
    for (int r = group; r < kClearRows; r += groups) {
      if (full[r]) continue;
      for (int64_t c = (int64_t)lane * V; c < a.g.cols; c += (int64_t)V << sh)
        store_piece<TO, V>((TO*)a.g.d_table + (v0 + r) * a.g.ld_table + c, (int)(a.g.cols - c < V ? a.g.cols - c : V), zero);
    }
    return;
  }
  __shared__ float4 part[kJoin];
  __shared__ int32_t keys[kJoinRuns], spans[kJoinRuns];     // runs that the segment reaches, 0 where there is none
  const int64_t run0 = id * kJoinRuns;
  if (threadIdx.x < kJoinRuns) {
    const int64_t run = run0 + threadIdx.x, p0 = run * a.run, p1 = p0 + a.run;
    int32_t key = 0, span = 0;
    if (p1 < n) {
      key = a.sorted[p1 - 1];
      span = key != (int32_t)a.g.rows && a.sorted[p1] == key && !(p0 > 0 && a.sorted[p0 - 1] == key);
    }
    keys[threadIdx.x] = key;
    spans[threadIdx.x] = span;
  }
  __syncthreads();
  const int wave = threadIdx.x / kWave;
#pragma unroll
  for (int q = 0; q < kJoinRuns / (kJoin / kWave); ++q) {
    const int r = wave + q * (kJoin / kWave);
    if (spans[r] == 0) continue;
    const int32_t span = wave_span(a, run0 + r, keys[r]);
    if (threadIdx.x % kWave == 0) spans[r] = span;
  }
  __syncthreads();
  for (int r = group; r < kJoinRuns; r += groups) {
    if (spans[r] == 0 || spans[r] > kShortSpan) continue;
    const int64_t run = run0 + r;
    for (int64_t c = (int64_t)lane * V; c < a.g.cols; c += (int64_t)V << sh) {
      const int valid = (int)(a.g.cols - c < V ? a.g.cols - c : V);
      float s[V] = {0.f, 0.f, 0.f, 0.f};
      add_carries<V>(a, run, run, 1, run + spans[r] - 1, c, valid, s);
      write_row<TO, V, ADD>(a.g, keys[r], c, valid, s);
    }
  }
  const int64_t wide = (((a.g.cols + V - 1) / V + (1 << sh) - 1) >> sh << sh) * V;       // every lane makes the same number of turns
  static_assert(kJoinRuns == kWave, "a run a lane");
  for (uint64_t left = __ballot(spans[threadIdx.x % kWave] > kShortSpan); left != 0; left &= left - 1) {
    const int r = __builtin_ctzll(left);
    const int64_t run = run0 + r;
    for (int64_t c = (int64_t)lane * V; c < wide; c += (int64_t)V << sh) {
      const int valid = c < a.g.cols ? (int)(a.g.cols - c < V ? a.g.cols - c : V) : 0;
      float s[V] = {0.f, 0.f, 0.f, 0.f};
      add_carries<V>(a, run, run + group, groups, run + spans[r] - 1, c, valid, s);
      __syncthreads();
      part[threadIdx.x] = make_float4(s[0], s[1], s[2], s[3]);
      __syncthreads();
      if (group == 0 && valid > 0) {
        for (int q = 1; q < groups; ++q) {
          const float4 t = part[(q << sh) + lane];
          s[0] += t.x; s[1] += t.y; s[2] += t.z; s[3] += t.w;
        }
        write_row<TO, V, ADD>(a.g, keys[r], c, valid, s);
      }
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
  // Whole calls with runs of 8 / 16 / 32 / 64 / 128 / 256: 1,000,000 ids of 128 columns, bfloat16, skewed: 290 / 194 / 158 / 143 / 174 / 251 us
  // (the rule takes 32); 9001 ids of 75 columns, float32: 38 / 39.6 / 44 / 54 / 70 / 109 (the rule takes 16).
  const int64_t lanes = (cols + 7) / 8;
  l.run = 256;
  while (l.run > 16 && n / l.run * lanes < 256 * 1024) l.run /= 2;
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
  if (r.runs > 0) {                                      // (at most 2^23 runs of 64 lanes: in one launch)
    const int sh = lane_shift(r.g.cols, V);
    const int64_t slabs = (r.g.cols + ((int64_t)V << sh) - 1) / ((int64_t)V << sh);
    for (int64_t slab = 0; slab < slabs; slab += kMostAcross) {
      const unsigned across = (unsigned)(slabs - slab < kMostAcross ? slabs - slab : kMostAcross);
      embed_runs_kernel<TI, TO, ADD><<<dim3((unsigned)(((r.runs << sh) + kBlock - 1) / kBlock), across), kBlock, 0, st>>>(r, sh, slab);
    }
  }
  const int64_t clear = ADD ? 0 : (r.g.rows + kClearRows - 1) / kClearRows;
  const int64_t joins = (r.runs + kJoinRuns - 1) / kJoinRuns;
  return in_parts(joins + clear, kJoin, [&](int64_t first, unsigned blocks) {
    embed_join_kernel<TO, ADD><<<blocks, kJoin, 0, st>>>(r, lane_shift(r.g.cols, 4), joins, first);
  });
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
      if (p == 0) id_hist_kernel<true><<<chunks, kSort, 0, st>>>(kin, a.n, rows, kBits * p, chunks, hist);
      else id_hist_kernel<false><<<chunks, kSort, 0, st>>>(kin, a.n, rows, kBits * p, chunks, hist);
      id_scan_kernel<<<kBins, kBlock, 0, st>>>(hist, chunks, totals);
      if (p == 0) id_scatter_kernel<true><<<chunks, kSort, 0, st>>>(kin, vin, a.n, rows, kBits * p, chunks, hist, totals, kout, vout);
      else id_scatter_kernel<false><<<chunks, kSort, 0, st>>>(kin, vin, a.n, rows, kBits * p, chunks, hist, totals, kout, vout);
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
