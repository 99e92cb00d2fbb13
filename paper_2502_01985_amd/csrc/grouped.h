// Products over ragged groups of rows: where the groups lie, and the kernels' arguments (kernels_grouped.hip, kernels_grouped16.hip).
#ifndef ILARGI_GROUPED_H_
#define ILARGI_GROUPED_H_

#include "mm_epilogue.h"

namespace ilargi {

// Up to 64 groups every wavefront works out of the offsets itself where they lie, a group a lane: no launch stands before the products
// (it took 3 to 8 us).  With more, one launch does it for all others and leaves:
struct GroupIndex {
  const int32_t* offsets;
  int groups, n;
  int* start;       // groups + 1: first rows, ascending, in [0, n]
  int* tiles;       // prefix of the blocks of rows of every group
  int* order;       // groups by their rows, the longest first (up to kMostSorted groups; else as they come)
  int* parts;       // prefix, in that order, of the parts of rows that the products over rows are split into, one at least of every group
  int* slots;       // prefix, in that order, of those of groups of several parts
  int* chunks;      // prefix of the chunks of rows of the column sums
};
constexpr int kMostSorted = 512, kMostInLanes = kWave;
// (a prefix p has p[q] <= u < p[q + 1] for the units u of place q)

// Products of the rows of every group with its own matrix.  P's rows and the result's are the groups'; Q's matrices are far_q elements apart.
template <class Prod>
struct GroupedRows {
  Prod p;                     // M = n
  GroupIndex at;
  int64_t far_q, far_bias;    // elements
  int64_t share;              // of k, in the block's units
  float* partial;             // shares of n x (N to a multiple of 4) where k is split
};
// Products over the rows of every group: P and Q are n rows over k, C a matrix a group.
template <class Prod>
struct GroupedSums {
  Prod p;                     // K = n
  GroupIndex at;
  int64_t far_out;
  int part;                   // rows
  float* partial;             // M x (N to a multiple of 4) a slot
};

template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
// Over the lanes up to this one, of values that are not negative: their sum or the largest.
template <bool MOST>
__device__ __forceinline__ int scan_lanes(int v) {
  auto take = [&](int o) { v = MOST ? (v > o ? v : o) : v + o; };
  take(from_lane<0x111, 0xf>(v));       // 1, 2, 4 and 8 lanes before, in sixteen
  take(from_lane<0x112, 0xf>(v));
  take(from_lane<0x114, 0xf>(v));
  take(from_lane<0x118, 0xf>(v));
  take(from_lane<0x142, 0xa>(v));       // the last of the sixteen before
  take(from_lane<0x143, 0xc>(v));       // ... of the thirty-two before
  return v;
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// The place of unit u in a prefix of n places: the last one that begins at or before it.  A wavefront looks at 64 places at a time.
__device__ __forceinline__ int place_of(const int* __restrict__ prefix, int n, int u) {
  int lo = 0, count = n;
  while (count > 1) {
    const int step = (count + kWave - 1) / kWave, at = (int)(threadIdx.x % kWave) * step;
    const bool before = at < count && prefix[lo + at] <= u;
    const int last = __popcll(__ballot(before)) - 1;
    lo += last * step;
    count = count - last * step < step ? count - last * step : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The groups' first rows and their ends, a group a lane.
struct Lanes {
  int start, end;
  __device__ __forceinline__ explicit Lanes(const GroupIndex& at) {
    const int lane = threadIdx.x % kWave;
    auto inside = [&](int v) { return v < 0 ? 0 : v > at.n ? at.n : v; };
    const bool is = lane < at.groups;
    const int v = is ? inside(at.offsets[lane]) : 0, next = is ? inside(at.offsets[lane + 1]) : 0;
    start = scan_lanes<true>(v);                  // (an offset below an earlier one counts as that)
    end = next > start ? next : start;
  }
};
__device__ __forceinline__ bool in_lanes(const GroupIndex& at) { return at.groups <= kMostInLanes; }
__device__ __forceinline__ int blocks_of_rows(int rows, int size) { return (int)(((uint32_t)rows + (uint32_t)size - 1) / (uint32_t)size); }

// Where unit u of a launch lies: its group, the group's rows, and which of the group's units it is.
struct Unit {
  int group, first, rows, number;
};
// Blocks of `size` rows of every group; `prefix` where the groups are not in lanes.
struct Blocks {
  const GroupIndex& at;
  const int* prefix;
  int start, end, before, total;
  __device__ __forceinline__ Blocks(const GroupIndex& at, const int* prefix, int size) : at(at), prefix(prefix) {
    if (in_lanes(at)) {
      const Lanes l(at);
      const int mine = blocks_of_rows(l.end - l.start, size), upto = scan_lanes<false>(mine);
      start = l.start; end = l.end; before = upto - mine;
      total = lane_value(upto, kWave - 1);
    } else {
      start = end = before = 0;
      total = prefix[at.groups];
    }
  }
  __device__ __forceinline__ Unit find(int u) const {
    if (in_lanes(at)) {
      const int g = __popcll(__ballot((int)(threadIdx.x % kWave) < at.groups && before <= u)) - 1, first = lane_value(start, g);
      return {g, first, lane_value(end, g) - first, u - lane_value(before, g)};
    }
    const int g = place_of(prefix, at.groups, u), first = at.start[g];
    return {g, first, at.start[g + 1] - first, u - prefix[g]};
  }
  // the first unit of a group, and that of the next
  __device__ __forceinline__ void of_group(int g, int* first, int* end) const {
    *first = in_lanes(at) ? lane_value(before, g) : prefix[g];
    *end = !in_lanes(at) ? prefix[g + 1] : g + 1 < at.groups ? lane_value(before, g + 1) : total;
  }
};

// Parts of `size` rows, the longest groups first, one at least of every group; those of groups of several have a slot each.
struct Parts {
  const GroupIndex& at;
  int start, end, group, before, slot, total;       // of the place that is this lane
  __device__ __forceinline__ Parts(const GroupIndex& at, int size) : at(at) {
    if (in_lanes(at)) {
      const Lanes l(at);
      const int lane = threadIdx.x % kWave, mine = l.end - l.start;
      int place = 0;
      for (int o = 0; o < at.groups; ++o) {
        const int other = lane_value(mine, o);
        place += other > mine || (other == mine && o < lane);
      }
      if (lane >= at.groups) place = lane;
      group = __builtin_amdgcn_ds_permute(place * 4, lane);
      start = __shfl(l.start, group);
      end = __shfl(l.end, group);
      const int b = blocks_of_rows(end - start, size), parts = lane < at.groups ? (b > 1 ? b : 1) : 0, held = parts > 1 ? parts : 0;
      const int upto = scan_lanes<false>(parts);
      before = upto - parts;
      slot = scan_lanes<false>(held) - held;
      total = lane_value(upto, kWave - 1);
    } else {
      start = end = group = before = slot = 0;
      total = at.parts[at.groups];
    }
  }
  struct Place {
    int group, first, end, parts, slot, number;
  };
  __device__ __forceinline__ Place place(int q, int u) const {
    if (in_lanes(at)) {
      const int b = lane_value(before, q), next = q + 1 < at.groups ? lane_value(before, q + 1) : total;
      return {lane_value(group, q), lane_value(start, q), lane_value(end, q), next - b, lane_value(slot, q), u - b};
    }
    const int g = at.order[q], b = at.parts[q];
    return {g, at.start[g], at.start[g + 1], at.parts[q + 1] - b, at.slots[q], u - b};
  }
  __device__ __forceinline__ Place find(int u) const {
    return place(in_lanes(at) ? __popcll(__ballot((int)(threadIdx.x % kWave) < at.groups && before <= u)) - 1 : place_of(at.parts, at.groups, u), u);
  }
};

template <class T>
__device__ __forceinline__ void move_to(T*& p, int64_t elements, int size) {
  if (p != nullptr) p = (T*)((const char*)p + elements * size);
}

// The product of one block of a group's rows: r0 .. r0 + rows with matrix g.
template <class Prod>
__device__ __forceinline__ Prod rows_of(const GroupedRows<Prod>& a, int g, int64_t r0, int64_t rows, int size) {
  Prod b = a.p;
  b.M = rows;
  move_to(b.P.p, r0 * b.P.ld, size);
  move_to(b.Q.p, g * a.far_q, size);
  move_to(b.epi.bias, g * a.far_bias, size);
  move_to(b.epi.src, r0 * b.epi.ld_src, size);
  move_to(b.epi.pre, r0 * b.epi.ld_pre, size);
  move_to(b.epi.out, r0 * b.epi.ld_out, size);
  return b;
}
template <class Prod>
__device__ __forceinline__ Prod sums_of(const GroupedSums<Prod>& a, int g, int64_t r0, int64_t rows, int size) {
  Prod b = a.p;
  b.K = rows;
  move_to(b.P.p, r0 * b.P.ld, size);
  move_to(b.Q.p, r0 * b.Q.ld, size);
  move_to(b.epi.src, g * a.far_out, size);
  move_to(b.epi.out, g * a.far_out, size);
  return b;
}

// run(product, block of rows, block of columns, first row of the group) for block `id` of a launch of rows, `tn` blocks of columns.
template <int SIZE, class Prod, class F>
__device__ __forceinline__ void grouped_rows_block(const GroupedRows<Prod>& a, const Blocks& blocks, int id, int tn, F run) {
  int u, tj;
  block_of(id, blocks.total, tn, &u, &tj);
  const Unit b = blocks.find(u);
  run(rows_of(a, b.group, b.first, b.rows, SIZE), b.number, tj, (int64_t)b.first);
}
template <class Prod>
__device__ __forceinline__ float* sums_of_rows(const GroupedRows<Prod>& a, int64_t first) {
  return a.partial != nullptr ? a.partial + ((int64_t)blockIdx.z * a.p.M + first) * ((a.p.N + 3) / 4 * 4) : nullptr;
}
// A group without rows has a matrix of zeros: they are stored as they are.  (126 groups of 4000 x 96, of which 3 rows fill some, float32: 74 us in all, 99
// with blocks of no steps instead.)
template <int SIZE>
__device__ __forceinline__ void zero_block(const Epilogue& e, int64_t i0, int64_t j0, int tile, int64_t M, int64_t N) {
  const int quads = tile / 4;
  const float none[4] = {0.f, 0.f, 0.f, 0.f};
  for (int q = threadIdx.x; q < tile * quads; q += blockDim.x) {
    const int64_t i = i0 + q / quads, j = j0 + q % quads * 4;
    const int valid = quad_valid(i, j, M, N);
    if (valid > 0) store4_any(e.out, i * e.ld_out + j, SIZE == 2, valid, none);
  }
}
template <int SIZE, class Prod, class F>
__device__ __forceinline__ void grouped_sums_block(const GroupedSums<Prod>& a, int id, int tile, int tm, int tn, F run) {
  const Parts parts(a.at, a.part);
  const int u = id / (tm * tn);
  if (u >= parts.total) return;
  int ti, tj;
  block_of(id - u * (tm * tn), tm, tn, &ti, &tj);
  const Parts::Place q = parts.find(u);
  const int64_t r0 = q.first + (int64_t)q.number * a.part, rows = q.end - r0 < a.part ? q.end - r0 : a.part;
  if (rows == 0) {
    if (a.p.epi.src == nullptr) zero_block<SIZE>(sums_of(a, q.group, r0, rows, SIZE).epi, (int64_t)ti * tile, (int64_t)tj * tile, tile, a.p.M, a.p.N);
    return;                                                  // (or nothing to add)
  }
  float* to = q.parts > 1 ? a.partial + (int64_t)(q.slot + q.number) * a.p.M * ((a.p.N + 3) / 4 * 4) : nullptr;
  run(sums_of(a, q.group, r0, rows, SIZE), ti, tj, to);
}

// The elementwise pass of a gradient and its column sums.
struct GroupedGrad {
  LayerGradArgs g;
  GroupIndex at;
  int chunk;
  int64_t ld_dbias;
  float* partial;        // m sums a chunk
};

// The chunks of every group, sixteen threads a column: each adds every sixteenth, then they are added in order, in float64: they cancel
// each other as the rows do.  16 columns from 16 `block` on, of group g.
struct BiasLds {
  double part[16][17];
};
template <class T>
__device__ __forceinline__ void bias_block(const GroupedGrad& a, int64_t block, int g, BiasLds& lds) {
  const int c = threadIdx.x % 16, q = threadIdx.x / 16;
  const int64_t j = block * 16 + c, m = a.g.m;
  double s = 0.0;
  int first_chunk, end_chunk;
  Blocks(a.at, a.at.chunks, a.chunk).of_group(g, &first_chunk, &end_chunk);
  if (j < m) {
#pragma unroll 4
    for (int u = first_chunk + q; u < end_chunk; u += 16) s += a.partial[(int64_t)u * m + j];
  }
  lds.part[q][c] = s;
  __syncthreads();
  if (q != 0 || j >= m) return;
  for (int u = 1; u < 16; ++u) s += lds.part[u][c];
  T* const out = (T*)a.g.d_bias + g * a.ld_dbias + j;
  *out = (T)(float)(a.g.accumulate ? (double)(float)*out + s : s);
}

// Blocks of 256: one workgroup fits a compute unit, so the blocks go in rounds of kUnits, and those of the last round, where they are less
// than half of one, are split into shares of k that fill it (`partial`: kTailBytes for their sums; a launch adds them).
constexpr int kUnits = 256;
constexpr size_t kTailBytes = (size_t)kUnits * 256 * 256 * 4;
struct Tail {
  int full, rest, shares, share;      // blocks of whole rounds, blocks of the last, shares of each of those, steps of a share
};
__host__ __device__ inline Tail tail_of(int total, int steps) {
  Tail t{total - total % kUnits, total % kUnits, 1, steps};
  if (t.rest == 0) return t;
  const int most = kUnits / t.rest < steps / 4 ? kUnits / t.rest : steps / 4;
  if (most < 2) return t;
  t.share = (steps + most - 1) / most;
  t.shares = (steps + t.share - 1) / t.share;
  return t;
}
hipError_t launch_grouped16_rows(const GroupedRows<Product16>& a, int tile, int64_t tiles, int splits, hipStream_t st);
hipError_t launch_grouped16_sums(const GroupedSums<Product16>& a, int tile, int64_t parts, hipStream_t st);
// Both products of a small gradient and its bias in one launch: `tile` of the rows 128 or 32, of the sums 128.
hipError_t launch_grouped16_both(const GroupedSums<Product16>& w, int64_t w_blocks, const GroupedRows<Product16>& x, int tile, int64_t x_blocks, const GroupedGrad& b,
                                 int64_t b_blocks, hipStream_t st);

}  // namespace ilargi
#endif
