// Products over ragged groups of rows: where the groups lie, and the kernels' arguments (kernels_grouped.hip, kernels_grouped16.hip).
#ifndef ILARGI_GROUPED_H_
#define ILARGI_GROUPED_H_

#include "mm_epilogue.h"

namespace ilargi {

// What one launch works out of the offsets for all others.  A prefix p has p[q] <= u < p[q + 1] for the units u of place q.
struct GroupIndex {
  int* start;       // groups + 1: first rows, ascending, in [0, n]
  int* tiles;       // prefix of the blocks of rows of every group
  int* order;       // groups by their rows, the longest first (up to kMostSorted groups; else as they come)
  int* parts;       // prefix, in that order, of the parts of rows that the products over rows are split into, one at least of every group
  int* slots;       // prefix, in that order, of those of groups of several parts
  int* chunks;      // prefix of the chunks of rows of the column sums
};
constexpr int kMostSorted = 512;

// Products of the rows of every group with its own matrix.  P's rows and the result's are the groups'; Q's matrices are far_q elements apart.
template <class Prod>
struct GroupedRows {
  Prod p;                     // M = n
  GroupIndex at;
  int groups;
  int64_t far_q, far_bias;    // elements
  int64_t share;              // of k, in the block's units
  float* partial;             // shares of n x (N to a multiple of 4) where k is split
};
// Products over the rows of every group: P and Q are n rows over k, C a matrix a group.
template <class Prod>
struct GroupedSums {
  Prod p;                     // K = n
  GroupIndex at;
  int groups;
  int64_t far_out;
  int part;                   // rows
  float* partial;             // M x (N to a multiple of 4) a slot
};

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

// run(product, block of rows, block of columns, sums_to) for block `id` of a launch of rows, `tn` blocks of columns.
template <int SIZE, class Prod, class F>
__device__ __forceinline__ void grouped_rows_block(const GroupedRows<Prod>& a, int id, int tn, F run) {
  const int tm = a.at.tiles[a.groups];
  if (id >= tm * tn) return;
  int u, tj;
  block_of(id, tm, tn, &u, &tj);
  const int g = place_of(a.at.tiles, a.groups, u);
  const int64_t r0 = a.at.start[g], rows = a.at.start[g + 1] - r0;
  float* to = a.partial != nullptr ? a.partial + ((int64_t)blockIdx.z * a.p.M + r0) * ((a.p.N + 3) / 4 * 4) : nullptr;
  run(rows_of(a, g, r0, rows, SIZE), u - a.at.tiles[g], tj, to);
}
template <int SIZE, class Prod, class F>
__device__ __forceinline__ void grouped_sums_block(const GroupedSums<Prod>& a, int id, int tm, int tn, F run) {
  const int u = id / (tm * tn);
  if (u >= a.at.parts[a.groups]) return;
  int ti, tj;
  block_of(id - u * (tm * tn), tm, tn, &ti, &tj);
  const int q = place_of(a.at.parts, a.groups, u), g = a.at.order[q], c = u - a.at.parts[q];
  const int64_t r0 = a.at.start[g] + (int64_t)c * a.part, end = a.at.start[g + 1], rows = end - r0 < a.part ? end - r0 : a.part;
  if (rows == 0 && a.p.epi.src != nullptr) return;         // nothing to add
  float* to = a.at.parts[q + 1] - a.at.parts[q] > 1 ? a.partial + (int64_t)(a.at.slots[q] + c) * a.p.M * ((a.p.N + 3) / 4 * 4) : nullptr;
  run(sums_of(a, g, r0, rows, SIZE), ti, tj, to);
}

hipError_t launch_grouped16_rows(const GroupedRows<Product16>& a, int tile, int64_t tiles, int splits, hipStream_t st);
hipError_t launch_grouped16_sums(const GroupedSums<Product16>& a, int tile, int64_t parts, hipStream_t st);

}  // namespace ilargi
#endif
