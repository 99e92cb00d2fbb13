// Products over ragged groups of rows on the 16-bit matrix cores: the blocks of mm16_block.h, each of one group.
#include "mm16_block.h"

#include "grouped.h"

namespace ilargi {

namespace {

// blockIdx: block (from `first` on), none, share of k.  Q: a matrix for each group, its rows over k (QK) or its columns.
template <bool QK, int B, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64, 512 / (WM * WN * 64)) void grouped16_rows_kernel(GroupedRows<Product16> a, int first, int tn) {
  __shared__ __attribute__((aligned(1024))) char lds[mm16_lds<false, QK, B, B, WM, WN>()];
  grouped_rows_block<2>(a, first + blockIdx.x, tn, [&](Product16 b, int ti, int tj, float* to) {
    b.P.across = b.M;
    mm16_block<false, QK, B, B, WM, WN>(b, ti, tj, (int)blockIdx.z, (int)a.share, to, lds);
  });
}

// blockIdx: block of a part of a group's rows (from `first` on).
template <int B, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64, 512 / (WM * WN * 64)) void grouped16_sums_kernel(GroupedSums<Product16> a, int first, int tm, int tn) {
  __shared__ __attribute__((aligned(1024))) char lds[mm16_lds<true, true, B, B, WM, WN>()];
  grouped_sums_block<2>(a, first + blockIdx.x, tm, tn, [&](const Product16& b, int ti, int tj, float* to) {
    mm16_block<true, true, B, B, WM, WN>(b, ti, tj, 0, (int)((b.K + kBK - 1) / kBK), to, lds);
  });
}

}  // namespace

hipError_t launch_grouped16_rows(const GroupedRows<Product16>& a, int tile, int64_t tiles, int splits, hipStream_t st) {
  const int tn = (int)((a.p.N + tile - 1) / tile);
  return in_parts(tiles * tn, tile * 2, [&](int64_t first, unsigned blocks) {
    const dim3 grid(blocks, 1, (unsigned)splits);
    if (tile == 256) {
      if (a.p.Q.k_rows) grouped16_rows_kernel<true, 256, 2, 4><<<grid, 512, 0, st>>>(a, (int)first, tn);
      else grouped16_rows_kernel<false, 256, 2, 4><<<grid, 512, 0, st>>>(a, (int)first, tn);
    } else {
      if (a.p.Q.k_rows) grouped16_rows_kernel<true, 128, 2, 2><<<grid, 256, 0, st>>>(a, (int)first, tn);
      else grouped16_rows_kernel<false, 128, 2, 2><<<grid, 256, 0, st>>>(a, (int)first, tn);
    }
  });
}

hipError_t launch_grouped16_sums(const GroupedSums<Product16>& a, int tile, int64_t parts, hipStream_t st) {
  const int tm = (int)((a.p.M + tile - 1) / tile), tn = (int)((a.p.N + tile - 1) / tile);
  return in_parts(parts * tm * tn, tile * 2, [&](int64_t first, unsigned blocks) {
    if (tile == 256) grouped16_sums_kernel<256, 2, 4><<<blocks, 512, 0, st>>>(a, (int)first, tm, tn);
    else grouped16_sums_kernel<128, 2, 2><<<blocks, 256, 0, st>>>(a, (int)first, tm, tn);
  });
}

}  // namespace ilargi
