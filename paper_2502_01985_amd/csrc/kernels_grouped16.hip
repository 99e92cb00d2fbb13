// Products over ragged groups of rows on the 16-bit matrix cores: the blocks of mm16_block.h, each of one group.
//
// Groups of equal size take as long as one layer of all rows (16384 x 2048 x 4096, gelu and z kept: 287 us both; the product without them
// 235, the library's 232).  Skewed ones pay for the blocks that their ends leave part empty and for the last round: 1088 blocks for 1024
// 327 us.  Bound by the matrix cores; the epilogue, 50 us of it, is not hidden, as one workgroup of 256 x 256 fills a compute unit (blocks of 128,
// two to a unit: 386 us).
#include "mm16_block.h"

#include "grouped.h"

namespace ilargi {

namespace {

// Block `id` of 128.  Q: a matrix for each group, its rows over k (QK) or its columns.
template <bool QK>
__device__ __forceinline__ void rows128_block(const GroupedRows<Product16>& a, int id, int tn, char* lds) {
  constexpr int B = 128;
  const Blocks blocks(a.at, a.at.tiles, B);
  if (id >= blocks.total * tn) return;
  grouped_rows_block<2>(a, blocks, id, tn, [&](Product16 b, int ti, int tj, int64_t row) {
    b.P.across = b.M;
    mm16_block<false, QK, B, B, 2, 2>(b, ti, tj, (int)blockIdx.z, (int)a.share, sums_of_rows(a, row), lds);
  });
}
// blockIdx: block (from `first` on), none, share of k.
template <bool QK>
__global__ __launch_bounds__(256, 2) void grouped16_rows_kernel(GroupedRows<Product16> a, int first, int tn) {
  __shared__ __attribute__((aligned(1024))) char lds[mm16_lds<false, QK, 128, 128, 2, 2>()];
  rows128_block<QK>(a, first + blockIdx.x, tn, lds);
}

// A block of 256 as a product of its own.
__device__ __forceinline__ Product16 block_alone(const Product16& b, int ti, int tj) {
  Product16 c = b;
  const int64_t i = (int64_t)ti * 256, j = (int64_t)tj * 256;
  shift_operand(&c.P, i);
  shift_operand(&c.Q, j);
  c.M = b.M - i < 256 ? b.M - i : 256;
  c.N = b.N - j < 256 ? b.N - j : 256;
  return c;
}

// blockIdx: block of 256, or a share of one of the last round (from `first` on).  (544 blocks of 64 steps: 327 us where the last 32 take a
// round of their own, 260 in shares of eight steps and 17 for their sums.)
template <bool QK>
__global__ __launch_bounds__(512, 1) void grouped16_rounds_kernel(GroupedRows<Product16> a, int first, int tn) {
  constexpr int B = 256;
  __shared__ __attribute__((aligned(1024))) char lds[mm16_lds<false, QK, B, B, 2, 4>()];
  const Blocks blocks(a.at, a.at.tiles, B);
  const int steps = (int)((a.p.K + kBK - 1) / kBK), id = first + blockIdx.x;
  const Tail tail = tail_of(blocks.total * tn, steps);
  const int over = id - tail.full, block = over < 0 ? id : tail.full + over / tail.shares;
  if (block >= tail.full + tail.rest) return;
  grouped_rows_block<2>(a, blocks, block, tn, [&](Product16 b, int ti, int tj, int64_t) {
    b.P.across = b.M;
    int z = 0, share = steps;
    float* to = nullptr;
    if (over >= 0 && tail.shares > 1) {
      b = block_alone(b, ti, tj);
      ti = tj = 0;
      z = over % tail.shares;
      share = tail.share;
      to = a.partial + (int64_t)over * (B * B);
    }
    mm16_block<false, QK, B, B, 2, 4>(b, ti, tj, z, share, to, lds);
  });
}

// The shares of the last round's blocks, four sums of a row a thread and kTailRows rows of a block a workgroup.  blockIdx: rows, block.
constexpr int kTailRows = 8;
__global__ __launch_bounds__(256) void grouped16_tail_kernel(GroupedRows<Product16> a, int tn) {
  constexpr int B = 256;
  const Blocks blocks(a.at, a.at.tiles, B);
  const Tail tail = tail_of(blocks.total * tn, (int)((a.p.K + kBK - 1) / kBK));
  if (tail.shares < 2 || (int)blockIdx.y >= tail.rest) return;
  grouped_rows_block<2>(a, blocks, tail.full + blockIdx.y, tn, [&](const Product16& b, int ti, int tj, int64_t) {
    const Product16 c = block_alone(b, ti, tj);
    const int64_t j = threadIdx.x % 64 * 4, ldp = (c.N + 3) / 4 * 4, col = (int64_t)tj * B + j;
    float bias[4];
    epilogue_bias(b.epi, col, (int)(c.N - j < 4 ? c.N - j : 4), bias);
#pragma unroll
    for (int t = 0; t < kTailRows; t += 4) {
      const int64_t i = blockIdx.x * kTailRows + t + threadIdx.x / 64, row = (int64_t)ti * B + i;
      const int valid = quad_valid(i, j, c.M, c.N);
      if (valid == 0) continue;
      const SrcQuad raw = epilogue_ask(b.epi, 0, row, col, valid);
      const float* p = a.partial + (int64_t)blockIdx.y * tail.shares * (B * B) + i * ldp + j;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
      for (int z = 0; z < tail.shares; ++z) {
        const f32x4 s = *reinterpret_cast<const f32x4*>(p + (int64_t)z * (B * B));
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += s[q];
      }
      epilogue4(b.epi, 1.0f, 0, row, col, valid, bias, raw, v);
    }
  });
}

// The same where groups have few rows: what counts is the bytes of the matrices, and so how many of them are on their way.  A workgroup
// forms 32 rows by 64 columns, its steps of 64 k fetched kFewStages - 1 ahead; each wavefront has 16 of the columns.  8 rows, 16 groups of
// 2048 x 2048: 13 us, 4.2 TB/s of 54 MB, in one launch; in blocks of 128 with shares of k 22 in three.  Shares for two workgroups a compute unit
// instead of one: 17.6 with the launch that adds them; eight stages: the same.
constexpr int kFewRows = 32, kFewCols = 64, kFewStages = 6, kFewLds = kFewStages * (kFewRows + kFewCols) * kBK * 2;
template <bool QK>
__device__ __forceinline__ void few_block(const GroupedRows<Product16>& a, int id, int tn, char* lds_all) {
  constexpr int NT = 256, FM = kFewRows / 16;
  using TileP = Tile<false, kFewRows, NT>;
  using TileQ = Tile<QK, kFewCols, NT>;
  constexpr int kStage = TileP::kBytes + TileQ::kBytes, kEach = TileP::kLoads + TileQ::kLoads;
  static_assert(kFewStages * kStage == kFewLds, "the stages fill it");
  const Blocks blocks(a.at, a.at.tiles, kFewRows);
  if (id >= blocks.total * tn) return;
  grouped_rows_block<2>(a, blocks, id, tn, [&](const Product16& b, int ti, int tj, int64_t row) {
    float* const to = sums_of_rows(a, row);
    const int64_t i0 = (int64_t)ti * kFewRows, j0 = (int64_t)tj * kFewCols;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t step_q = QK ? kBK * b.Q.ld * 2 : kBK * 2;
    const int first = (int)(blockIdx.z * a.share), all = (int)((b.K + kBK - 1) / kBK), steps = all - first < a.share ? all - first : (int)a.share;
    const char* P = (const char*)b.P.p + 2 * i0 * b.P.ld + (int64_t)first * kBK * 2;
    const char* Q = (const char*)b.Q.p + 2 * (QK ? j0 : j0 * b.Q.ld) + first * step_q;
    TileP tp;
    TileQ tq;
    tp.plan(b.P.ld, b.M - i0);
    tq.plan(b.Q.ld, b.Q.across - j0);
    Fragments<false, kFewRows, FM> fp;
    Fragments<QK, kFewCols, 1> fq;
    fp.plan(0);
    fq.plan(16 * wave);
    const uint32_t base = lds_address(lds_all);
    auto fetch = [&](int t, int stage) {
      const char *p = P + (int64_t)t * kBK * 2, *q = Q + t * step_q;
      const int64_t left = b.K - (int64_t)(first + t) * kBK;
      const uint32_t at = base + stage * kStage;
      if (left >= kBK) {
        tp.template fetch_some<0, TileP::kLoads>(p, at);
        tq.template fetch_some<0, TileQ::kLoads>(q, at + TileP::kBytes);
      } else {
        tp.fetch_last(p, at, (int)left);
        tq.fetch_last(q, at + TileP::kBytes, (int)left);
      }
    };
    f32x4 acc[FM];
#pragma unroll
    for (int x = 0; x < FM; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int t = 0; t < kFewStages - 1 && t < steps; ++t) fetch(t, t);
    int stage = 0;
    for (int t = 0; t < steps; ++t) {
      // step t is in LDS, and everyone has done with the one before, whose place the next fetch takes
      if (t + kFewStages - 1 <= steps) arrived_and_together<kEach*(kFewStages - 2)>();
      else arrived_and_together<0>();
      const uint32_t here = base + stage * kStage;
      if (t + kFewStages - 1 < steps) fetch(t + kFewStages - 1, stage == 0 ? kFewStages - 1 : stage - 1);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const s16x8 q = fq.read(here + TileP::kBytes, half, 0);
#pragma unroll
        for (int x = 0; x < FM; ++x) acc[x] = mfma16<kMm16Bf16>(q, fp.read(here, half, x), acc[x]);
      }
      stage = stage + 1 == kFewStages ? 0 : stage + 1;
    }
    const int64_t j = j0 + 16 * wave + (lane >> 4) * 4;
    float bias[4];
    epilogue_bias(b.epi, j, (int)(b.N - j < 4 ? b.N - j : 4), bias);
#pragma unroll
    for (int x = 0; x < FM; ++x) {
      const int64_t i = i0 + 16 * x + (lane & 15);
      const int valid = quad_valid(i, j, b.M, b.N);
      if (valid == 0) continue;
      if (to != nullptr) {
        *reinterpret_cast<f32x4*>(to + i * ((b.N + 3) / 4 * 4) + j) = acc[x];
        continue;
      }
      float v[4] = {acc[x][0], acc[x][1], acc[x][2], acc[x][3]};
      epilogue4(b.epi, 1.0f, 0, i, j, valid, bias, epilogue_ask(b.epi, 0, i, j, valid), v);
    }
  });
}

template <bool QK>
__global__ __launch_bounds__(256, 2) void grouped16_few_kernel(GroupedRows<Product16> a, int first, int tn) {
  __shared__ __attribute__((aligned(1024))) char lds[kFewLds];
  few_block<QK>(a, first + blockIdx.x, tn, lds);
}

// blockIdx: block of a part of a group's rows (from `first` on).
template <int B, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64, 512 / (WM * WN * 64)) void grouped16_sums_kernel(GroupedSums<Product16> a, int first, int tm, int tn) {
  __shared__ __attribute__((aligned(1024))) char lds[mm16_lds<true, true, B, B, WM, WN>()];
  grouped_sums_block<2>(a, first + blockIdx.x, B, tm, tn, [&](const Product16& b, int ti, int tj, float* to) {
    mm16_block<true, true, B, B, WM, WN>(b, ti, tj, 0, (int)((b.K + kBK - 1) / kBK), to, lds);
  });
}

// Both products of a small gradient and its bias: `sums` blocks of d_W, `rows` of d_X (FEW: of few rows), and those of the bias.  2102 rows in 4
// groups, 64 x 512: 24 us in all for 36 in launches of their own; 4000 in 8, 1024 x 1024: 68 for 79.
template <bool FEW>
__global__ __launch_bounds__(256, 2) void grouped16_both_kernel(GroupedSums<Product16> w, int sums, int tm, int tn, GroupedRows<Product16> x, int rows, int tn_x, GroupedGrad b, int columns) {
  constexpr int kSumsLds = mm16_lds<true, true, 128, 128, 2, 2>(), kRowsLds = FEW ? kFewLds : mm16_lds<false, false, 128, 128, 2, 2>();
  __shared__ __attribute__((aligned(1024))) char lds[kSumsLds > kRowsLds ? kSumsLds : kRowsLds];
  static_assert(sizeof(BiasLds) <= sizeof(lds), "the column sums fit too");
  const int id = blockIdx.x;
  if (id < sums) {
    grouped_sums_block<2>(w, id, 128, tm, tn, [&](const Product16& p, int ti, int tj, float* to) {
      mm16_block<true, true, 128, 128, 2, 2>(p, ti, tj, 0, (int)((p.K + kBK - 1) / kBK), to, lds);
    });
  } else if (id - sums < rows) {
    if constexpr (FEW) few_block<false>(x, id - sums, tn_x, lds);
    else rows128_block<false>(x, id - sums, tn_x, lds);
  } else {
    bias_block<bf16_t>(b, (id - sums - rows) % columns, (id - sums - rows) / columns, *reinterpret_cast<BiasLds*>(lds));
  }
}

}  // namespace

hipError_t launch_grouped16_rows(const GroupedRows<Product16>& a, int tile, int64_t tiles, int splits, hipStream_t st) {
  if (tile == kFewRows) {
    const int tn = (int)((a.p.N + kFewCols - 1) / kFewCols);
    return in_parts(tiles * tn, 256, [&](int64_t first, unsigned blocks) {
      const dim3 grid(blocks, 1, (unsigned)splits);
      if (a.p.Q.k_rows) grouped16_few_kernel<true><<<grid, 256, 0, st>>>(a, (int)first, tn);
      else grouped16_few_kernel<false><<<grid, 256, 0, st>>>(a, (int)first, tn);
    });
  }
  const int tn = (int)((a.p.N + tile - 1) / tile);
  if (tile == 128)
    return in_parts(tiles * tn, 256, [&](int64_t first, unsigned blocks) {
      const dim3 grid(blocks, 1, (unsigned)splits);
      if (a.p.Q.k_rows) grouped16_rows_kernel<true><<<grid, 256, 0, st>>>(a, (int)first, tn);
      else grouped16_rows_kernel<false><<<grid, 256, 0, st>>>(a, (int)first, tn);
    });
  // (a last round of less than half has at most kUnits shares)
  const hipError_t e = in_parts(tiles * tn + kUnits, 512, [&](int64_t first, unsigned blocks) {
    if (a.p.Q.k_rows) grouped16_rounds_kernel<true><<<blocks, 512, 0, st>>>(a, (int)first, tn);
    else grouped16_rounds_kernel<false><<<blocks, 512, 0, st>>>(a, (int)first, tn);
  });
  if (e != hipSuccess || (a.p.K + kBK - 1) / kBK < 8) return e;       // (shares have four steps at least)
  grouped16_tail_kernel<<<dim3(256 / kTailRows, kUnits / 2), 256, 0, st>>>(a, tn);
  return hipGetLastError();
}

hipError_t launch_grouped16_sums(const GroupedSums<Product16>& a, int tile, int64_t parts, hipStream_t st) {
  const int tm = (int)((a.p.M + tile - 1) / tile), tn = (int)((a.p.N + tile - 1) / tile);
  return in_parts(parts * tm * tn, tile * 2, [&](int64_t first, unsigned blocks) {
    if (tile == 256) grouped16_sums_kernel<256, 2, 4><<<blocks, 512, 0, st>>>(a, (int)first, tm, tn);
    else grouped16_sums_kernel<128, 2, 2><<<blocks, 256, 0, st>>>(a, (int)first, tm, tn);
  });
}

hipError_t launch_grouped16_both(const GroupedSums<Product16>& w, int64_t w_blocks, const GroupedRows<Product16>& x, int tile, int64_t x_blocks, const GroupedGrad& b,
                                 int64_t b_blocks, hipStream_t st) {
  const int tm = (int)((w.p.M + 127) / 128), tn = (int)((w.p.N + 127) / 128), cols = tile == kFewRows ? kFewCols : 128, tn_x = (int)((x.p.N + cols - 1) / cols);
  const int columns = (int)((b.g.m + 15) / 16);
  const unsigned all = (unsigned)(w_blocks + x_blocks + b_blocks);
  if (tile == kFewRows) grouped16_both_kernel<true><<<all, 256, 0, st>>>(w, (int)w_blocks, tm, tn, x, (int)x_blocks, tn_x, b, columns);
  else grouped16_both_kernel<false><<<all, 256, 0, st>>>(w, (int)w_blocks, tm, tn, x, (int)x_blocks, tn_x, b, columns);
  return hipGetLastError();
}

}  // namespace ilargi
