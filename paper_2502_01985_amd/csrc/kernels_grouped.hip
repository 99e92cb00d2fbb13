// Layers by group of rows: the index of the groups, products in float32, the elementwise pass of the gradient, the sums of parts, and
// what runs where.
#include "grouped.h"
#include "mm_f32_block.h"

namespace ilargi {

namespace {

// --------------------------------------------------------------------------------------------------- the index of the groups
constexpr int kIndexThreads = 1024;

struct Scan {
  int wave[kIndexThreads / kWave];
};
// The sum (or the largest) of the values of this thread and those before it, and that of all threads.
template <bool MOST>
__device__ __forceinline__ int scan_of(int v, Scan& lds, int* all) {
  auto both = [](int x, int y) { return MOST ? (x > y ? x : y) : x + y; };
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
  for (int s = 1; s < kWave; s *= 2) {
    const int o = __shfl_up(v, s);
    if (lane >= s) v = both(v, o);
  }
  __syncthreads();
  if (lane == kWave - 1) lds.wave[wave] = v;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < kIndexThreads / kWave; ++w) {
    if (w < wave) before = both(before, lds.wave[w]);
    total = both(total, lds.wave[w]);
  }
  *all = total;
  return both(before, v);
}

// units(q): of place q; writes their prefix of n + 1 places.
template <class F>
__device__ __forceinline__ void write_prefix(int* __restrict__ to, int n, Scan& lds, F units) {
  int before = 0;
  for (int q0 = 0; q0 < n; q0 += kIndexThreads) {
    const int q = q0 + threadIdx.x, v = q < n ? units(q) : 0;
    int all;
    const int upto = scan_of<false>(v, lds, &all);
    if (q < n) to[q] = before + upto - v;
    before += all;
  }
  if (threadIdx.x == 0) to[n] = before;
}

// One workgroup.  tile, part, chunk: rows of a block, a part, a chunk; 0 where the call has no use for them.
__global__ __launch_bounds__(kIndexThreads) void group_index_kernel(GroupIndex at, int tile, int part, int chunk) {
  const int groups = at.groups, n = at.n;
  __shared__ Scan lds;
  __shared__ int sizes[kMostSorted];
  int most = 0;                                // the largest offset so far: a later one below it counts as that
  for (int q0 = 0; q0 <= groups; q0 += kIndexThreads) {
    const int q = q0 + threadIdx.x;
    int v = q <= groups ? at.offsets[q] : 0;
    v = v < 0 ? 0 : v > n ? n : v;
    int all;
    v = scan_of<true>(v, lds, &all);
    if (q <= groups) at.start[q] = v > most ? v : most;
    most = all > most ? all : most;
  }
  __syncthreads();
  auto rows = [&](int g) { return at.start[g + 1] - at.start[g]; };
  auto blocks = [&](int g, int size) { return (int)(((int64_t)rows(g) + size - 1) / size); };
  if (tile > 0) write_prefix(at.tiles, groups, lds, [&](int g) { return blocks(g, tile); });
  if (chunk > 0) write_prefix(at.chunks, groups, lds, [&](int g) { return blocks(g, chunk); });
  if (part == 0) return;
  if (groups <= kMostSorted) {
    const int g = threadIdx.x, mine = g < groups ? rows(g) : 0;
    if (g < groups) sizes[g] = mine;
    __syncthreads();
    if (g < groups) {
      int place = 0;
      for (int o = 0; o < groups; ++o) place += sizes[o] > mine || (sizes[o] == mine && o < g);
      at.order[place] = g;
    }
  } else {
    for (int g = threadIdx.x; g < groups; g += kIndexThreads) at.order[g] = g;
  }
  __syncthreads();
  auto parts = [&](int q) { const int b = blocks(at.order[q], part); return b > 1 ? b : 1; };
  write_prefix(at.parts, groups, lds, parts);
  write_prefix(at.slots, groups, lds, [&](int q) { const int b = parts(q); return b > 1 ? b : 0; });
}

// --------------------------------------------------------------------------------------------------------- float32 products
// As in kernels_mm.hip, bound by the starts and ends of short products: 10,000 rows in 64 groups, 220 x 256: 24 us (46 TFLOP/s).  Fetching
// two steps ahead instead of one changed nothing there and cost large products 9 %.
template <class T, bool QK, int TILE, int STEP>
__device__ __forceinline__ void rows_block(const GroupedRows<Product>& a, int id, int tn, MmF32Lds<TILE, STEP>& lds) {
  const Blocks blocks(a.at, a.at.tiles, TILE);
  if (id >= blocks.total * tn) return;
  grouped_rows_block<sizeof(T)>(a, blocks, id, tn, [&](const Product& b, int ti, int tj, int64_t row) {
    mm_f32_block<T, T, false, QK, TILE, STEP>(b, ti, tj, 0, blockIdx.z, a.share, sums_of_rows(a, row), lds);
  });
}
template <class T, int TILE, int STEP>
__device__ __forceinline__ void sums_block(const GroupedSums<Product>& a, int id, int tm, int tn, MmF32Lds<TILE, STEP>& lds) {
  grouped_sums_block<sizeof(T)>(a, id, TILE, tm, tn, [&](const Product& b, int ti, int tj, float* to) {
    mm_f32_block<T, T, true, true, TILE, STEP>(b, ti, tj, 0, 0, b.K, to, lds);
  });
}

// blockIdx: block (from `first` on), none, share of k.
template <class T, bool QK, int TILE, int STEP>
__global__ __launch_bounds__(256) void grouped_rows_kernel(GroupedRows<Product> a, int first, int tn) {
  __shared__ __attribute__((aligned(16))) MmF32Lds<TILE, STEP> lds;
  rows_block<T, QK, TILE, STEP>(a, first + blockIdx.x, tn, lds);
}

template <class T, int TILE, int STEP>
__global__ __launch_bounds__(256) void grouped_sums_kernel(GroupedSums<Product> a, int first, int tm, int tn) {
  __shared__ __attribute__((aligned(16))) MmF32Lds<TILE, STEP> lds;
  sums_block<T, TILE, STEP>(a, first + blockIdx.x, tm, tn, lds);
}

template <class T>
hipError_t rows_f32(const GroupedRows<Product>& a, int tile, int64_t tiles, int splits, hipStream_t st) {
  const int tn = (int)((a.p.N + tile - 1) / tile);
  return in_parts(tiles * tn, 256, [&](int64_t first, unsigned blocks) {
    const dim3 grid(blocks, 1, (unsigned)splits);
    if (tile == 64) {
      if (a.p.Q.k_rows) grouped_rows_kernel<T, true, 64, 32><<<grid, 256, 0, st>>>(a, (int)first, tn);
      else grouped_rows_kernel<T, false, 64, 32><<<grid, 256, 0, st>>>(a, (int)first, tn);
    } else {
      if (a.p.Q.k_rows) grouped_rows_kernel<T, true, 128, 16><<<grid, 256, 0, st>>>(a, (int)first, tn);
      else grouped_rows_kernel<T, false, 128, 16><<<grid, 256, 0, st>>>(a, (int)first, tn);
    }
  });
}
template <class T>
hipError_t sums_f32(const GroupedSums<Product>& a, int tile, int64_t parts, hipStream_t st) {
  const int tm = (int)((a.p.M + tile - 1) / tile), tn = (int)((a.p.N + tile - 1) / tile);
  return in_parts(parts * tm * tn, 256, [&](int64_t first, unsigned blocks) {
    if (tile == 64) grouped_sums_kernel<T, 64, 32><<<blocks, 256, 0, st>>>(a, (int)first, tm, tn);
    else grouped_sums_kernel<T, 128, 16><<<blocks, 256, 0, st>>>(a, (int)first, tm, tn);
  });
}

// ------------------------------------------------------------------------------------------------------------ sums of parts
// Adds the shares of k and finishes, a thread for four sums of a row (from workgroup `first` on); rows of no group are left alone.
__global__ __launch_bounds__(256) void grouped_rows_join_kernel(Epilogue epi, int64_t N, GroupIndex at, int64_t far_bias, int64_t first, int splits, const float* __restrict__ partial) {
  const int64_t quads = (N + 3) / 4, e = (first + blockIdx.x) * 256 + threadIdx.x, i = e / quads, j = (e - i * quads) * 4;
  int lo = 0, hi = at.groups;                    // start[lo] <= i < start[hi]
  bool is;
  if (in_lanes(at)) {
    const Lanes l(at);
    is = i >= lane_value(l.start, 0) && i < lane_value(l.end, at.groups - 1);
    for (int s = kWave / 2; s > 0; s /= 2) {
      const int mid = lo + s, from = __shfl(l.start, mid);       // (lo is below 64 - s)
      if (mid < at.groups && from <= i) lo = mid;
    }
  } else {
    is = i >= at.start[0] && i < at.start[at.groups];
    while (is && hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (at.start[mid] <= i) lo = mid;
      else hi = mid;
    }
  }
  if (!is) return;
  move_to(epi.bias, lo * far_bias, epi.out_bf16 ? 2 : 4);
  const int valid = N - j < 4 ? (int)(N - j) : 4;
  const SrcQuad raw = epilogue_ask(epi, 0, i, j, valid);
  float bias[4];
  epilogue_bias(epi, j, valid, bias);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int z = 0; z < splits; ++z) {
    const float4 t = *reinterpret_cast<const float4*>(partial + ((int64_t)z * at.n + i) * quads * 4 + j);
    v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
  }
  epilogue4(epi, 1.0f, 0, i, j, valid, bias, raw, v);
}

// blockIdx: four sums a thread (from workgroup `first` on), place of the group.
__global__ __launch_bounds__(256) void grouped_sums_join_kernel(Epilogue epi, int64_t M, int64_t N, GroupIndex at, int part, int64_t far_out, int64_t first, const float* __restrict__ partial) {
  const Parts::Place q = Parts(at, part).place(blockIdx.y, 0);
  const int parts = q.parts, size = epi.out_bf16 ? 2 : 4;
  const int64_t quads = (N + 3) / 4, e = (first + blockIdx.x) * 256 + threadIdx.x, i = e / quads, j = (e - i * quads) * 4;
  if (parts < 2 || i >= M) return;
  move_to(epi.src, q.group * far_out, size);
  move_to(epi.out, q.group * far_out, size);
  const int valid = N - j < 4 ? (int)(N - j) : 4;
  const SrcQuad raw = epilogue_ask(epi, 0, i, j, valid);
  const float* p = partial + ((int64_t)q.slot * M + i) * quads * 4 + j;
  const float none[4] = {0.f, 0.f, 0.f, 0.f};
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int c = 0; c < parts; ++c) {
    const float4 t = *reinterpret_cast<const float4*>(p + c * M * quads * 4);
    v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
  }
  epilogue4(epi, 1.0f, 0, i, j, valid, none, raw, v);
}

// ------------------------------------------------------------------------------------- the elementwise pass of the gradient
// g = d_out f'(pre) of a chunk of a group's rows, and the column sums of the unrounded g.  g is rounded to the layer's type: in bfloat16 the products then
// run on the 16-bit matrix cores, and are off by 2.3e-3 of themselves where a g in float32 would leave the 1.7e-3 of rounding them alone.  As layer_grad_kernel, with
// chunks that end where groups do, 16 bytes a lane and kTurns rows of a lane on their way.  16384 x 4096, bfloat16, gelu: 90 us for 403 MB
// (4.5 TB/s), 126 with 8 bytes a lane and two rows.  blockIdx: kGradCols columns (from `first` on),
// chunk.
constexpr int kGradCols = 128, kTurns = 4;
template <class T>
__global__ __launch_bounds__(256) void grouped_grad_kernel(GroupedGrad a, int64_t first, int first_chunk) {
  constexpr int V = ElemOf<T>::kVec, kLanes = kGradCols / V, kRows = 256 / kLanes;
  using Raw = Piece<T, V>;
  __shared__ float part[kRows][kGradCols];
  const int u = first_chunk + blockIdx.y;
  const Blocks chunks(a.at, a.at.chunks, a.chunk);
  if (u >= chunks.total) return;
  const LayerGradArgs& y = a.g;
  const Unit b = chunks.find(u);
  const int cl = threadIdx.x % kLanes, rl = threadIdx.x / kLanes;
  const int64_t j = ((first + blockIdx.x) * kLanes + cl) * V;
  const int64_t r0 = b.first + (int64_t)b.number * a.chunk, end = (int64_t)b.first + b.rows, r1 = end - r0 < a.chunk ? end : r0 + a.chunk;
  const int valid = (int)(y.m - j < 0 ? 0 : y.m - j < V ? y.m - j : V);
  const bool stored = y.dz != nullptr && j < y.ld_dz, bent = y.act != ILARGI_ACT_NONE;
  float s[V];
#pragma unroll
  for (int q = 0; q < V; ++q) s[q] = 0.0f;
  auto finish = [&](int64_t i, const Raw& d, const Raw& z) {
    float f[V];
#pragma unroll
    for (int q = 0; q < V; ++q) {
      f[q] = (float)d.v[q];
      if (bent) f[q] *= act_slope((float)z.v[q], y.act);
      s[q] += f[q];
    }
    // (rows of dz are whole pieces of eight, with zeros behind their end)
    if (stored) store_piece<T, V>((T*)y.dz + i * y.ld_dz + j, V, f);
  };
  if (valid == V) {
    for (int64_t i0 = r0 + rl; i0 < r1; i0 += kRows * kTurns) {
      Raw d[kTurns], z[kTurns];
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        const int64_t i = i0 + t * kRows < r1 ? i0 + t * kRows : r1 - 1;
        d[t] = *reinterpret_cast<const Raw*>((const T*)y.d_out + i * y.ld_out + j);
        if (bent) z[t] = *reinterpret_cast<const Raw*>((const T*)y.pre + i * y.ld_pre + j);
      }
#pragma unroll
      for (int t = 0; t < kTurns; ++t)
        if (i0 + t * kRows < r1) finish(i0 + t * kRows, d[t], z[t]);
    }
  } else if (valid > 0 || stored) {
    for (int64_t i = r0 + rl; i < r1; i += kRows) {
      Raw d, z;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        d.v[q] = q < valid ? ((const T*)y.d_out)[i * y.ld_out + j + q] : (T)0.0f;
        z.v[q] = bent && q < valid ? ((const T*)y.pre)[i * y.ld_pre + j + q] : (T)0.0f;
      }
      finish(i, d, z);
    }
  }
  if (a.partial == nullptr) return;
#pragma unroll
  for (int q = 0; q < V; ++q) part[rl][cl * V + q] = s[q];
  __syncthreads();
  const int64_t c = (first + blockIdx.x) * kGradCols + threadIdx.x;
  if (threadIdx.x >= kGradCols || c >= y.m) return;
  float t = part[0][threadIdx.x];
#pragma unroll
  for (int q = 1; q < kRows; ++q) t += part[q][threadIdx.x];
  a.partial[(int64_t)u * y.m + c] = t;
}

// blockIdx: 16 columns (from `first` on), group.
template <class T>
__global__ __launch_bounds__(256) void grouped_bias_kernel(GroupedGrad a, int64_t first) {
  __shared__ BiasLds lds;
  bias_block<T>(a, first + blockIdx.x, blockIdx.y, lds);
}

// Both products of a gradient and the bias's in one launch, where none of them fills the card for long: `sums` blocks of d_W, `rows`
// of d_X, and those of the column sums.  (5003 rows in 40 groups, 333 x 129: 50 us for 58 in three launches.)
template <class T>
__global__ __launch_bounds__(256) void grouped_both_kernel(GroupedSums<Product> w, int sums, int tm, int tn, GroupedRows<Product> x, int rows, int tn_x, GroupedGrad b, int columns) {
  __shared__ __attribute__((aligned(16))) union {
    MmF32Lds<64, 32> products;
    BiasLds bias;
  } lds;
  const int id = blockIdx.x;
  if (id < sums) sums_block<T, 64, 32>(w, id, tm, tn, lds.products);
  else if (id - sums < rows) rows_block<T, false, 64, 32>(x, id - sums, tn_x, lds.products);
  else bias_block<T>(b, (id - sums - rows) % columns, (id - sums - rows) / columns, lds.bias);
}

// Matrices of bfloat16 at any address, laid out in whole 16-byte pieces with zeros behind their rows' ends; 2^sh lanes a row.
__global__ __launch_bounds__(256) void pack_matrices_kernel(const bf16_t* __restrict__ src, int64_t ld, int64_t stride, int64_t rows, int64_t cols, int64_t all, int64_t first,
                                                            bf16_t* __restrict__ dst, int sh) {
  const int64_t r = ((first + blockIdx.x) * 256 + threadIdx.x) >> sh, ldp = (cols + 7) / 8 * 8;
  if (r >= all) return;
  const int64_t b = r / rows, from = b * stride + (r - b * rows) * ld;
  for (int64_t c = (int64_t)(threadIdx.x & ((1 << sh) - 1)) * 8; c < cols; c += 8ll << sh) {
    const bf16_t* p = src + from + c;
    Piece<bf16_t, 8> t;
    if (cols - c >= 8) {
      t = *reinterpret_cast<const Piece<bf16_t, 8>*>(p);
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) t.v[q] = q < cols - c ? p[q] : (bf16_t)0.0f;
    }
    *reinterpret_cast<uint4*>(dst + r * ldp + c) = __builtin_bit_cast(uint4, t);
  }
}

hipError_t pack_matrices(const void* src, int64_t ld, int64_t stride, int64_t batch, int64_t rows, int64_t cols, void* dst, hipStream_t st) {
  int sh = ilog2_ceil((cols + 7) / 8);
  if (sh > 6) sh = 6;
  return in_parts((((batch * rows) << sh) + 255) / 256, 256, [&](int64_t first, unsigned blocks) {
    pack_matrices_kernel<<<blocks, 256, 0, st>>>((const bf16_t*)src, ld, stride, rows, cols, batch * rows, first, (bf16_t*)dst, sh);
  });
}

// -------------------------------------------------------------------------------------------------------- what runs where
int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
int64_t up4(int64_t v) { return (v + 3) / 4 * 4; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }
int64_t blocks_in(int64_t v, int64_t size) { return (v + size - 1) / size; }
int64_t filled(const ilargi_groups_t& y) { return y.groups < y.n ? y.groups : y.n; }      // most groups that have rows

struct RowsPlan {
  int tile, splits;
  int64_t share, tiles;       // of k, in the block's units; blocks of rows at most
  size_t partial_bytes;
};
// Blocks and shares of k by what they cost in microseconds, as mm16_plan and mm_f32_plan count it; the groups are taken to be of equal size, as
// the host does not know better.  Where they are not, blocks of few rows read a long group's matrix once for every 32 rows of it: 2000 groups, 40,000 rows, 512 x
// 512, bfloat16: 250 us with 20 rows each, 285 with 30,005 in one of them (by themselves those take 31, the others 214); all in one, the most it can cost, 105 for 37.
RowsPlan rows_plan(const ilargi_groups_t& y, int64_t N, int64_t K, bool h) {
  RowsPlan best{};
  double least = 1e300;
  const double some = (double)filled(y), each = (double)y.n / (some > 0 ? some : 1.0);
  if (h && each <= 24.0) {
    const int64_t blocks = filled(y) * blocks_in(N, 64), steps = K > 64 ? blocks_in(K, 64) : 1;
    int64_t splits = blocks > 0 ? 256 / blocks : 1;
    if (splits > steps / 8) splits = steps / 8;
    if (splits < 1) splits = 1;
    const int64_t share = blocks_in(steps, splits);
    splits = blocks_in(steps, share);
    return {32, (int)splits, share, y.n / 32 + filled(y), splits > 1 ? (size_t)splits * (size_t)y.n * (size_t)up4(N) * 4 : 0};
  }
  for (int tile = h ? 256 : 128; tile >= (h ? 128 : 64); tile /= 2) {
    const double rows = some * (each > 0.5 * tile ? each / tile + 0.5 : 1.0), blocks = rows * (double)blocks_in(N, tile);
    const int64_t step = h ? 64 : tile == 64 ? 32 : 16, steps = K > step ? blocks_in(K, step) : 1;
    for (int64_t splits = 1; splits <= 64 && splits <= steps; ++splits) {
      const int64_t share = blocks_in(steps, splits);
      if (splits > 1 && (blocks_in(steps, share) != splits || blocks * (double)splits > 2048.0 || (h && share < 4))) continue;
      if (tile == 256 && splits > 1) continue;         // (they split what does not fill a round by themselves)
      const double groups = blocks * (double)splits, rounds = ceil(groups / 256.0);
      double cost;
      if (!h) {
        const double work = tile == 64 ? 0.47 : 0.8, alone = tile == 64 ? 0.8 : 1.1;
        cost = (double)share * (rounds * work > alone ? rounds * work : alone);
      } else if (tile == 256) {
        const Tail t = tail_of(groups < 1e9 ? (int)ceil(groups) : 0, (int)steps);
        cost = 1.7 * ((double)t.full / kUnits * (double)steps + (t.rest > 0 ? (double)t.share : 0.0)) + (t.shares > 1 ? 3.0 + 2.0 * t.rest * t.shares * 0.26 / 8.0 : 0.0);
      } else {
        cost = (double)share * (groups <= 256.0 ? 0.75 : 1.08 * ceil(groups / 512.0));
      }
      const double bytes = (double)splits * (double)y.n * (double)up4(N) * 4.0;
      if (splits > 1) cost += 3.0 + 2.0 * bytes / 8e6;
      if (cost < least) {
        least = cost;
        best = {tile, (int)splits, h ? share : share * step, y.n / tile + filled(y), splits > 1 ? (size_t)bytes : tile == 256 ? kTailBytes : 0};
      }
    }
  }
  return best;
}

struct SumsPlan {
  int tile, part;             // rows
  int64_t parts, several;     // most parts; most groups of several
  size_t partial_bytes;
};
// Long groups are split into parts of rows where the blocks of one matrix fill less than half of the card: then a group of most rows
// would run on while the rest of it is idle.  (40 skewed groups of 5003 rows, 333 x 129: parts for 128 / 256 / 512 / 1024 blocks 81 / 62 /
// 58 / 58 us in all.  8 groups of 16384 rows, 2048 x 4096, 128 blocks each: one part 712, two 724, four 777, eight 858: the longest
// first, they fill the card by themselves.)
SumsPlan sums_plan(const ilargi_groups_t& y, bool h) {
  SumsPlan p{};
  int tile = h ? 256 : 128;
  const int least = h ? 128 : 64;
  auto blocks = [&](int t) { return blocks_in(y.k, t) * blocks_in(y.m, t); };
  if (blocks(tile) * filled(y) < 512) tile = least;
  p.tile = tile;
  const int64_t aim = blocks(tile) < 128 ? 512 / blocks(tile) : 1;
  int64_t rows = aim > 1 ? blocks_in(y.n, aim) : y.n;
  rows = rows < 256 ? 256 : (rows + 63) / 64 * 64;
  p.part = (int)(rows < (1 << 30) ? rows : 1 << 30);
  p.parts = y.n / p.part + y.groups;
  p.several = y.n / (p.part + 1);
  if (p.several > y.groups) p.several = y.groups;
  // a group of several parts has more rows than one, and so at most twice as many parts as whole ones
  p.partial_bytes = p.several > 0 ? (size_t)(2 * (y.n / p.part)) * (size_t)y.k * (size_t)up4(y.m) * 4 : 0;
  return p;
}

int chunk_rows(const ilargi_groups_t& y) {
  int64_t rows = blocks_in(y.n * blocks_in(y.m, kGradCols), 2048);
  rows = rows < 32 ? 32 : (rows + 7) / 8 * 8;
  return (int)(rows < 65536 ? rows : 65536);
}
int64_t chunks_in(const ilargi_groups_t& y) { return y.n / chunk_rows(y) + filled(y); }

// bfloat16 operands with odd rows or addresses are laid out first where the 16-bit cores save more than the copies take: 100 TFLOP/s on
// the float32 cores against a pass over each operand at 4 TB/s and two launches.
bool worth_packing(const ilargi_groups_t& y) {
  const double ops = 2.0 * (double)y.n * (double)y.k * (double)y.m, bytes = 4.0 * ((double)y.groups * (double)y.k * (double)y.m + (double)y.n * (double)y.k);
  return y.type == ILARGI_TYPE_BF16 && ops / 1e14 > bytes / 4e12 + 1e-5;
}

struct GroupedLayout {
  size_t index, x, w, partial, forward;              // partial: shares of k
  size_t dz, chunks, shares, gradient;
};
GroupedLayout grouped_layout(const ilargi_groups_t& y) {
  GroupedLayout l{};
  const bool h = y.type == ILARGI_TYPE_BF16;
  auto most = [&](auto f) { const size_t a = f(false), b = h ? f(true) : 0; return up256(a > b ? a : b); };
  l.x = up256((size_t)(y.groups + 1) * 6 * 4);
  l.w = l.x + (worth_packing(y) ? up256(2 * (size_t)y.n * (size_t)up8(y.k)) : 0);
  l.partial = l.w + (worth_packing(y) ? up256(2 * (size_t)y.groups * (size_t)y.k * (size_t)up8(y.m)) : 0);
  l.forward = l.partial + most([&](bool b) { return rows_plan(y, y.m, y.k, b).partial_bytes; });
  l.dz = l.partial;
  l.chunks = l.dz + up256((size_t)y.n * (size_t)up8(y.m) * (h ? 2 : 4));
  l.shares = l.chunks + up256((size_t)chunks_in(y) * (size_t)y.m * 4);
  const size_t dx = most([&](bool b) { return rows_plan(y, y.k, y.m, b).partial_bytes; }), dw = most([&](bool b) { return sums_plan(y, b).partial_bytes; });
  l.gradient = l.shares + (dx > dw ? dx : dw);
  return l;
}
GroupIndex index_in(char* ws, const ilargi_groups_t& y, const int32_t* offsets) {
  int* p = (int*)ws;
  const int64_t far = y.groups + 1;
  return {offsets, (int)y.groups, (int)y.n, p, p + far, p + 2 * far, p + 3 * far, p + 4 * far, p + 5 * far};
}

hipError_t find_groups(const GroupIndex& at, int tile, int part, int chunk, hipStream_t st) {
  if (at.groups <= kMostInLanes) return hipSuccess;
  group_index_kernel<<<1, kIndexThreads, 0, st>>>(at, tile, part, chunk);
  return hipGetLastError();
}

// A matrix, or the matrices of all groups, as they lie or laid out in whole pieces (then with zeros behind their rows).
struct Held {
  const void* p;
  int64_t ld, rows, cols, stride;
  bool padded;
};
bool in_pieces(const Held& m) {
  return reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.ld % 8 == 0 && m.ld < (1 << 22) && m.stride % 8 == 0 && (m.padded || m.cols % 8 == 0);
}
hipError_t lay_out(const ilargi_groups_t& y, Held* m, int64_t batch, char* at, hipStream_t st) {
  if (!worth_packing(y) || in_pieces(*m)) return hipSuccess;
  const hipError_t e = pack_matrices(m->p, m->ld, m->stride, batch, m->rows, m->cols, at, st);
  *m = {at, up8(m->cols), m->rows, m->cols, m->rows * up8(m->cols), true};
  return e;
}

// out = P Q_g by group (Q's rows over k, or its columns).
template <class Prod>
GroupedRows<Prod> rows_of_layer(const ilargi_groups_t& y, int64_t N, int64_t K, const Epilogue& epi, int64_t far_q, int64_t far_bias, const GroupIndex& at, const RowsPlan& plan, float* partial) {
  GroupedRows<Prod> a{};
  a.p.M = y.n; a.p.N = N; a.p.K = K; a.p.batches = 1;
  a.p.epi = epi;
  a.at = at; a.far_q = far_q; a.far_bias = far_bias; a.share = plan.share;
  a.partial = plan.splits > 1 || plan.tile == 256 ? partial : nullptr;
  return a;
}
GroupedRows<Product> rows_in_f32(const ilargi_groups_t& y, const Held& P, const Held& Q, int q_rows, int64_t N, int64_t K, const Epilogue& epi, int64_t far_bias, const GroupIndex& at,
                                 const RowsPlan& plan, float* partial) {
  const int bf16 = y.type == ILARGI_TYPE_BF16;
  GroupedRows<Product> a = rows_of_layer<Product>(y, N, K, epi, Q.stride, far_bias, at, plan, partial);
  a.p.P = {P.p, P.ld, 0, bf16, 0};
  a.p.Q = {Q.p, Q.ld, q_rows, bf16, 0};
  return a;
}
GroupedRows<Product16> rows_in_16(const ilargi_groups_t& y, const Held& P, const Held& Q, int q_rows, int64_t N, int64_t K, const Epilogue& epi, int64_t far_bias, const GroupIndex& at,
                                  const RowsPlan& plan, float* partial) {
  GroupedRows<Product16> a = rows_of_layer<Product16>(y, N, K, epi, Q.stride, far_bias, at, plan, partial);
  a.p.P = {P.p, P.ld, 0, 0, 0, y.n};
  a.p.Q = {Q.p, Q.ld, q_rows, 0, 0, q_rows ? up8(Q.cols) : Q.rows};
  a.p.kind = kMm16Bf16;
  a.p.past = plan.splits == 1 && (epi.pre != nullptr ? 4 : 2) * y.n * N >= kStreamBytes;
  return a;
}
hipError_t rows_product(const ilargi_groups_t& y, const Held& P, const Held& Q, int q_rows, int64_t N, int64_t K, const Epilogue& epi, int64_t far_bias, const GroupIndex& at,
                        const RowsPlan& plan, bool h16, float* partial, hipStream_t st) {
  hipError_t e;
  if (h16) {
    e = launch_grouped16_rows(rows_in_16(y, P, Q, q_rows, N, K, epi, far_bias, at, plan, partial), plan.tile, plan.tiles, plan.splits, st);
  } else {
    const GroupedRows<Product> a = rows_in_f32(y, P, Q, q_rows, N, K, epi, far_bias, at, plan, partial);
    e = y.type == ILARGI_TYPE_BF16 ? rows_f32<bf16_t>(a, plan.tile, plan.tiles, plan.splits, st) : rows_f32<float>(a, plan.tile, plan.tiles, plan.splits, st);
  }
  if (e != hipSuccess || plan.splits == 1) return e;
  return in_parts(blocks_in(y.n * (up4(N) / 4), 256), 256, [&](int64_t first, unsigned blocks) {
    grouped_rows_join_kernel<<<blocks, 256, 0, st>>>(epi, N, at, far_bias, first, plan.splits, partial);
  });
}

template <class Prod>
GroupedSums<Prod> sums_of_layer(const ilargi_groups_t& y, const Epilogue& epi, int64_t far_out, const GroupIndex& at, const SumsPlan& plan, float* partial) {
  GroupedSums<Prod> a{};
  a.p.M = y.k; a.p.N = y.m; a.p.K = y.n; a.p.batches = 1;
  a.p.epi = epi;
  a.at = at; a.far_out = far_out; a.part = plan.part; a.partial = partial;
  return a;
}
GroupedSums<Product> sums_in_f32(const ilargi_groups_t& y, const Held& P, const Held& Q, const Epilogue& epi, int64_t far_out, const GroupIndex& at, const SumsPlan& plan, float* partial) {
  const int bf16 = y.type == ILARGI_TYPE_BF16;
  GroupedSums<Product> a = sums_of_layer<Product>(y, epi, far_out, at, plan, partial);
  a.p.P = {P.p, P.ld, 1, bf16, 0};
  a.p.Q = {Q.p, Q.ld, 1, bf16, 0};
  return a;
}
hipError_t add_parts(const ilargi_groups_t& y, const Epilogue& epi, int64_t far_out, const GroupIndex& at, const SumsPlan& plan, const float* partial, hipStream_t st) {
  if (plan.several == 0) return hipSuccess;
  // (the longest groups come first, where they are sorted)
  const unsigned places = (unsigned)(y.groups <= kMostSorted ? plan.several : y.groups);
  return in_parts(blocks_in(y.k * (up4(y.m) / 4), 256), 256, [&](int64_t first, unsigned blocks) {
    grouped_sums_join_kernel<<<dim3(blocks, places), 256, 0, st>>>(epi, y.k, y.m, at, plan.part, far_out, first, partial);
  });
}
GroupedSums<Product16> sums_in_16(const ilargi_groups_t& y, const Held& P, const Held& Q, const Epilogue& epi, int64_t far_out, const GroupIndex& at, const SumsPlan& plan, float* partial) {
  GroupedSums<Product16> a = sums_of_layer<Product16>(y, epi, far_out, at, plan, partial);
  a.p.P = {P.p, P.ld, 1, 0, 0, up8(P.cols)};
  a.p.Q = {Q.p, Q.ld, 1, 0, 0, up8(Q.cols)};
  a.p.kind = kMm16Bf16;
  return a;
}
hipError_t sums_product(const ilargi_groups_t& y, const Held& P, const Held& Q, const Epilogue& epi, int64_t far_out, const GroupIndex& at, const SumsPlan& plan, bool h16, float* partial,
                        hipStream_t st) {
  hipError_t e;
  if (h16) {
    e = launch_grouped16_sums(sums_in_16(y, P, Q, epi, far_out, at, plan, partial), plan.tile, plan.parts, st);
  } else {
    const GroupedSums<Product> a = sums_in_f32(y, P, Q, epi, far_out, at, plan, partial);
    e = y.type == ILARGI_TYPE_BF16 ? sums_f32<bf16_t>(a, plan.tile, plan.parts, st) : sums_f32<float>(a, plan.tile, plan.parts, st);
  }
  return e != hipSuccess ? e : add_parts(y, epi, far_out, at, plan, partial, st);
}

}  // namespace

bool grouped_blocks_fit(const ilargi_groups_t& y) {
  const double rows = (double)(y.n / 64 + y.groups), k = (double)blocks_in(y.k, 64), m = (double)blocks_in(y.m, 64);
  return rows * k < 2147483647.0 && rows * m < 2147483647.0 && (double)(y.n / 256 + y.groups) * k * m < 2147483647.0;
}

void grouped_bytes(const ilargi_groups_t& y, size_t* forward, size_t* gradient) {
  const GroupedLayout l = grouped_layout(y);
  if (forward != nullptr) *forward = l.forward;
  if (gradient != nullptr) *gradient = l.gradient;
}

hipError_t launch_grouped(const GroupedArgs& a, char* ws, hipStream_t st) {
  const ilargi_groups_t& y = a.y;
  const GroupedLayout l = grouped_layout(y);
  const GroupIndex at = index_in(ws, y, a.offsets);
  Held x{a.X, a.ld_x, y.n, y.k, 0, false}, w{a.W, a.ld_w, y.k, y.m, a.stride_w, false};
  if (hipError_t e = lay_out(y, &x, 1, ws + l.x, st); e != hipSuccess) return e;
  if (hipError_t e = lay_out(y, &w, y.groups, ws + l.w, st); e != hipSuccess) return e;
  const bool h16 = y.type == ILARGI_TYPE_BF16 && in_pieces(x) && in_pieces(w);
  const RowsPlan plan = rows_plan(y, y.m, y.k, h16);
  if (hipError_t e = find_groups(at, plan.tile, 0, 0, st); e != hipSuccess) return e;
  Epilogue epi{};
  epi.mode = kEpiLinear;
  epi.bias = a.bias; epi.src = a.residual; epi.ld_src = a.ld_res; epi.src_bf16 = y.type == ILARGI_TYPE_BF16;
  epi.pre = a.pre; epi.ld_pre = a.ld_pre; epi.act = y.act;
  epi.out = a.out; epi.ld_out = a.ld_out; epi.out_bf16 = y.type == ILARGI_TYPE_BF16;
  return rows_product(y, x, w, 1, y.m, y.k, epi, a.ld_bias, at, plan, h16, (float*)(ws + l.partial), st);
}

hipError_t launch_grouped_grad(const GroupedArgs& a, char* ws, hipStream_t st) {
  const ilargi_groups_t& y = a.y;
  const GroupedLayout l = grouped_layout(y);
  const GroupIndex at = index_in(ws, y, a.offsets);
  const int bf16 = y.type == ILARGI_TYPE_BF16;
  const bool bent = y.act != ILARGI_ACT_NONE, products = a.d_X != nullptr || a.d_W != nullptr;
  Held x{a.X, a.ld_x, y.n, y.k, 0, false}, w{a.W, a.ld_w, y.k, y.m, a.stride_w, false}, z{a.d_out, a.ld_dout, y.n, y.m, 0, false};
  void* dz = nullptr;
  if (products && (bent || (worth_packing(y) && !in_pieces(z)))) {
    dz = ws + l.dz;
    z = {dz, up8(y.m), y.n, y.m, 0, true};
  }
  if (a.d_X != nullptr)
    if (hipError_t e = lay_out(y, &w, y.groups, ws + l.w, st); e != hipSuccess) return e;
  if (a.d_W != nullptr)
    if (hipError_t e = lay_out(y, &x, 1, ws + l.x, st); e != hipSuccess) return e;
  const bool rows16 = bf16 && in_pieces(z) && in_pieces(w), sums16 = bf16 && in_pieces(z) && in_pieces(x);
  const RowsPlan rows = rows_plan(y, y.k, y.m, rows16);
  const SumsPlan sums = sums_plan(y, sums16);
  const int chunk = chunk_rows(y);
  const bool passes = dz != nullptr || a.d_bias != nullptr;
  if (hipError_t e = find_groups(at, a.d_X != nullptr ? rows.tile : 0, a.d_W != nullptr ? sums.part : 0, passes ? chunk : 0, st); e != hipSuccess) return e;
  const int64_t side = sums16 ? 128 : 64, cols = rows16 && rows.tile != 32 ? 128 : 64;
  const int64_t tm = blocks_in(y.k, side), tn = blocks_in(y.m, side), bias_columns = blocks_in(y.m, 16);
  const int64_t w_blocks = sums.parts * tm * tn, x_blocks = rows.tiles * blocks_in(y.k, cols), b_blocks = a.d_bias != nullptr ? y.groups * bias_columns : 0;
  const bool alike = rows16 == sums16 && sums.tile == side && rows.splits == 1 && (rows16 ? rows.tile != 256 : rows.tile == 64);
  const bool together = a.d_X != nullptr && a.d_W != nullptr && y.n > 0 && alike && w_blocks + x_blocks + b_blocks <= kMostThreads / 256;
  GroupedGrad g{};
  g.g = {y.n, y.m, a.d_out, a.ld_dout, a.pre_in, a.ld_pre, y.act, bf16, dz, up8(y.m), a.d_bias, a.accumulate};
  g.at = at; g.chunk = chunk; g.ld_dbias = a.ld_dbias;
  g.partial = a.d_bias != nullptr ? (float*)(ws + l.chunks) : nullptr;
  if (passes) {
    const int64_t chunks = chunks_in(y), wide = blocks_in(dz != nullptr ? up8(y.m) : y.m, kGradCols);
    for (int64_t c = 0; c < chunks; c += kMostAcross) {
      const hipError_t e = in_parts(wide, 256, [&](int64_t first, unsigned blocks) {
        const dim3 grid(blocks, (unsigned)(chunks - c < kMostAcross ? chunks - c : kMostAcross));
        if (bf16) grouped_grad_kernel<bf16_t><<<grid, 256, 0, st>>>(g, first, (int)c);
        else grouped_grad_kernel<float><<<grid, 256, 0, st>>>(g, first, (int)c);
      });
      if (e != hipSuccess) return e;
    }
  }
  if (a.d_bias != nullptr && !together) {
    const hipError_t e = in_parts(bias_columns, 256, [&](int64_t first, unsigned blocks) {
      const dim3 grid(blocks, (unsigned)y.groups);
      if (bf16) grouped_bias_kernel<bf16_t><<<grid, 256, 0, st>>>(g, first);
      else grouped_bias_kernel<float><<<grid, 256, 0, st>>>(g, first);
    });
    if (e != hipSuccess) return e;
  }
  Epilogue epi{}, epi_w{};
  epi.mode = epi_w.mode = kEpiLinear;
  epi.out_bf16 = epi_w.out_bf16 = bf16;
  epi.out = a.d_X; epi.ld_out = a.ld_dx;
  epi_w.out = a.d_W; epi_w.ld_out = a.ld_dw;
  if (a.accumulate) { epi_w.src = a.d_W; epi_w.ld_src = a.ld_dw; epi_w.src_bf16 = bf16; }
  float* partial = (float*)(ws + l.shares);
  if (together) {
    hipError_t e;
    if (rows16) {
      e = launch_grouped16_both(sums_in_16(y, x, z, epi_w, a.stride_dw, at, sums, partial), w_blocks, rows_in_16(y, z, w, 0, y.k, y.m, epi, 0, at, rows, partial), rows.tile, x_blocks, g,
                                b_blocks, st);
    } else {
      const GroupedSums<Product> sw = sums_in_f32(y, x, z, epi_w, a.stride_dw, at, sums, partial);
      const GroupedRows<Product> rx = rows_in_f32(y, z, w, 0, y.k, y.m, epi, 0, at, rows, partial);
      const unsigned all = (unsigned)(w_blocks + x_blocks + b_blocks);
      if (bf16) grouped_both_kernel<bf16_t><<<all, 256, 0, st>>>(sw, (int)w_blocks, (int)tm, (int)tn, rx, (int)x_blocks, (int)tm, g, (int)bias_columns);
      else grouped_both_kernel<float><<<all, 256, 0, st>>>(sw, (int)w_blocks, (int)tm, (int)tn, rx, (int)x_blocks, (int)tm, g, (int)bias_columns);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    return add_parts(y, epi_w, a.stride_dw, at, sums, partial, st);
  }
  if (a.d_X != nullptr && y.n > 0)
    if (hipError_t e = rows_product(y, z, w, 0, y.k, y.m, epi, 0, at, rows, rows16, partial, st); e != hipSuccess) return e;
  return a.d_W != nullptr ? sums_product(y, x, z, epi_w, a.stride_dw, at, sums, sums16, partial, st) : hipSuccess;
}

}  // namespace ilargi
