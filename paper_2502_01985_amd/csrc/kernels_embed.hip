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
namespace {

constexpr int kRun = 64;      // sorted ids that one group of lanes sums

// Ids that name no row become -1, which the sort puts behind all rows.
__global__ __launch_bounds__(kBlock) void clean_ids_kernel(const int32_t* __restrict__ ids, int64_t n, int64_t rows,
                                                           int32_t* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i < n) out[i] = ids[i] >= 0 && ids[i] < rows ? ids[i] : -1;
}

struct RunArgs {
  EmbedGradArgs g;
  const int32_t *rowptr, *perm, *sorted;
  float* carry;            // 2 rows of cols floats for every run: sums of the segments that reach into it, and out of it
  int64_t runs;
};

template <class TO, bool ADD>
__device__ __forceinline__ void write_row(const EmbedGradArgs& g, int64_t v, int64_t c, int valid, float* f) {
  constexpr int V = 4;
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

// A group of 2^sh lanes walks kRun sorted ids over columns [blockIdx.y 4 2^sh, ...): rows whose ids all lie in the run are
// written, the sums of the others left as carries.
template <class TI, class TO, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_runs_kernel(RunArgs a, int sh) {
  constexpr int V = 4;
  const int64_t run = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh;
  const int lane = threadIdx.x & ((1 << sh) - 1);
  const int64_t c = ((int64_t)blockIdx.y << sh) * V + (int64_t)lane * V;
  const int64_t live = a.rowptr[a.g.rows];
  const int64_t p0 = run * kRun, p1 = p0 + kRun < live ? p0 + kRun : live;
  if (run >= a.runs || p0 >= live || c >= a.g.cols) return;
  const int valid = (int)(a.g.cols - c < V ? a.g.cols - c : V);
  float s[V] = {0.f, 0.f, 0.f, 0.f};
  int32_t key = a.sorted[p0];
  bool open = p0 > 0 && a.sorted[p0 - 1] == key;       // the segment began in an earlier run
  for (int64_t p = p0; p < p1; ++p) {
    float f[V];
    load_piece<TI, V>((const TI*)a.g.d_out + (int64_t)a.perm[p] * a.g.ld_out + c, valid, f);
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] += f[j];
    const int32_t next = p + 1 < live ? a.sorted[p + 1] : -1;
    const bool last = p + 1 == p1;
    if (next != key || last) {
      if (open || next == key) {
        // slot 0: a segment from before (through the whole run, perhaps); slot 1: one that begins here and goes on
        store_piece<float, V>(a.carry + (2 * run + (open ? 0 : 1)) * a.g.cols + c, valid, s);
      } else {
        write_row<TO, ADD>(a.g, key, c, valid, s);
      }
      open = false;
      key = next;
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] = 0.0f;
    }
  }
}

// Rows without ids are zeroed (unless the caller accumulates); rows whose ids lie in several runs get the sum of the carries.
template <class TO, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_join_kernel(RunArgs a, int sh) {
  constexpr int V = 4;
  const int64_t v = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh;
  const int lane = threadIdx.x & ((1 << sh) - 1);
  const int64_t c = ((int64_t)blockIdx.y << sh) * V + (int64_t)lane * V;
  if (v >= a.g.rows || c >= a.g.cols) return;
  const int valid = (int)(a.g.cols - c < V ? a.g.cols - c : V);
  const int64_t b = a.rowptr[v], e = a.rowptr[v + 1];
  float s[V] = {0.f, 0.f, 0.f, 0.f};
  if (b == e) {
    if (!ADD) store_piece<TO, V>((TO*)a.g.d_table + v * a.g.ld_table + c, valid, s);
    return;
  }
  const int64_t r0 = b / kRun, r1 = (e - 1) / kRun;
  if (r0 == r1) return;
  for (int64_t r = r0; r <= r1; ++r) {
    const int slot = r == r0 ? 1 : 0;
    float f[V];
    load_piece<float, V>(a.carry + (2 * r + slot) * a.g.cols + c, valid, f);
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] += f[j];
  }
  write_row<TO, ADD>(a.g, v, c, valid, s);
}

struct GradLayout {
  size_t clean, keys_a, vals_a, keys_b, vals_b, hist, rowptr, perm, carry, total;
  int64_t runs;
};
size_t up256(size_t v) { return (v + 255) / 256 * 256; }
GradLayout grad_layout(int64_t n, int64_t rows, int64_t cols) {
  GradLayout l{};
  size_t at = 0;
  auto take = [&at](size_t bytes) { const size_t o = at; at += up256(bytes); return o; };
  l.runs = (n + kRun - 1) / kRun;
  l.clean = take(4 * (size_t)n);
  l.keys_a = take(4 * (size_t)n);
  l.vals_a = take(4 * (size_t)n);
  l.keys_b = take(4 * (size_t)n);
  l.vals_b = take(4 * (size_t)n);
  l.hist = take(4 * sort_hist_ints(n));
  l.rowptr = take(4 * (size_t)(rows + 1));
  l.perm = take(4 * (size_t)n);
  l.carry = take(4 * 2 * (size_t)l.runs * (size_t)cols);
  l.total = at;
  return l;
}

template <class TI, class TO>
hipError_t grad_typed(const RunArgs& r, hipStream_t st) {
  int sh = ilog2_ceil((r.g.cols + 3) / 4);
  if (sh > 6) sh = 6;
  const unsigned slabs = (unsigned)((r.g.cols + (4ll << sh) - 1) / (4ll << sh));
  const dim3 runs((unsigned)(((r.runs << sh) + kBlock - 1) / kBlock), slabs);
  const dim3 rows((unsigned)(((r.g.rows << sh) + kBlock - 1) / kBlock), slabs);
  if (r.g.accumulate) {
    if (r.runs > 0) embed_runs_kernel<TI, TO, true><<<runs, kBlock, 0, st>>>(r, sh);
    embed_join_kernel<TO, true><<<rows, kBlock, 0, st>>>(r, sh);
  } else {
    if (r.runs > 0) embed_runs_kernel<TI, TO, false><<<runs, kBlock, 0, st>>>(r, sh);
    embed_join_kernel<TO, false><<<rows, kBlock, 0, st>>>(r, sh);
  }
  return hipGetLastError();
}

}  // namespace

size_t embed_grad_bytes(int64_t n, int64_t rows, int64_t cols) { return grad_layout(n, rows, cols).total; }

hipError_t launch_embed_grad(const EmbedGradArgs& a, char* ws, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const GradLayout l = grad_layout(a.n, a.rows, a.cols);
  int32_t* clean = (int32_t*)(ws + l.clean);
  if (a.n > 0) clean_ids_kernel<<<(unsigned)((a.n + kBlock - 1) / kBlock), kBlock, 0, st>>>(a.ids, a.n, a.rows, clean);
  int32_t *ka = (int32_t*)(ws + l.keys_a), *kb = (int32_t*)(ws + l.keys_b);
  if (hipError_t e = launch_sort_by_source_row(clean, a.n, a.rows, ka, (int32_t*)(ws + l.vals_a), kb, (int32_t*)(ws + l.vals_b),
                                               (int32_t*)(ws + l.hist), (int32_t*)(ws + l.rowptr), (int32_t*)(ws + l.perm), st);
      e != hipSuccess)
    return e;
  int bits = ilog2_ceil(a.rows + 1);
  const int passes = (bits < 1 ? 1 : bits) + 7;
  RunArgs r{a, (int32_t*)(ws + l.rowptr), (int32_t*)(ws + l.perm), passes / 8 % 2 == 1 ? ka : kb, (float*)(ws + l.carry), l.runs};
  if (a.out_bf16) return a.table_bf16 ? grad_typed<bf16_t, bf16_t>(r, st) : grad_typed<bf16_t, float>(r, st);
  return a.table_bf16 ? grad_typed<float, bf16_t>(r, st) : grad_typed<float, float>(r, st);
}

}  // namespace ilargi
