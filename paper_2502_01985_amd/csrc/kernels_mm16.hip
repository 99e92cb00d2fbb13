// Matrix products of 16-bit operands on the matrix cores, sums in float32.
//
// A workgroup forms a BM x BN block of C in steps of 64 k.  Each step's two operand tiles go from memory straight into LDS
// (16 bytes a lane, no registers between), two steps ahead of their use; a wavefront reads its fragments for one half of a
// step while the matrix cores work on the other half, so one barrier a step suffices.
//   rows over k inside (K contiguous): tile rows of 64 k = 8 pieces of 16 bytes; piece p of row r lies at p ^ (r & 7), which
//     spreads the 16 rows that a fragment read touches over all banks.
//   k_rows (rows of the matrix run over k): tile rows of BM or BN neighbours; blocks of 32 bytes lie at b ^ swap(k), and the
//     transposing LDS read gives each lane its four k of one column.
// LDS is filled in lane order, so the places are permuted by the addresses that the lanes fetch from.
// The columns of the result are the first operand of the matrix instruction: a lane then holds four neighbouring columns.
#include "mm_epilogue.h"

namespace ilargi {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kBK = 64, kOutPad = 68;

__device__ __attribute__((aligned(16))) const unsigned int kZeros[4] = {0, 0, 0, 0};   // what lies behind the end of k

template <int PLANES>
__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (PLANES == 2) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
// 16 bytes a lane from base + offset (offset by lane) to LDS at `to` + 16 lane.  The caller waits for it.  (Written out because
// the compiler, which cannot tell the two halves of the LDS buffer apart, would wait for every such load before the next LDS
// read.  M0 holds no value of the compiler's from one instruction to another.)
__device__ __forceinline__ void fetch16(const void* base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void fetch16_at(const void* p, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(p) : "memory");
}

// One operand's tile of R rows or columns by 64 k.
template <bool KROWS, int R, int NT>
struct Tile {
  static constexpr int kLoads = R * 8 / NT, kBytes = R * kBK * 2;
  uint32_t off[kLoads];     // bytes from the step's first element to this lane's piece

  __device__ __forceinline__ void plan(int64_t ld, int64_t left) {      // left: rows or columns of the matrix from the tile's first on
    const int t = threadIdx.x;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int c = q * NT + t;
      if constexpr (KROWS) {
        const int k = c / (R / 8), pos = c % (R / 8), swap = (k & 3) | ((k >> 3) & 1) << 2;
        int col = (((pos >> 1) ^ (swap & (R / 16 - 1))) << 1 | (pos & 1)) * 8;
        if (col > left - 8) col = (int)(left - 8);
        off[q] = (uint32_t)((k * ld + col) * 2);
      } else {
        int row = c >> 3;
        const int piece = (c & 7) ^ (row & 7);
        if (row > left - 1) row = (int)(left - 1);
        off[q] = (uint32_t)((row * ld + piece * 8) * 2);
      }
    }
  }
  // `base`: the step's first element of the tile
  __device__ __forceinline__ void fetch(const char* base, uint32_t to) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) fetch16(base, off[q], to + (uint32_t)(q * NT + wave * 64) * 16);
  }
  // the last step, of `left` k
  __device__ __forceinline__ void fetch_last(const char* base, uint32_t to, int left) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      const int c = q * NT + (int)threadIdx.x, k = KROWS ? c / (R / 8) : (((c & 7) ^ ((c >> 3) & 7)) * 8);
      fetch16_at(k < left ? (const void*)(base + off[q]) : (const void*)kZeros, to + (uint32_t)(q * NT + wave * 64) * 16);
    }
  }
};

// Fragments of F blocks of 16 rows (from `first` on) and 32 k.
template <bool KROWS, int R, int F>
struct Fragments {
  uint32_t at[KROWS ? F : 1];
  __device__ __forceinline__ void plan(int first) {
    const int lane = threadIdx.x % 64, g = lane >> 4, i = lane & 15;
    if constexpr (KROWS) {
      const int k = 8 * g + (i >> 2), swap = ((i >> 2) | (g & 1) << 2) & (R / 16 - 1);
#pragma unroll
      for (int f = 0; f < F; ++f) at[f] = (uint32_t)(k * R * 2 + (((first / 16 + f) ^ swap) * 32) + (i & 3) * 8);
    } else {
      at[0] = (uint32_t)((first + i) * 128);
    }
  }
  __device__ __forceinline__ void read(uint32_t lds, int half, s16x8 (&v)[F]) const {
    if constexpr (KROWS) {
#pragma unroll
      for (int f = 0; f < F; ++f) {
        typedef __attribute__((address_space(3))) s16x4 l4;
        const uint32_t p = lds + at[f] + half * 32 * R * 2;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(uintptr_t)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(uintptr_t)(p + 4 * R * 2));
        v[f] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    } else {
      const int lane = threadIdx.x % 64;
      typedef __attribute__((address_space(3))) s16x8 l8;
      const uint32_t p = lds + at[0] + (uint32_t)(((half * 4 + (lane >> 4)) ^ (lane & 7)) * 16);
#pragma unroll
      for (int f = 0; f < F; ++f) v[f] = *(const l8*)(uintptr_t)(p + f * 16 * 128);
    }
  }
};

__device__ __forceinline__ void arrived_and_together() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Workgroups go to the eight XCDs in turn.  Each XCD takes a run of neighbouring blocks, walked eight rows of blocks at a time,
// so that its L2 keeps the operand tiles they share.
__device__ __forceinline__ void block_of(int id, int tm, int tn, int* ti, int* tj) {
  const int total = tm * tn, q = total / 8, r = total % 8, x = id % 8, l = id / 8;
  id = (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + l;
  constexpr int kGroup = 8;
  const int g = id / (kGroup * tn), first = g * kGroup, rows = tm - first < kGroup ? tm - first : kGroup, in = id % (kGroup * tn);
  *ti = first + in % rows;
  *tj = in / rows;
}

template <int PLANES, bool PK, bool QK, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64) void mm16_kernel(Product16 a, int tm, int tn) {
  constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
  using TileP = Tile<PK, BM, NT>;
  using TileQ = Tile<QK, BN, NT>;
  static_assert(TN == 64 && TM % 64 == 0, "wavefronts of 64 columns and whole 64 rows");
  constexpr int kTiles = 2 * (TileP::kBytes + TileQ::kBytes), kOut = NT * kOutPad * 4;
  __shared__ __attribute__((aligned(1024))) char lds_all[kTiles > kOut ? kTiles : kOut];
  char(*lds)[TileP::kBytes + TileQ::kBytes] = reinterpret_cast<char(*)[TileP::kBytes + TileQ::kBytes]>(lds_all);
  int ti, tj;
  block_of(blockIdx.x, tm, tn, &ti, &tj);
  const int64_t i0 = (int64_t)ti * BM, j0 = (int64_t)tj * BN, b = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wi = (wave / WN) * TM, wj = (wave % WN) * TN;
  const char* P = (const char*)a.P.p + 2 * (b * a.P.batch + (PK ? i0 : i0 * a.P.ld));
  const char* Q = (const char*)a.Q.p + 2 * (b * a.Q.batch + (QK ? j0 : j0 * a.Q.ld));
  const int64_t step_p = PK ? kBK * a.P.ld * 2 : kBK * 2, step_q = QK ? kBK * a.Q.ld * 2 : kBK * 2;
  TileP tp;
  TileQ tq;
  tp.plan(a.P.ld, a.M - i0);
  tq.plan(a.Q.ld, a.N - j0);
  Fragments<PK, BM, FM> fp;
  Fragments<QK, BN, FN> fq;
  fp.plan(wi);
  fq.plan(wj);
  const int ks = (int)((a.K + kBK - 1) / kBK), steps = PLANES == 2 ? 3 * ks : ks;
  const bool whole = a.K % kBK == 0;
  auto fetch = [&](int t) {
    int k = t;
    const char *p = P, *q = Q;
    if constexpr (PLANES == 2) {
      const int part = t / ks;                       // lo hi, hi lo, hi hi
      k = t - part * ks;
      if (part == 0) p += 2 * a.P.plane;
      if (part == 1) q += 2 * a.Q.plane;
    }
    const uint32_t to = lds_address(lds[t & 1]);
    p += k * step_p;
    q += k * step_q;
    if (k + 1 < ks || whole) {
      tp.fetch(p, to);
      tq.fetch(q, to + TileP::kBytes);
    } else {
      tp.fetch_last(p, to, (int)(a.K - (int64_t)k * kBK));
      tq.fetch_last(q, to + TileP::kBytes, (int)(a.K - (int64_t)k * kBK));
    }
  };
  f32x4 acc[FM][FN];
#pragma unroll
  for (int x = 0; x < FM; ++x)
#pragma unroll
    for (int y = 0; y < FN; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  s16x8 p0[FM], q0[FN], p1[FM], q1[FN];
  if (steps > 0) fetch(0);
  arrived_and_together();
  if (steps > 1) fetch(1);
  if (steps > 0) {
    fp.read(lds_address(lds[0]), 0, p0);
    fq.read(lds_address(lds[0]) + TileP::kBytes, 0, q0);
  }
  for (int t = 0; t < steps; ++t) {
    const uint32_t here = lds_address(lds[t & 1]), next = lds_address(lds[(t & 1) ^ 1]);
    if constexpr (PLANES == 2) {
      if (t == 2 * ks) {
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
          for (int y = 0; y < FN; ++y) acc[x][y] *= 0x1p-11f;
      }
    }
    fp.read(here, 1, p1);
    fq.read(here + TileP::kBytes, 1, q1);
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
      for (int y = 0; y < FN; ++y) acc[x][y] = mfma16<PLANES>(q0[y], p0[x], acc[x][y]);
    arrived_and_together();                          // step t is in registers, step t + 1 in LDS
    if (t + 2 < steps) fetch(t + 2);
    if (t + 1 < steps) {
      fp.read(next, 0, p0);
      fq.read(next + TileP::kBytes, 0, q0);
    }
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
      for (int y = 0; y < FN; ++y) acc[x][y] = mfma16<PLANES>(q1[y], p1[x], acc[x][y]);
  }
  // The sums go through LDS, 64 rows of a wavefront at a time, so that stores run along the result's rows.
  const int lane = threadIdx.x % 64;
  float* mine = (float*)(&lds[0][0]) + wave * 64 * kOutPad;
  __syncthreads();
#pragma unroll
  for (int h = 0; h < TM / 64; ++h) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int y = 0; y < FN; ++y)
        *reinterpret_cast<f32x4*>(mine + (16 * x + (lane & 15)) * kOutPad + 16 * y + (lane >> 4) * 4) = acc[4 * h + x][y];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // a row of 64 columns takes 16 lanes; a flipped result is written along its own rows, which run over i
#pragma unroll 1
    for (int q = 0; q < 16; ++q) {
      const int r = a.epi.flip ? lane : 4 * q + (lane >> 4), c = a.epi.flip ? 4 * q : (lane & 15) * 4;
      const f32x4 t = *reinterpret_cast<const f32x4*>(mine + r * kOutPad + c);
      const int64_t i = i0 + wi + 64 * h + r, j = j0 + wj + c;
      if (i < a.M && j < a.N) {
        float v[4] = {t[0], t[1], t[2], t[3]};
        epilogue4(a.epi, b, i, j, (int)(a.N - j < 4 ? a.N - j : 4), v);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <int PLANES, bool PK, bool QK>
hipError_t mm16_order(const Product16& a, hipStream_t st) {
  const int64_t tm = (a.M + 255) / 256, tn = (a.N + 255) / 256;
  if (tm * tn * a.batches >= 160) {
    mm16_kernel<PLANES, PK, QK, 256, 256, 2, 4><<<dim3((unsigned)(tm * tn), (unsigned)a.batches), 512, 0, st>>>(a, (int)tm, (int)tn);
  } else {
    const int64_t sm = (a.M + 127) / 128, sn = (a.N + 127) / 128;
    mm16_kernel<PLANES, PK, QK, 128, 128, 2, 2><<<dim3((unsigned)(sm * sn), (unsigned)a.batches), 256, 0, st>>>(a, (int)sm, (int)sn);
  }
  return hipGetLastError();
}

}  // namespace

// Whether the kernel reads this operand as it lies: 16-byte pieces that begin at 16-byte addresses and end with the matrix,
// offsets within a tile of 32 bits.
bool mm16_takes(const Operand16& x, int64_t across, int64_t K) {
  return reinterpret_cast<uintptr_t>(x.p) % 16 == 0 && x.ld % 8 == 0 && x.ld < (1 << 22) && (x.k_rows ? across : K) % 8 == 0;
}

hipError_t launch_mm16(const Product16& a, hipStream_t st) {
  if (a.M == 0 || a.N == 0 || a.batches == 0) return hipSuccess;
  if (a.planes == 1) {
    if (a.P.k_rows) return a.Q.k_rows ? mm16_order<1, true, true>(a, st) : hipErrorInvalidValue;
    return a.Q.k_rows ? mm16_order<1, false, true>(a, st) : mm16_order<1, false, false>(a, st);
  }
  if (a.P.k_rows) return hipErrorInvalidValue;
  return a.Q.k_rows ? mm16_order<2, false, true>(a, st) : mm16_order<2, false, false>(a, st);
}

}  // namespace ilargi
