// A block of a product of 16-bit operands on the matrix cores, sums in float32 (kernels_mm16.hip, kernels_grouped16.hip).
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
//
// Bound by the matrix cores and, in blocks of 256, by the power they take (the clock falls to 2.0 GHz).  256-blocks: 8192 x 8192 x 4096
// 1240 TFLOP/s with K contiguous on both sides, 1245 with one and 1250 with both operands' rows over k; the library's product 1210.
// 128-blocks, two to a compute unit, for results of fewer than 256 large blocks: 2048 x 2048 x 2048 545 TFLOP/s.
#ifndef ILARGI_MM16_BLOCK_H_
#define ILARGI_MM16_BLOCK_H_

#include <utility>

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

template <int KIND>
__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (KIND != kMm16Bf16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
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
  template <int FIRST, int COUNT>
  __device__ __forceinline__ void fetch_some(const char* base, uint32_t to) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
    for (int q = FIRST; q < FIRST + COUNT && q < kLoads; ++q) fetch16(base, off[q], to + (uint32_t)(q * NT + wave * 64) * 16);
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
  __device__ __forceinline__ s16x8 read(uint32_t lds, int half, int f) const {
    if constexpr (KROWS) {
      typedef __attribute__((address_space(3))) s16x4 l4;
      const uint32_t p = lds + at[f] + half * 32 * R * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(uintptr_t)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(uintptr_t)(p + 4 * R * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int lane = threadIdx.x % 64;
      typedef __attribute__((address_space(3))) s16x8 l8;
      const uint32_t p = lds + at[0] + (uint32_t)(((half * 4 + (lane >> 4)) ^ (lane & 7)) * 16);
      return *(const l8*)(uintptr_t)(p + f * 16 * 128);
    }
  }
};

// All but the last LEFT fetches of every wavefront are in LDS, and all LDS reads done (0xc07f waits for those alone, in a form that
// the compiler counts with: it would else wait for them again behind the next reads).
template <int LEFT>
__device__ __forceinline__ void arrived_and_together() {
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// The products of the second half of a step, between them the fetches of a later step into the buffer that has become free
// and the reads of the next step's first half.
template <class TileP, class TileQ, int KIND, int FM, int FN, class FragP, class FragQ>
__device__ __forceinline__ void second_half(bool fetching, const TileP& tp, const TileQ& tq, const char* from_p, const char* from_q, uint32_t to, const FragP& fp,
                                            const FragQ& fq, uint32_t next, s16x8 (&p0)[FM], s16x8 (&q0)[FN], const s16x8 (&p1)[FM],
                                            const s16x8 (&q1)[FN], f32x4 (&acc)[FM][FN]) {
  constexpr int kP = (TileP::kLoads + FM - 1) / FM, kQ = (TileQ::kLoads + FM - 1) / FM;
  q0[0] = fq.read(next + TileP::kBytes, 0, 0);
  [&]<int... X>(std::integer_sequence<int, X...>) {
    (
        [&] {
          p0[X] = fp.read(next, 0, X);
          if constexpr (X + 1 < FN) q0[X + 1] = fq.read(next + TileP::kBytes, 0, X + 1);
          if (fetching) {
            tp.template fetch_some<X * kP, kP>(from_p, to);
            tq.template fetch_some<X * kQ, kQ>(from_q, to + TileP::kBytes);
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int y = 0; y < FN; ++y) acc[X][y] = mfma16<KIND>(q1[y], p1[X], acc[X][y]);
          __builtin_amdgcn_sched_barrier(0);
        }(),
        ...);
  }(std::make_integer_sequence<int, FM>());
}

// Eight neighbouring columns of a row of a layer's bfloat16 result, past the caches where the outputs are larger than they hold.
__device__ __forceinline__ void store8(bf16_t* p, int valid, bool past, const float (&v)[8]) {
  if (past && valid >= 8) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
    Piece<bf16_t, 8> t;
#pragma unroll
    for (int j = 0; j < 8; ++j) t.v[j] = (bf16_t)v[j];
    __builtin_nontemporal_store(__builtin_bit_cast(words, t), reinterpret_cast<words*>(p));
  } else {
    store_piece<bf16_t, 8>(p, valid, v);
  }
}

// The sums of a wavefront (TM x 64) of a bfloat16 layer go through LDS, 64 rows at a time, so that stores run along the result's rows,
// 16 bytes a lane.  The residual is added in a pass of its own, in which the loads of four rows are on their way together.
// 16384 x 2048 x 8192, gelu, z kept: 628 us in one pass of 8 bytes a lane for every kind of result, 597 with this, 562 to 571 past the
// caches (whose lines the operands then keep); with a residual 785 and 720.
template <int TM, int FN>
__device__ __forceinline__ void store_layer(const Product16& a, float* __restrict__ sums_to, char* lds, const f32x4 (&acc)[TM / 16][FN], int64_t i0, int64_t j0) {
  const int lane = threadIdx.x % 64, c = (lane & 7) * 8;
  float* mine = (float*)lds + threadIdx.x / 64 * 64 * kOutPad;
  const Epilogue& e = a.epi;
  const int64_t j = j0 + c;
  const int valid = j >= a.N ? 0 : a.N - j < 8 ? (int)(a.N - j) : 8;
  float bias[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) bias[q] = 0.0f;
  if (e.bias != nullptr && valid > 0) load_piece<bf16_t, 8>((const bf16_t*)e.bias + j, valid, bias);
  const bool added = e.src != nullptr;
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
    const int64_t ih = i0 + 64 * h + (lane >> 3);
    float* const at = mine + (lane >> 3) * kOutPad + c;
    if (sums_to != nullptr) {
      const int64_t ldp = (a.N + 3) / 4 * 4;
      float* part = sums_to + j;
#pragma unroll 2
      for (int q = 0; q < 8; ++q) {
        const int64_t i = ih + 8 * q;
        if (i >= a.M) continue;
        if (valid > 0) *reinterpret_cast<f32x4*>(part + i * ldp) = *reinterpret_cast<const f32x4*>(at + 8 * q * kOutPad);
        if (valid > 4) *reinterpret_cast<f32x4*>(part + i * ldp + 4) = *reinterpret_cast<const f32x4*>(at + 8 * q * kOutPad + 4);
      }
    } else {
#pragma unroll 1
      for (int q = 0; q < 8; ++q) {
        const int64_t i = ih + 8 * q;
        if (i >= a.M || valid == 0) continue;
        f32x4* const sums = reinterpret_cast<f32x4*>(at + 8 * q * kOutPad);
        const f32x4 s0 = sums[0], s1 = sums[1];
        float v[8] = {s0[0] + bias[0], s0[1] + bias[1], s0[2] + bias[2], s0[3] + bias[3], s1[0] + bias[4], s1[1] + bias[5], s1[2] + bias[6], s1[3] + bias[7]};
        if (e.pre != nullptr) store8((bf16_t*)e.pre + i * e.ld_pre + j, valid, a.past, v);
        act_values(v, e.act);
        if (added) {
          sums[0] = f32x4{v[0], v[1], v[2], v[3]};
          sums[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
          store8((bf16_t*)e.out + i * e.ld_out + j, valid, a.past, v);
        }
      }
      if (added) {
#pragma unroll 1
        for (int q = 0; q < 8; q += 4) {
          float r[4][8];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int64_t i = ih + 8 * (q + u);
            load_piece<bf16_t, 8>((const bf16_t*)e.src + i * e.ld_src + j, i < a.M ? valid : 0, r[u]);
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int64_t i = ih + 8 * (q + u);
            if (i >= a.M || valid == 0) continue;
            const f32x4* const sums = reinterpret_cast<const f32x4*>(at + 8 * (q + u) * kOutPad);
#pragma unroll
            for (int w = 0; w < 8; ++w) r[u][w] += sums[w / 4][w % 4];
            store8((bf16_t*)e.out + i * e.ld_out + j, valid, a.past, r[u]);
          }
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// The bytes of LDS of a block.
template <bool PK, bool QK, int BM, int BN, int WM, int WN>
constexpr int mm16_lds() {
  constexpr int NT = WM * WN * 64, tiles = 2 * (Tile<PK, BM, NT>::kBytes + Tile<QK, BN, NT>::kBytes), out = NT * kOutPad * 4;
  return tiles > out ? tiles : out;
}

// Block (ti, tj) of C over share z of k.  With `sums_to` the sums go there, a matrix of M x (N to a multiple of 4).
template <bool PK, bool QK, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void mm16_block(const Product16& a, int ti, int tj, int z, int share, float* __restrict__ sums_to, char* lds_all) {
  constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16, STAGES = 2, KIND = kMm16Bf16;
  using TileP = Tile<PK, BM, NT>;
  using TileQ = Tile<QK, BN, NT>;
  static_assert(TN == 64 && TM % 64 == 0, "wavefronts of 64 columns and whole 64 rows");
  char(*lds)[TileP::kBytes + TileQ::kBytes] = reinterpret_cast<char(*)[TileP::kBytes + TileQ::kBytes]>(lds_all);
  const int64_t i0 = (int64_t)ti * BM, j0 = (int64_t)tj * BN;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wi = (wave / WN) * TM, wj = (wave % WN) * TN;
  const int64_t step_p = PK ? kBK * a.P.ld * 2 : kBK * 2, step_q = QK ? kBK * a.Q.ld * 2 : kBK * 2;
  const int first = z * share, ks_all = (int)((a.K + kBK - 1) / kBK), ks = ks_all - first < share ? ks_all - first : share;
  const char* P = (const char*)a.P.p + 2 * (PK ? i0 : i0 * a.P.ld) + first * step_p;
  const char* Q = (const char*)a.Q.p + 2 * (QK ? j0 : j0 * a.Q.ld) + first * step_q;
  TileP tp;
  TileQ tq;
  tp.plan(a.P.ld, a.P.across - i0);
  tq.plan(a.Q.ld, a.Q.across - j0);
  Fragments<PK, BM, FM> fp;
  Fragments<QK, BN, FN> fq;
  fp.plan(wi);
  fq.plan(wj);
  const int steps = ks;
  const bool whole = a.K % kBK == 0 || first + ks < ks_all;
  // Where step t's pieces come from, and the k that its last step has.
  auto source = [&](int t, const char** p, const char** q) {
    *p = P + t * step_p;
    *q = Q + t * step_q;
    return t + 1 < ks || whole ? kBK : (int)(a.K - (int64_t)(first + t) * kBK);
  };
  auto fetch = [&](int t) {
    const char *p, *q;
    const int left = source(t, &p, &q);
    const uint32_t to = lds_address(lds[t % STAGES]);
    if (left == kBK) {
      tp.template fetch_some<0, TileP::kLoads>(p, to);
      tq.template fetch_some<0, TileQ::kLoads>(q, to + TileP::kBytes);
    } else {
      tp.fetch_last(p, to, left);
      tq.fetch_last(q, to + TileP::kBytes, left);
    }
  };
  f32x4 acc[FM][FN];
#pragma unroll
  for (int x = 0; x < FM; ++x)
#pragma unroll
    for (int y = 0; y < FN; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  s16x8 p0[FM], q0[FN], p1[FM], q1[FN];
  constexpr int kEach = TileP::kLoads + TileQ::kLoads;
  for (int t = 0; t < STAGES && t < steps; ++t) fetch(t);
  if (steps >= STAGES) arrived_and_together<kEach*(STAGES - 1)>();
  else arrived_and_together<0>();
#pragma unroll
  for (int y = 0; y < FN; ++y) q0[y] = fq.read(lds_address(lds[0]) + TileP::kBytes, 0, y);
#pragma unroll
  for (int x = 0; x < FM; ++x) p0[x] = fp.read(lds_address(lds[0]), 0, x);
  for (int t = 0; t < steps; ++t) {
    const uint32_t here = lds_address(lds[t % STAGES]), next = lds_address(lds[(t + 1) % STAGES]);
    // A wavefront issues in order: the reads of the second half stand between the products of the first, else the matrix cores
    // would wait for their issue.
    q1[0] = fq.read(here + TileP::kBytes, 1, 0);
#pragma unroll
    for (int x = 0; x < FM; ++x) {
      p1[x] = fp.read(here, 1, x);
      if (x + 1 < FN) q1[x + 1] = fq.read(here + TileP::kBytes, 1, x + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int y = 0; y < FN; ++y) acc[x][y] = mfma16<KIND>(q0[y], p0[x], acc[x][y]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // step t is in registers, step t + 1 in LDS
    if (t + STAGES <= steps) arrived_and_together<kEach*(STAGES - 2)>();
    else arrived_and_together<0>();
    const char *from_p = P, *from_q = Q;
    const int left = t + STAGES < steps ? source(t + STAGES, &from_p, &from_q) : 0;
    // the next step's first half between the products of the second (behind the last step: of an old one, for nothing)
    if (left > 0 && left < kBK) fetch(t + STAGES);
    second_half<TileP, TileQ, KIND, FM, FN>(left == kBK, tp, tq, from_p, from_q, here, fp, fq, next, p0, q0, p1, q1, acc);
  }
  store_layer<TM, FN>(a, sums_to, lds_all, acc, i0 + wi, j0 + wj);
}

}  // namespace

}  // namespace ilargi
#endif
