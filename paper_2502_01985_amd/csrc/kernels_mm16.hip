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
//
// Bound by the matrix cores and, in blocks of 256, by the power they take (the clock falls to 2.0 GHz).  256-blocks: 8192 x 8192 x 4096
// 1240 TFLOP/s with K contiguous on both sides, 1245 with one and 1250 with both operands' rows over k; the library's product 1210.
// 128-blocks, two to a compute unit, for results of fewer than 256 large blocks: 2048 x 2048 x 2048 545 TFLOP/s.
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

// The n-th block on or above the diagonal of tn x tn blocks, row by row.
__device__ __forceinline__ void upper_block(int id, int tn, int* ti, int* tj) {
  int r = 0;
  while (id >= tn - r) id -= tn - r++;
  *ti = r;
  *tj = r + id;
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
__device__ __forceinline__ void store_layer(const Product16& a, float* __restrict__ partial, char* lds, const f32x4 (&acc)[TM / 16][FN], int64_t i0, int64_t j0) {
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
    if (partial != nullptr) {
      const int64_t ldp = (a.N + 3) / 4 * 4;
      float* part = partial + (int64_t)blockIdx.z * a.M * ldp + j;
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

// The same of a product of pairs, scaled and added to `src`, into planes, float32 or bfloat16.
template <int TM, int FN>
__device__ __forceinline__ void store_sums(const Product16& a, float by, float* __restrict__ partial, char* lds, const f32x4 (&acc)[TM / 16][FN], int64_t b,
                                           int64_t i0, int64_t j0, bool mirrored) {
  constexpr int kRows = TM < 64 ? TM : 64, kQ = kRows / 4;      // rows of a pass, and its turns of 64 quads
  const int lane = threadIdx.x % 64;
  float* mine = (float*)lds + threadIdx.x / 64 * kRows * kOutPad;
  __syncthreads();
#pragma unroll
  for (int h = 0; h < TM / kRows; ++h) {
#pragma unroll
    for (int x = 0; x < kRows / 16; ++x)
#pragma unroll
      for (int y = 0; y < FN; ++y)
        *reinterpret_cast<f32x4*>(mine + (16 * x + (lane & 15)) * kOutPad + 16 * y + (lane >> 4) * 4) = acc[kRows / 16 * h + x][y];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int64_t ri = i0 + kRows * h;
    const float none[4] = {0.f, 0.f, 0.f, 0.f};
    const int c = (lane & 15) * 4;                     // a row of 64 columns takes 16 lanes
    if (partial != nullptr) {
      const int64_t ldp = (a.N + 3) / 4 * 4;
      float* part = partial + ((int64_t)blockIdx.z * a.batches + b) * a.M * ldp;
#pragma unroll 4
      for (int q = 0; q < kQ; ++q) {
        const int r = 4 * q + (lane >> 4);
        if (ri + r < a.M && j0 + c < a.N) *reinterpret_cast<f32x4*>(part + (ri + r) * ldp + j0 + c) = *reinterpret_cast<const f32x4*>(mine + r * kOutPad + c);
      }
    } else {
      auto row = [&](int r, int at) { return *reinterpret_cast<const float4*>(mine + r * kOutPad + at); };
      if (!a.epi.flip) {
        if (a.epi.src == nullptr) {
#pragma unroll 2
          for (int q = 0; q < kQ; ++q) {
            const int r = 4 * q + (lane >> 4), valid = quad_valid(ri + r, j0 + c, a.M, a.N);
            if (valid == 0) continue;
            const float4 t = row(r, c);
            float v[4] = {t.x, t.y, t.z, t.w};
            epilogue4<false>(a.epi, by, b, ri + r, j0 + c, valid, none, SrcQuad{}, v);
          }
        } else {
#pragma unroll 1
          for (int q = 0; q < kQ; q += 4)
            epilogue_quads<4>(a.epi, by, b, a.M, a.N, none, [&](int u, int64_t* i, int64_t* j) { *i = ri + 4 * (q + u) + (lane >> 4); *j = j0 + c; },
                              [&](int u) { return row(4 * (q + u) + (lane >> 4), c); });
        }
      } else {                                         // written along j's rows, which run over i
        constexpr int kSide = 64 / kRows;              // quads side by side
        const int r = lane % kRows, s = lane / kRows;
#pragma unroll 1
        for (int q = 0; q < kQ; q += 4)
          epilogue_quads<4>(a.epi, by, b, a.M, a.N, none, [&](int u, int64_t* i, int64_t* j) { *i = ri + r; *j = j0 + 4 * ((q + u) * kSide + s); },
                            [&](int u) { return row(r, 4 * ((q + u) * kSide + s)); });
      }
      if (mirrored) {                                // the sums of a symmetric result at their places below the diagonal
        constexpr int kAcross = kRows / 4, kDown = 64 / kAcross;
        const int ci = lane % kAcross * 4, rj = lane / kAcross;
#pragma unroll 1
        for (int q = 0; q < kQ; q += 4)
          epilogue_quads<4>(a.epi, by, b, a.N, a.M, none, [&](int u, int64_t* i, int64_t* j) { *i = j0 + kDown * (q + u) + rj; *j = ri + ci; },
                            [&](int u) {
                              const float* m = mine + ci * kOutPad + kDown * (q + u) + rj;
                              return make_float4(m[0], m[kOutPad], m[2 * kOutPad], m[3 * kOutPad]);
                            });
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// blockIdx: block, none, share of k.  With several shares the sums go to `partial`, one M x (N to a multiple of 4) matrix after the
// other.
template <bool PK, bool QK, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64, 512 / (WM * WN * 64)) void mm16_kernel(Product16 a, int tm, int tn, int share, float* __restrict__ partial) {
  constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16, STAGES = 2, KIND = kMm16Bf16;
  using TileP = Tile<PK, BM, NT>;
  using TileQ = Tile<QK, BN, NT>;
  static_assert(TN == 64 && TM % 64 == 0, "wavefronts of 64 columns and whole 64 rows");
  constexpr int kTiles = STAGES * (TileP::kBytes + TileQ::kBytes), kOut = NT * kOutPad * 4;
  __shared__ __attribute__((aligned(1024))) char lds_all[kTiles > kOut ? kTiles : kOut];
  char(*lds)[TileP::kBytes + TileQ::kBytes] = reinterpret_cast<char(*)[TileP::kBytes + TileQ::kBytes]>(lds_all);
  int ti, tj;
  block_of(blockIdx.x, tm, tn, &ti, &tj);
  const int64_t i0 = (int64_t)ti * BM, j0 = (int64_t)tj * BN;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wi = (wave / WN) * TM, wj = (wave % WN) * TN;
  const int64_t step_p = PK ? kBK * a.P.ld * 2 : kBK * 2, step_q = QK ? kBK * a.Q.ld * 2 : kBK * 2;
  const int first = (int)blockIdx.z * share, ks_all = (int)((a.K + kBK - 1) / kBK), ks = ks_all - first < share ? ks_all - first : share;
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
  store_layer<TM, FN>(a, partial, lds_all, acc, i0 + wi, j0 + wj);
}

// Pairs: a step's four tiles (both planes of both operands) lie in LDS together, and three products are formed from the fragments
// read once: 64 KB fetched for 96 matrix instructions where the planes one after the other would take 96 KB.  Blocks of 128 in
// eight wavefronts: four have 64 x 64 sums of the first half of every step, four the same sums of the second half, and they exchange
// halves of their sums at the end.  So two wavefronts share a SIMD, and one's products run while the other's reads and fetches are
// issued (four wavefronts with both halves: 2048 x 2048 x 2048 takes 55 us, of which the products alone are 33; the fifteen products of
// an orthogonalised 2048 x 2048 took 840 us so, and 750 with eight wavefronts).  Q's rows run over k
// (QK) or its columns do.
// (LDS is asked for at the launch: told of it, the compiler would take the accumulators to the other half of a wavefront's
// registers, and move them to and fro.)
constexpr int kPairsLds = 2 * 4 * 128 * kBK * 2;
template <bool QK>
__global__ __launch_bounds__(512, 1) void mm16_pairs_kernel(Product16 a, int tm, int tn, int share, float* __restrict__ partial) {
  constexpr int NT = 512, FM = 4, FN = 4, kB = 128;
  using TileP = Tile<false, kB, NT>;
  using TileQ = Tile<QK, kB, NT>;
  constexpr int kP = TileP::kBytes, kQ = TileQ::kBytes, kStage = 2 * (kP + kQ), kEach = TileP::kLoads;
  static_assert(kEach == 2 && TileQ::kLoads == 2, "a piece of two tiles between the products of a row of blocks");
  static_assert(2 * kStage == kPairsLds && 8 * 32 * kOutPad * 4 <= kPairsLds, "the sums fit too");
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  int ti, tj;
  if (a.symmetric) upper_block(blockIdx.x, tn, &ti, &tj);
  else block_of(blockIdx.x, tm, tn, &ti, &tj);
  const int64_t i0 = (int64_t)ti * kB, j0 = (int64_t)tj * kB, b = blockIdx.y;
  const float by = a.epi.by != nullptr ? a.epi.by[b] : 1.0f;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = wave / 4, wi = (wave % 4 / 2) * 64, wj = (wave % 2) * 64;
  const int64_t step_q = QK ? kBK * a.Q.ld * 2 : kBK * 2;
  const int first = (int)blockIdx.z * share, ks_all = (int)((a.K + kBK - 1) / kBK), steps = ks_all - first < share ? ks_all - first : share;
  const char* P = (const char*)a.P.p + 2 * (b * a.P.batch + i0 * a.P.ld) + (int64_t)first * kBK * 2;
  const char* Q = (const char*)a.Q.p + 2 * (b * a.Q.batch + (QK ? j0 : j0 * a.Q.ld)) + first * step_q;
  const int64_t lo_p = 2 * a.P.plane, lo_q = 2 * a.Q.plane;
  TileP tp;
  TileQ tq;
  tp.plan(a.P.ld, a.P.across - i0);
  tq.plan(a.Q.ld, a.Q.across - j0);
  Fragments<false, kB, FM> fp;
  Fragments<QK, kB, FN> fq;
  fp.plan(wi);
  fq.plan(wj);
  const uint32_t base = lds_address(lds_all);
  auto left_of = [&](int t) { const int64_t left = a.K - (int64_t)(first + t) * kBK; return left < kBK ? (int)left : kBK; };
  auto fetch = [&](int t) {
    const char *p = P + (int64_t)t * kBK * 2, *q = Q + t * step_q;
    const uint32_t to = base + (t & 1) * kStage;
    if (left_of(t) == kBK) {
      tp.template fetch_some<0, kEach>(p, to);
      tp.template fetch_some<0, kEach>(p + lo_p, to + kP);
      tq.template fetch_some<0, kEach>(q, to + 2 * kP);
      tq.template fetch_some<0, kEach>(q + lo_q, to + 2 * kP + kQ);
    } else {
      tp.fetch_last(p, to, left_of(t));
      tp.fetch_last(p + lo_p, to + kP, left_of(t));
      tq.fetch_last(q, to + 2 * kP, left_of(t));
      tq.fetch_last(q + lo_q, to + 2 * kP + kQ, left_of(t));
    }
  };
  f32x4 acc[FM][FN];
#pragma unroll
  for (int x = 0; x < FM; ++x)
#pragma unroll
    for (int y = 0; y < FN; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  s16x8 ph[2][FM], pl[2][FM], qh[2][FN], ql[2][FN];      // of this step and the next
  auto read = [&](auto set, uint32_t at, auto xs) {
    constexpr int S = decltype(set)::value, X = decltype(xs)::value;
    ph[S][X] = fp.read(at, half, X);
    pl[S][X] = fp.read(at + kP, half, X);
    qh[S][X] = fq.read(at + 2 * kP, half, X);
    ql[S][X] = fq.read(at + 2 * kP + kQ, half, X);
  };
  auto products = [&](auto set, auto xs) {
    constexpr int S = decltype(set)::value, X = decltype(xs)::value;
#pragma unroll
    for (int y = 0; y < FN; ++y) acc[X][y] = mfma16<kMm16Pairs>(ql[S][y], ph[S][X], acc[X][y]);
#pragma unroll
    for (int y = 0; y < FN; ++y) acc[X][y] = mfma16<kMm16Pairs>(qh[S][y], pl[S][X], acc[X][y]);
#pragma unroll
    for (int y = 0; y < FN; ++y) acc[X][y] = mfma16<kMm16Pairs>(qh[S][y], ph[S][X], acc[X][y]);
  };
  auto each = [](auto f) { [&]<int... X>(std::integer_sequence<int, X...>) { (f(std::integral_constant<int, X>()), ...); }(std::make_integer_sequence<int, FM>()); };
  for (int t = 0; t < 2 && t < steps; ++t) fetch(t);
  if (steps >= 2) arrived_and_together<4 * kEach>();
  else arrived_and_together<0>();
  each([&](auto x) { read(std::integral_constant<int, 0>(), base, x); });
  // a step: its fragments are in registers, and so its half of LDS is free for the step after the next
  auto step = [&](int t, auto set) {
    constexpr int S = decltype(set)::value;
    const uint32_t here = base + S * kStage, next = base + (1 - S) * kStage;
    arrived_and_together<0>();                           // step t + 1 is in LDS
    const bool more = t + 2 < steps, whole = more && left_of(t + 2) == kBK;
    const char *p = P + (int64_t)(t + 2) * kBK * 2, *q = Q + (t + 2) * step_q;
    if (more && !whole) fetch(t + 2);
    each([&](auto x) {
      constexpr int X = decltype(x)::value;
      read(std::integral_constant<int, 1 - S>(), next, x);      // (behind the last step: of an old one, for nothing)
      if (whole) {
        if constexpr (X == 0) tp.template fetch_some<0, kEach>(p, here);
        if constexpr (X == 1) tp.template fetch_some<0, kEach>(p + lo_p, here + kP);
        if constexpr (X == 2) tq.template fetch_some<0, kEach>(q, here + 2 * kP);
        if constexpr (X == 3) tq.template fetch_some<0, kEach>(q + lo_q, here + 2 * kP + kQ);
      }
      __builtin_amdgcn_sched_barrier(0);
      products(set, x);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  int t = 0;
  for (; t + 2 <= steps; t += 2) {
    step(t, std::integral_constant<int, 0>());
    step(t + 1, std::integral_constant<int, 1>());
  }
  if (t < steps) step(t, std::integral_constant<int, 0>());
  // Both halves' sums: this wavefront keeps rows 32 half .. of its 64 x 64 and hands the others over.
  __syncthreads();
  float* given = (float*)lds_all + (wave ^ 4) * 32 * kOutPad;
  const int lane = threadIdx.x % 64;
  const auto at = [&](int x, int y) { return (16 * x + (lane & 15)) * kOutPad + 16 * y + (lane >> 4) * 4; };
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int y = 0; y < FN; ++y) *reinterpret_cast<f32x4*>(given + at(x, y)) = half ? acc[x][y] : acc[2 + x][y];
  __syncthreads();
  const float* taken = (const float*)lds_all + wave * 32 * kOutPad;
  f32x4 sum[2][FN];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int y = 0; y < FN; ++y) {
      const f32x4 other = *reinterpret_cast<const f32x4*>(taken + at(x, y));
      sum[x][y] = half ? acc[2 + x][y] + other : acc[x][y] + other;
    }
  store_sums<32, FN>(a, by, partial, lds_all, sum, b, i0 + wi + 32 * half, j0 + wj, a.symmetric && ti != tj);
}

struct Join {
  int64_t M, N, batches;
  int symmetric;
  Epilogue epi;
};

// Four sums of every share, added in order; eight shares are on their way at a time.
__device__ __forceinline__ f32x4 add_shares(const float* __restrict__ p, int64_t far, int splits) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  int z = 0;
  for (; z + 8 <= splits; z += 8) {
    f32x4 t[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) t[u] = *reinterpret_cast<const f32x4*>(p + (z + u) * far);
#pragma unroll
    for (int u = 0; u < 8; ++u) s += t[u];
  }
  f32x4 t[7];
#pragma unroll
  for (int u = 0; u < 7; ++u)
    if (z + u < splits) t[u] = *reinterpret_cast<const f32x4*>(p + (z + u) * far);
#pragma unroll
  for (int u = 0; u < 7; ++u)
    if (z + u < splits) s += t[u];
  return s;
}

// Adds the shares of k and finishes, a thread for four sums of a row.  (BY: the result has a factor.  Asking whether it has one cost every
// layer 0.3 us here.)
template <bool BY>
__global__ __launch_bounds__(256) void mm_join_rows_kernel(Join a, int splits, const float* __restrict__ partial) {
  const int64_t quads = (a.N + 3) / 4, at = (int64_t)blockIdx.x * 256 + threadIdx.x, i = at / quads, j = (at - i * quads) * 4, b = blockIdx.y;
  if (i >= a.M) return;
  const int64_t ldp = quads * 4;
  const int valid = quad_valid(i, j, a.M, a.N);
  const float by = BY ? a.epi.by[b] : 1.0f;
  const SrcQuad raw = epilogue_ask(a.epi, b, i, j, valid);
  float bias[4];
  epilogue_bias(a.epi, j, valid, bias);
  const f32x4 s = add_shares(partial + (b * a.M + i) * ldp + j, a.batches * a.M * ldp, splits);
  float v[4] = {s[0], s[1], s[2], s[3]};
  epilogue4(a.epi, by, b, i, j, valid, bias, raw, v);
}

// The same for results that are written along j too, 32 x 32 sums a workgroup: those on and above the diagonal of a symmetric
// result, or all of a flipped one.
__global__ __launch_bounds__(256) void mm_join_kernel(Join a, int tn, int splits, const float* __restrict__ partial) {
  __shared__ __attribute__((aligned(16))) float tile[32][36];
  int ti, tj;
  if (a.symmetric) upper_block(blockIdx.x, tn, &ti, &tj);
  else { ti = blockIdx.x / tn; tj = blockIdx.x % tn; }
  const int64_t b = blockIdx.y, i0 = (int64_t)ti * 32, j0 = (int64_t)tj * 32, ldp = (a.N + 3) / 4 * 4;
  const int r = threadIdx.x / 8, c = (threadIdx.x % 8) * 4;
  const float none[4] = {0.f, 0.f, 0.f, 0.f}, by = a.epi.by != nullptr ? a.epi.by[b] : 1.0f;
  const bool turned = a.epi.flip || (a.symmetric && ti != tj);
  // where this thread's quad goes, and where that of the turned tile does
  const int x = threadIdx.x % 32, y = threadIdx.x / 32 * 4;
  const int64_t ti_row = a.epi.flip ? i0 + x : j0 + r, ti_col = a.epi.flip ? j0 + y : i0 + c;
  const int valid = quad_valid(i0 + r, j0 + c, a.M, a.N), turned_valid = quad_valid(ti_row, ti_col, a.epi.flip ? a.M : a.N, a.epi.flip ? a.N : a.M);
  const SrcQuad raw = epilogue_ask(a.epi, b, i0 + r, j0 + c, a.epi.flip ? 0 : valid), turned_raw = epilogue_ask(a.epi, b, ti_row, ti_col, turned ? turned_valid : 0);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (valid > 0) s = add_shares(partial + (b * a.M + i0 + r) * ldp + j0 + c, a.batches * a.M * ldp, splits);
  if (!a.epi.flip && valid > 0) {
    float v[4] = {s[0], s[1], s[2], s[3]};
    epilogue4(a.epi, by, b, i0 + r, j0 + c, valid, none, raw, v);
  }
  if (!turned) return;
  *reinterpret_cast<f32x4*>(&tile[r][c]) = s;
  __syncthreads();
  if (turned_valid == 0) return;
  float v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = a.epi.flip ? tile[x][y + q] : tile[c + q][r];
  epilogue4(a.epi, by, b, ti_row, ti_col, turned_valid, none, turned_raw, v);
}

int64_t blocks_of(int64_t M, int64_t N, int tile, int symmetric) {
  const int64_t tm = (M + tile - 1) / tile, tn = (N + tile - 1) / tile;
  return symmetric ? tm * (tm + 1) / 2 : tm * tn;
}

hipError_t finish_shares(const Product16& a, const MmPlan& plan, float* part, hipStream_t st) {
  if (part != nullptr) return launch_mm_join(a.M, a.N, a.batches, a.symmetric, a.epi, plan.splits, part, st);
  return hipGetLastError();
}

template <bool PK, bool QK>
hipError_t mm16_order(const Product16& a, const MmPlan& plan, float* partial, hipStream_t st) {
  const int tm = (int)((a.M + plan.tile - 1) / plan.tile), tn = (int)((a.N + plan.tile - 1) / plan.tile);
  const int ks = (int)((a.K + kBK - 1) / kBK), share = (ks + plan.splits - 1) / plan.splits;
  const dim3 grid((unsigned)blocks_of(a.M, a.N, plan.tile, 0), 1, (unsigned)plan.splits);
  float* part = plan.splits > 1 ? partial : nullptr;
  Product16 l = a;
  l.past = part == nullptr && (a.epi.pre != nullptr ? 4 : 2) * a.M * a.N >= kStreamBytes;
  if (plan.tile == 256) mm16_kernel<PK, QK, 256, 256, 2, 4><<<grid, 512, 0, st>>>(l, tm, tn, share, part);
  else mm16_kernel<PK, QK, 128, 128, 2, 2><<<grid, 256, 0, st>>>(l, tm, tn, share, part);
  return finish_shares(a, plan, part, st);
}

hipError_t mm16_pairs(const Product16& a, const MmPlan& plan, float* partial, hipStream_t st) {
  const int tm = (int)((a.M + 127) / 128), tn = (int)((a.N + 127) / 128);
  const int ks = (int)((a.K + kBK - 1) / kBK), share = (ks + plan.splits - 1) / plan.splits;
  const dim3 grid((unsigned)blocks_of(a.M, a.N, 128, a.symmetric), (unsigned)a.batches, (unsigned)plan.splits);
  float* part = plan.splits > 1 ? partial : nullptr;
  const void* kernel = a.Q.k_rows ? (const void*)mm16_pairs_kernel<true> : (const void*)mm16_pairs_kernel<false>;
  if (hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kPairsLds); e != hipSuccess) return e;
  if (a.Q.k_rows) mm16_pairs_kernel<true><<<grid, 512, kPairsLds, st>>>(a, tm, tn, share, part);
  else mm16_pairs_kernel<false><<<grid, 512, kPairsLds, st>>>(a, tm, tn, share, part);
  return finish_shares(a, plan, part, st);
}

}  // namespace

hipError_t launch_mm_join(int64_t M, int64_t N, int64_t batches, int symmetric, const Epilogue& epi, int splits, const float* partial, hipStream_t st) {
  const Join a{M, N, batches, symmetric, epi};
  if (!symmetric && !epi.flip) {
    const dim3 grid((unsigned)((M * ((N + 3) / 4) + 255) / 256), (unsigned)batches);
    if (epi.by != nullptr) mm_join_rows_kernel<true><<<grid, 256, 0, st>>>(a, splits, partial);
    else mm_join_rows_kernel<false><<<grid, 256, 0, st>>>(a, splits, partial);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)blocks_of(M, N, 32, symmetric), (unsigned)batches);
  mm_join_kernel<<<grid, 256, 0, st>>>(a, (int)((N + 31) / 32), splits, partial);
  return hipGetLastError();
}

// Blocks of 256 or 128 and the shares of k, by what they cost in microseconds: a step of a 256-block takes 1.7 (one workgroup fits a
// compute unit), of a 128-block 0.75 alone on its unit and 1.08 beside another, of a 128-block of pairs (one to a unit) 0.9; shares
// are written and added at 8 TB/s, in a launch of 3.  (What every block of pairs costs besides, its start and its sums, about 20 us, is
// the same for every number of shares that is one round, and is not counted: of 2048 x 2048 x 2048 the sum is 28.8 and the kernel takes
// 52, of 1024 x 4096 x 1024 14.4 and 31.)  Measured: 1024 x 1024 x 4096, bfloat16, 128-blocks: 50 us in one share, 27 in
// four, 32 in eight; 2048 x 2048 x 2048, bfloat16: 31; 4096 x 4096 x 4096, bfloat16: 117 in 256-blocks.
MmPlan mm16_plan(int64_t M, int64_t N, int64_t K, int64_t batches, int kind, int symmetric) {
  MmPlan best{128, 1, 0};
  double least = 1e300;
  const int64_t ks = (K + kBK - 1) / kBK;
  for (int tile = kind == kMm16Pairs ? 128 : 256; tile >= 128; tile /= 2) {
    const int64_t blocks = blocks_of(M, N, tile, symmetric) * batches;
    for (int64_t splits = 1; splits <= 32 && splits <= (ks > 0 ? ks : 1); ++splits) {
      const int64_t share = (ks + splits - 1) / splits;
      if (splits > 1 && ((ks + share - 1) / share != splits || share < (kind == kMm16Pairs ? 2 : 4) || blocks * splits > 1024)) continue;   // no empty shares, no tiny ones
      const int64_t groups = blocks * splits;
      double step;
      if (kind == kMm16Pairs) step = 0.9 * (double)((groups + 255) / 256);
      else if (tile == 256) step = 1.7 * (double)((groups + 255) / 256);
      else step = 1.08 * (double)(groups / 512) + (groups % 512 == 0 ? 0.0 : groups % 512 <= 256 ? 0.75 : 1.08);
      double cost = (double)share * step;
      const double bytes = (double)splits * (double)batches * (double)M * (double)((N + 3) / 4 * 4) * 4.0;
      if (splits > 1) cost += 3.0 + 2.0 * bytes / 8e6;
      if (cost < least) {
        least = cost;
        best = {tile, (int)splits, splits > 1 ? (size_t)bytes : 0};
      }
    }
  }
  return best;
}

namespace {

// Rows of bfloat16 at any address, laid out in whole 16-byte pieces with zeros behind their end; 2^sh lanes a row.
__global__ __launch_bounds__(256) void pack16_kernel(const bf16_t* __restrict__ src, int64_t ld, int64_t rows, int64_t cols, bf16_t* __restrict__ dst, int sh) {
  const int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> sh, ldp = (cols + 7) / 8 * 8;
  if (r >= rows) return;
  for (int64_t c = (int64_t)(threadIdx.x & ((1 << sh) - 1)) * 8; c < cols; c += 8ll << sh) {
    const bf16_t* p = src + r * ld + c;
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

}  // namespace

hipError_t launch_pack16(const void* src, int64_t ld, int64_t rows, int64_t cols, void* dst, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  int sh = ilog2_ceil((cols + 7) / 8);
  if (sh > 6) sh = 6;
  const int64_t ldp = (cols + 7) / 8 * 8;
  return in_parts(((rows << sh) + 255) / 256, 256, [&](int64_t first, unsigned blocks) {
    const int64_t row = first * (256 >> sh), some = (int64_t)blocks * (256 >> sh);
    pack16_kernel<<<blocks, 256, 0, st>>>((const bf16_t*)src + row * ld, ld, rows - row < some ? rows - row : some, cols, (bf16_t*)dst + row * ldp, sh);
  });
}

hipError_t launch_mm16(const Product16& a, const MmPlan& plan, float* partial, hipStream_t st) {
  if (a.M == 0 || a.N == 0 || a.batches == 0) return hipSuccess;
  if (a.kind == kMm16Bf16) {
    if (a.symmetric || a.batches != 1 || a.epi.mode != kEpiLinear || !a.epi.out_bf16) return hipErrorInvalidValue;
    return in_blocks(a, plan.tile, plan.tile, plan.tile * 2, [&](const Product16& b) {
      if (b.P.k_rows) return b.Q.k_rows ? mm16_order<true, true>(b, plan, partial, st) : hipErrorInvalidValue;
      return b.Q.k_rows ? mm16_order<false, true>(b, plan, partial, st) : mm16_order<false, false>(b, plan, partial, st);
    });
  }
  return a.P.k_rows ? hipErrorInvalidValue : mm16_pairs(a, plan, partial, st);
}

}  // namespace ilargi
