// Products of 16-bit matrices on the matrix cores, the sums in float32 (internal header).
//
//   D[n][m] = sum_k A(m, k) B(n, k), m next to one another in memory
//
// A block owns TILE x TILE of D: 256 by eight wavefronts of 128 m x 64 n, which has the most products a byte of LDS (1.2
// PFLOP/s at 8192 x 1024 x 32003, a large product of the library reaches 1.14 on this card), or 128 by four of 64 x 64, two
// blocks a compute unit, which fills the card with smaller problems and runs one block's end beside the other's products. A
// lane of a 16 x 16 x 32 product holds four neighbouring m of one n, so results go out in pieces of 8 or 16 bytes. A stage of
// 64 k of both operands is written to LDS by the load itself while the stage before it is multiplied; a stage costs one
// barrier.
// An operand lies in memory in one of two ways:
//   k along its rows (KS false): element (r, k) at p[r * ld + k]. In LDS a row's 128 bytes, its 16-byte pieces exchanged by
//       the row's lowest three bits, so that the 16 rows that a fragment reads are on all banks.
//   k down its rows (KS true): element (r, k) at p[k * ld + r]. In LDS a line per k, its 32-byte units (a tile's 16 rows)
//       exchanged by bits of k; ds_read_b64_tr_b16 turns 4 k x 16 rows into a lane's four k of one row on the way out.
// Operands are padded with zeros to whole tiles and begin at multiples of 16 bytes; nothing is checked in the loop.
#pragma once

#include "vectors.h"

namespace snn {
namespace gemm16 {

using rows::Bf16;
using rows::F16;

constexpr int kK = 64;     // of a stage
constexpr int kLoads = 4;  // 1 KB loads of a wavefront, operand and stage

template <int TILE>
struct Shape {
  static_assert(TILE == 256 || TILE == 128, "see Product");
  static constexpr int kThreads = 2 * TILE;
  static constexpr int kOperand = TILE * kK * 2;  // bytes of a stage's operand
  static constexpr int kLds = 4 * kOperand;
  static constexpr int kWaveM = TILE / 2, kWaveN = 64;
  static constexpr int kA = kWaveM / 16, kB = kWaveN / 16;  // 16 x 16 tiles of a wavefront
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char* LdsPtr;

template <class T>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (std::is_same<T, Bf16>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// 16 bytes a lane from base + off to LDS at lds + 16 * lane. Through asm: the compiler would wait for it before any LDS read.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}

// All of this wavefront's loads are in LDS and its LDS reads done; then those of the others too.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The exchange of a line's 32-byte units: 16 or 8 of them.
template <int TILE>
__device__ __forceinline__ int exchange(int k) {
  return ((k & 3) | ((k >> 3 & 3) << 2)) & (TILE / 16 - 1);
}

// Byte offsets of a wavefront's loads of an operand from (row 0, k 0) of a stage.
template <bool KS, int TILE>
__device__ __forceinline__ void load_offsets(int w, int l, int64_t ld, uint32_t (&off)[kLoads]) {
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int q = w * kLoads + j;
    if (KS) {
      constexpr int kLine = TILE / 8;  // 16-byte pieces of a line
      const int k = q * (kWave / kLine) + l / kLine, unit = (l % kLine) / 2;
      const int from = unit ^ exchange<TILE>(k);
      off[j] = (uint32_t)((k * ld + from * 16 + (l & 1) * 8) * 2);
    } else {
      off[j] = (uint32_t)(((8 * q + l / 8) * ld + 8 * ((l % 8) ^ (l / 8))) * 2);
    }
  }
}

// LDS offsets of a wavefront's fragments, tile `a` of 16 rows from row r0 on: what does not depend on the k step. One
// a tile with KS, one for all without (tiles are then 2048 bytes apart).
template <bool KS, int TILE, int TILES>
__device__ __forceinline__ void fragment_offsets(int r0, int l, uint32_t (&off)[TILES]) {
  const int i = l % 16, g = l / 16;
#pragma unroll
  for (int a = 0; a < TILES; ++a) {
    if (KS) {
      const int k = 8 * g + (i >> 2);
      off[a] = k * (TILE * 2) + (((r0 / 16 + a) ^ exchange<TILE>(k)) * 32) + (i & 3) * 8;
    } else {
      off[a] = (r0 + 16 * a + i) * 128 + ((g ^ (i & 7)) * 16);
    }
  }
}

template <bool KS, int TILE>
__device__ __forceinline__ s16x8 fragment(uint32_t lds, uint32_t off, int step) {
  if constexpr (KS) {
    typedef __attribute__((address_space(3))) s16x4* P;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + off + step * 32 * TILE * 2));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + off + (step * 32 + 4) * TILE * 2));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    typedef __attribute__((address_space(3))) s16x8* P;
    return *(P)(lds + (off ^ (step * 64)));  // pieces 4 g' + 4 step exchanged: bit 2 of the piece
  }
}

// This block's tile of D: sums over `stages` stages from k_first on.
template <class T, bool KSA, bool KSB, int TILE>
struct Product {
  using S = Shape<TILE>;
  f32x4 acc[S::kA][S::kB];  // tile a of m, b of n: lane l holds m = 16 a + 4 (l / 16) + v, n = 16 b + l % 16

  __device__ __forceinline__ static int wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave); }
  __device__ __forceinline__ static int m_of_wave() { return (wave() % 2) * S::kWaveM; }
  __device__ __forceinline__ static int n_of_wave() { return (wave() / 2) * S::kWaveN; }

  __device__ __forceinline__ void run(const T* A, int64_t lda, int m0, const T* B, int64_t ldb, int n0, int64_t k_first,
                                      int stages, char* smem) {
    const int w = wave(), l = lane_id();
    const uint32_t lds = (uint32_t)(uintptr_t)(LdsPtr)smem;
    uint32_t oa[kLoads], ob[kLoads];
    load_offsets<KSA, TILE>(w, l, lda, oa);
    load_offsets<KSB, TILE>(w, l, ldb, ob);
    uint32_t fa[S::kA], fb[S::kB];
    fragment_offsets<KSA, TILE, S::kA>(m_of_wave(), l, fa);
    fragment_offsets<KSB, TILE, S::kB>(n_of_wave(), l, fb);
    const T* pa = KSA ? A + k_first * lda + m0 : A + (int64_t)m0 * lda + k_first;
    const T* pb = KSB ? B + k_first * ldb + n0 : B + (int64_t)n0 * ldb + k_first;
    const int64_t step_a = KSA ? kK * lda : kK, step_b = KSB ? kK * ldb : kK;
#pragma unroll
    for (int a = 0; a < S::kA; ++a)
#pragma unroll
      for (int b = 0; b < S::kB; ++b) acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const auto load = [&](int buf) {
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds + buf * 2 * S::kOperand + w * kLoads * 1024);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) load_to_lds(pa, oa[j], to + j * 1024);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) load_to_lds(pb, ob[j], to + S::kOperand + j * 1024);
      pa += step_a;
      pb += step_b;
    };
    if (stages > 0) load(0);
    for (int s = 0; s < stages; ++s) {
      stage_barrier();
      if (s + 1 < stages) load((s + 1) & 1);
      const uint32_t at = lds + (s & 1) * 2 * S::kOperand;
#pragma unroll
      for (int step = 0; step < 2; ++step) {
        s16x8 xb[S::kB];
#pragma unroll
        for (int b = 0; b < S::kB; ++b) xb[b] = fragment<KSB, TILE>(at + S::kOperand, fb[b], step);
#pragma unroll
        for (int a = 0; a < S::kA; ++a) {
          const s16x8 xa = fragment<KSA, TILE>(at, fa[a], step);
#pragma unroll
          for (int b = 0; b < S::kB; ++b) acc[a][b] = mfma<T>(xa, xb[b], acc[a][b]);
        }
      }
    }
    stage_barrier();  // the LDS is free for what follows
  }
};

// Block -> tile: blocks are dealt to the eight XCDs in turn, each takes a run of tiles in an order of patches 8 m-tiles
// high, whose blocks share the operands' rows in its L2.
struct Tiles {
  int m, n, slice;
  bool ok;
};

__device__ __forceinline__ Tiles tile_of(int tiles_m, int tiles_n, int slices) {
  const int total = tiles_m * tiles_n * slices;
  const int per = (total + 7) / 8;
  const int t = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if (t >= total || (int)(blockIdx.x >> 3) >= per) return {0, 0, 0, false};
  const int slice = t / (tiles_m * tiles_n), u = t % (tiles_m * tiles_n);
  constexpr int kHigh = 8;
  const int patch = u / (kHigh * tiles_n), in = u % (kHigh * tiles_n);
  const int high = min(kHigh, tiles_m - patch * kHigh);
  return {patch * kHigh + in % high, in / high, slice, true};
}

inline unsigned grid_of(int tiles_m, int tiles_n, int slices) {
  return (unsigned)(((int64_t)tiles_m * tiles_n * slices + 7) / 8 * 8);
}

}  // namespace gemm16
}  // namespace snn
