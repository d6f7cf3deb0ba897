// Rows of logits: what the readout's operators on single rows share (internal header). A row is C values in float32,
// bfloat16 or float16 at any address its type allows; it is walked in 16-byte vectors of the aligned address below
// it, and only vectors that lie wholly inside the row are loaded as such.
#pragma once

#include "common.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <type_traits>

namespace snn {
namespace rows {

constexpr int kMaxClasses = 1 << 20;  // a row's weights of at most 2^31 sum below 2^53
constexpr int kMaxListed = 1024;      // listed classes of a teacher's record

struct Bf16 {
  uint16_t bits;
};
struct F16 {
  uint16_t bits;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float to_float(F16 x) { return (float)__builtin_bit_cast(_Float16, x.bits); }
template <class T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ Bf16 from_float<Bf16>(float x) {  // to nearest, ties to even
  return Bf16{__builtin_bit_cast(uint16_t, (__bf16)x)};
}
template <>
__device__ __forceinline__ F16 from_float<F16>(float x) {
  return F16{__builtin_bit_cast(uint16_t, (_Float16)x)};
}

template <class T>
struct Row {
  static constexpr int kVec = 16 / (int)sizeof(T);
  const T* base;  // the row's address rounded down to 16 bytes
  int lead;       // elements between base and the row
  int C;
  int Q;          // vectors that hold a part of the row

  __device__ __forceinline__ Row(const void* logits, int64_t r, int64_t ld, int C_)
      : Row(static_cast<const T*>(logits) + r * ld, C_) {}
  __device__ __forceinline__ Row(const T* p, int C_) : C(C_) {
    lead = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    base = p - lead;
    Q = (lead + C + kVec - 1) / kVec;
  }
  __device__ __forceinline__ int first(int q) const { return q * kVec - lead; }  // class of vector q's first element
  __device__ __forceinline__ bool whole(int q) const { return first(q) >= 0 && first(q) + kVec <= C; }
  __device__ __forceinline__ float at(int j) const { return to_float(base[lead + j]); }
  __device__ __forceinline__ void load(int q, float (&x)[kVec]) const;  // vector q, -inf outside the row
};

template <class T>
__device__ __forceinline__ T lowest();  // -inf
template <>
__device__ __forceinline__ float lowest<float>() {
  return -INFINITY;
}
template <>
__device__ __forceinline__ Bf16 lowest<Bf16>() {
  return Bf16{0xff80};
}
template <>
__device__ __forceinline__ F16 lowest<F16>() {
  return F16{0xfc00};
}

// Vector q of a row as it lies in memory, -inf outside the row. The ends of a row are put together in a loop: its code
// is in every pass.
template <class T>
__device__ __forceinline__ uint4 load_raw(const Row<T>& row, int q) {
  constexpr int kVec = Row<T>::kVec;
  constexpr int kBits = 8 * (int)sizeof(T);
  if (row.whole(q)) return *reinterpret_cast<const uint4*>(row.base + (size_t)q * kVec);
  uint64_t lo = 0, hi = 0;
#pragma unroll 1
  for (int i = kVec - 1; i >= 0; --i) {
    const int j = row.first(q) + i;
    T v = lowest<T>();
    if (j >= 0 && j < row.C) v = row.base[(size_t)q * kVec + i];
    uint32_t bits = 0;
    __builtin_memcpy(&bits, &v, sizeof(T));
    hi = hi << kBits | lo >> (64 - kBits);
    lo = lo << kBits | bits;
  }
  return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

// A vector that is not read again soon: past the caches, which keep what is (the rows of a second pass).
typedef uint32_t Vector4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void store_past(void* p, const uint4& u) {
  __builtin_nontemporal_store(Vector4{u.x, u.y, u.z, u.w}, static_cast<Vector4*>(p));
}

// Values of vector q back to a row, those inside it.
template <class T>
__device__ __forceinline__ void store_vec(const Row<T>& row, int q, const float (&x)[16 / sizeof(T)]) {
  constexpr int kVec = Row<T>::kVec;
  T v[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = from_float<T>(x[i]);
  T* p = const_cast<T*>(row.base) + (size_t)q * kVec;
  uint4 u;
  __builtin_memcpy(&u, v, 16);
  if (row.whole(q)) {
    store_past(p, u);
  } else {
    constexpr int kBits = 8 * (int)sizeof(T);
    uint64_t lo = (uint64_t)u.y << 32 | u.x, hi = (uint64_t)u.w << 32 | u.z;
#pragma unroll 1
    for (int i = 0; i < kVec; ++i) {
      T one;
      __builtin_memcpy(&one, &lo, sizeof(T));
      if (row.first(q) + i >= 0 && row.first(q) + i < row.C) p[i] = one;
      lo = lo >> kBits | hi << (64 - kBits);
      hi >>= kBits;
    }
  }
}

template <class T>
__device__ __forceinline__ void unpack(const uint4& u, float (&x)[16 / sizeof(T)]) {
  T v[16 / sizeof(T)];
  __builtin_memcpy(v, &u, 16);
#pragma unroll
  for (int i = 0; i < (int)(16 / sizeof(T)); ++i) x[i] = to_float(v[i]);
}

template <class T>
__device__ __forceinline__ void Row<T>::load(int q, float (&x)[kVec]) const {
  unpack<T>(load_raw(*this, q), x);
}

// Vectors q0 + i * NT + thread below q1 of a row, -inf outside. All loads are under way before anything waits: threads
// past the row's whole vectors load its last one.
template <class T, int NT, int NV>
__device__ __forceinline__ void load_vectors(const Row<T>& row, uint4 (&u)[NV], int q0, int q1) {
  constexpr int kVec = Row<T>::kVec;
  const int tid = (int)threadIdx.x;
  const int from = row.lead ? 1 : 0, to = (row.lead + row.C) / kVec;  // whole vectors
  uint4 none;
  {
    T v[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = lowest<T>();
    __builtin_memcpy(&none, v, 16);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) u[i] = none;
  if (to > from) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      u[i] = *reinterpret_cast<const uint4*>(row.base + (size_t)min(max(q0 + i * NT + tid, from), to - 1) * kVec);
  }
  uint4 first = none, last = none;  // the ends of the row
  if (q0 == 0 && from == 1 && tid == 0) first = load_raw(row, 0);
  if (to < row.Q && to >= from && to >= q0 && to < q1 && tid == (to - q0) % NT) last = load_raw(row, to);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int q = q0 + i * NT + tid;
    const bool in = q >= from && q < to && q < q1, end = q == to && to >= from && q < q1;
    uint4 e = make_uint4(end ? last.x : none.x, end ? last.y : none.y, end ? last.z : none.z, end ? last.w : none.w);
    if (i == 0) {
      const bool head = q < from;
      e = make_uint4(head ? first.x : e.x, head ? first.y : e.y, head ? first.z : e.z, head ? first.w : e.w);
    }
    u[i] = make_uint4(in ? u[i].x : e.x, in ? u[i].y : e.y, in ? u[i].z : e.z, in ? u[i].w : e.w);
  }
}

// A row in a block's registers: vector i * NT + thread of it as the words 4 i to 4 i + 3 of a register array (two of
// them beyond 8 vectors), where a load puts them without a move. Long passes over it are loops whose counter selects
// the registers: unrolled, the passes of a wide tile are straight code of tens of KB, and a block then waits for
// instructions at nearly every line (1024 rows of 65536 drawn from: 620 us unrolled, 210 so).
template <class T, int NT, int NV>
struct Tile {
  static constexpr int kVec = Row<T>::kVec;
  static constexpr int kPart = NV < 8 ? NV : 8;
  typedef uint32_t Words __attribute__((ext_vector_type(4 * kPart)));
  Words w[NV / kPart];

  __device__ __forceinline__ static uint4 take(const Words& p, int i) {
    return make_uint4(p[4 * i], p[4 * i + 1], p[4 * i + 2], p[4 * i + 3]);
  }
  __device__ __forceinline__ static void put(Words& p, int i, const uint4& u) {
    p[4 * i] = u.x;
    p[4 * i + 1] = u.y;
    p[4 * i + 2] = u.z;
    p[4 * i + 3] = u.w;
  }
  __device__ __forceinline__ uint4 get(int i) const {
    if (NV > kPart && i >= kPart) return take(w[NV / kPart - 1], i - kPart);
    return take(w[0], i);
  }
  __device__ __forceinline__ void load(const Row<T>& row) { load(row, 0, row.Q); }
  __device__ __forceinline__ void load(const Row<T>& row, int q0, int q1) {
    uint4 u[NV];
    load_vectors<T, NT>(row, u, q0, q1);
#pragma unroll
    for (int i = 0; i < NV; ++i) put(w[i / kPart], i % kPart, u[i]);
  }
  // f(values, vector, its number in the thread)
  template <class F>
  __device__ __forceinline__ void each(const Row<T>& row, F f) const {
#pragma unroll
    for (int h = 0; h < NV / kPart; ++h) {
#pragma unroll 1
      for (int i = 0; i < kPart; ++i) {
        if ((h * kPart + i) * NT >= row.Q) break;
        float x[kVec];
        unpack<T>(take(w[h], i), x);
        f(x, (h * kPart + i) * NT + (int)threadIdx.x, h * kPart + i);
      }
    }
  }
  // The same, unrolled: for a few instructions a value.
  template <class F>
  __device__ __forceinline__ void each_unrolled(const Row<T>& row, F f) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i * NT < row.Q) {
        float x[kVec];
        unpack<T>(get(i), x);
        f(x, i * NT + (int)threadIdx.x, i);
      }
  }
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Exponents of 2 relative to a largest value: fmaf(x, c, -mc) of the values x up to it. mc is the largest times c, rounded;
// 0 where there is nothing but -inf. The rounding, a factor that all of them share, is up to 2^-25 mc: from 2^31 on (masks
// of the type's lowest value, whose product may overflow as well) it would leave the range of the powers. There any
// other value lies 2^7 or more below the largest in the exponent, and its power counts for nothing: c is then a power
// of two, with which the product is exact, equals are at 0 and all others at least 2^6 below.
struct Exponent {
  float c, mc;
};
constexpr float kFarExponent = 0x1p31f;
__device__ __forceinline__ Exponent exponent_of(float most, float c) {
  float mc = most * c;
  if (fabsf(mc) >= kFarExponent) {
    if (!isinf(most)) c = ldexpf(1.0f, min(126 - ilogbf(most), 127));
    mc = most == -INFINITY ? 0.0f : most * c;
  }
  return Exponent{c, mc};
}

// Largest of the wave's values; the steps within 16 lanes and between them are operands of the maximum itself.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#define SNN_STEP(ctrl) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false))
  SNN_STEP(0x111);  // from 1, 2, 4, 8 lanes below, in rows of 16
  SNN_STEP(0x112);
  SNN_STEP(0x114);
  SNN_STEP(0x118);
  SNN_STEP(0x142);  // a row's last lane to the next row, then lane 31 to the upper half
  SNN_STEP(0x143);
#undef SNN_STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// The n-th largest of the wave's values, 1 <= n <= 64.
__device__ __forceinline__ uint32_t wave_nth(uint32_t v, int n) {
  for (;;) {
    const uint32_t m = wave_max_u32(v);
    if (--n == 0) return m;
    const int first = (int)__builtin_ctzll(__ballot(v == m));
    v = lane_id() == first ? 0 : v;
  }
}

// A value that all lanes of the wave have, in a scalar register: branches on it are branches.
__device__ __forceinline__ int same_in_wave(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float same_in_wave(float v) {
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}

// NaN as -inf: a class that is never listed or drawn.
__device__ __forceinline__ float no_nan(float x) { return x == x ? x : -INFINITY; }

// Every lane of 16 gets f over their values (f commutes). Each step's operand comes from another lane of the row in
// the instruction itself: neighbours, pairs, then the mirrored half rows and rows.
template <class F>
__device__ __forceinline__ float row16_reduce(float v, F f) {
#define SNN_STEP(ctrl) v = f(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), ctrl, 0xf, 0xf, true)))
  SNN_STEP(0xb1);
  SNN_STEP(0x4e);
  SNN_STEP(0x141);
  SNN_STEP(0x140);
#undef SNN_STEP
  return v;
}
// Rows of at most kShortRow classes go 16 lanes each, four in a wave: class 16 i + lane is the lane's value i.
constexpr int kShortRow = 128;
constexpr int kShortEach = kShortRow / 16;
constexpr int kShortRows = 16;  // of a block of 256

template <class T>
__device__ __forceinline__ void load_short(const Row<T>& row, float (&x)[kShortEach]) {
  const int l = threadIdx.x % 16;
#pragma unroll
  for (int i = 0; i < kShortEach; ++i) {
    const int j = 16 * i + l;
    x[i] = -INFINITY;
    if (16 * i < row.C) x[i] = j < row.C ? row.at(min(j, row.C - 1)) : -INFINITY;
  }
}
// Sums over the row's lanes up to each.
__device__ __forceinline__ uint64_t row16_upto64(uint64_t v);
// The lane's place among those of its row with `on`, and their number.
__device__ __forceinline__ int row16_place(bool on, int& count) {
  const uint64_t m = __ballot(on);
  const uint32_t bits = (uint32_t)(m >> (threadIdx.x % kWave / 16 * 16)) & 0xffffu;
  count = __popc(bits);
  return __popc(bits & ((1u << threadIdx.x % 16) - 1));
}

template <class F>
__device__ __forceinline__ float wave_reduce(float v, F f) {
  v = row16_reduce(v, f);
  v = f(v, __shfl_xor(v, 16, kWave));
  return f(v, __shfl_xor(v, 32, kWave));
}
struct Larger {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Plus {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// Integers in the order of the values; -0 and +0 are one.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// A 64-bit value from the lane that a step names, 0 where there is none or `rows` leaves the row of 16 out.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint64_t from_lane64(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t lane_of64(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
// Sums over the lanes up to each.
__device__ __forceinline__ uint64_t wave_upto64(uint64_t v) {
  v += from_lane64<0x111>(v);  // within rows of 16
  v += from_lane64<0x112>(v);
  v += from_lane64<0x114>(v);
  v += from_lane64<0x118>(v);
  v += from_lane64<0x142, 0xa>(v);  // rows 0 and 2 to the next, then the lower half to the upper
  v += from_lane64<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ uint64_t row16_upto64(uint64_t v) {
  v += from_lane64<0x111>(v);
  v += from_lane64<0x112>(v);
  v += from_lane64<0x114>(v);
  v += from_lane64<0x118>(v);
  return v;
}
// The value of the last lane of the row of 16.
__device__ __forceinline__ uint64_t lane_of_row16(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)v, 0x15f, 0xf, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(v >> 32), 0x15f, 0xf, 0xf, true);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) { return lane_of64(wave_upto64(v), kWave - 1); }

// Block reductions and scans; every thread of the block takes part and gets the result. `red` holds NT / kWave
// values in LDS and may be reused at once.
template <int NT, class V, class F>
__device__ __forceinline__ V block_reduce(V v, F f, V* red) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v = f(v, __shfl_xor(v, off, kWave));
  if (NT == kWave) return v;
  __syncthreads();
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = v;
  __syncthreads();
  v = red[threadIdx.x % (NT / kWave)];
#pragma unroll
  for (int off = NT / kWave / 2; off > 0; off >>= 1) v = f(v, __shfl_xor(v, off, kWave));
  return v;
}

template <int NT>
__device__ __forceinline__ uint64_t block_sum64(uint64_t v, uint64_t* red) {
  v = wave_sum64(v);
  if (NT == kWave) return v;
  __syncthreads();
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = v;
  __syncthreads();
  return wave_sum64(threadIdx.x % kWave < NT / kWave ? red[threadIdx.x % kWave] : 0);
}

template <int NT>
__device__ __forceinline__ uint64_t block_exclusive(uint64_t v, uint64_t* red) {
  const uint64_t upto = wave_upto64(v);
  const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
  __syncthreads();
  if (l == kWave - 1) red[w] = upto;
  __syncthreads();
  return wave_sum64(l < w ? red[l] : 0) + upto - v;
}

// v[0..n) in ascending order; v has room for the next power of two.
template <int NT>
__device__ __forceinline__ void block_sort(uint64_t* v, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int e = n + (int)threadIdx.x; e < size; e += NT) v[e] = UINT64_MAX;
  __syncthreads();
#pragma unroll 1
  for (int run = 2; run <= size; run <<= 1)
#pragma unroll 1
    for (int step = run >> 1; step > 0; step >>= 1) {
      for (int i = threadIdx.x; i < size / 2; i += NT) {
        const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
        const uint64_t x = v[lo], y = v[hi];
        if ((x > y) == ((lo & run) == 0)) {
          v[lo] = y;
          v[hi] = x;
        }
      }
      __syncthreads();
    }
}

// ------------------------------------------------------------------ cuts in one wave
//
// The first k of a row's order where one wave holds the row: their end is sought by halving a range of values whose
// larger end too few elements reach and whose smaller end enough. A step is one comparison a value and a count of lanes,
// without LDS, atomics or an order; it ends when k elements reach the smaller end, or with a single value, among whose
// elements the last class is sought in the same manner.

template <class T>
constexpr int kWaveVectors = 32 / Row<T>::kVec;  // 32 values a lane, 2048 classes

// Key bits that are alike in all of a type's values of one sign, and keys without them.
template <class T>
constexpr int kLow = sizeof(T) == 4 ? 0 : std::is_same<T, Bf16>::value ? 16 : 13;
template <class T>
__device__ __forceinline__ uint32_t short_key(float x) {
  return key_of(x) >> kLow<T>;
}
// A value that all elements of this short key reach and none of the one before; the elements' value.
template <class T>
__device__ __forceinline__ float least_of(uint32_t s) {
  return of_key(s << kLow<T>);
}
template <class T>
__device__ __forceinline__ float value_of(uint32_t s) {
  const uint32_t k = s << kLow<T>;
  return of_key(k >> 31 ? k : k | ((1u << kLow<T>) - 1));
}
// Between lo and hi, more than 1 apart: at first half way between the values, which lie evenly more often than their keys
// (whose half is below 1e-19 from 0 to 1); then between the keys, of which 32 steps see the end.
template <class T>
__device__ __forceinline__ uint32_t halfway(uint32_t lo, uint32_t hi, int step) {
  uint32_t mid = lo + (hi - lo) / 2;
  if (step < 8) mid = short_key<T>(0.5f * least_of<T>(lo) + 0.5f * least_of<T>(hi));
  return (uint32_t)same_in_wave((int)min(max(mid, lo + 1), hi - 1));
}

// Elements for which in(value, class).
template <class T, int NV, class F>
__device__ __forceinline__ int count_in_wave(const Tile<T, kWave, NV>& tile, const Row<T>& row, F in) {
  constexpr int kVec = Row<T>::kVec;
  int count = 0;
  tile.each_unrolled(row, [&](const float (&x)[kVec], int q, int) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) count += __popcll(__ballot(in(x[i], row.first(q) + i)));
  });
  return count;
}

// The first class c of [0, C) with enough(c), which holds for the last.
template <class F>
__device__ __forceinline__ int first_class(int C, F enough) {
  int from = -1, to = C - 1;
  while (to - from > 1) {
    const int mid = (from + to) >> 1;
    if (enough(mid)) to = mid;
    else from = mid;
  }
  return to;
}

// From lo with n_lo > k elements and top with none: the first k are those larger than cut and of its equals the classes up
// to last. lo moves to where the cut is, n_lo to the elements that reach it.
template <class T, int NV>
__device__ __forceinline__ void first_in_wave(const Tile<T, kWave, NV>& tile, const Row<T>& row, int C, int k, uint32_t& lo,
                                              uint32_t top, int& n_lo, float& cut, int& last) {
  uint32_t hi = top;
  int n_hi = 0;
  for (int step = 0; hi - lo > 1 && n_lo != k; ++step) {
    const uint32_t mid = halfway<T>(lo, hi, step);
    const float least = least_of<T>(mid);
    const int n = count_in_wave(tile, row, [&](float x, int) { return x >= least; });
    if (n >= k) {
      lo = mid;
      n_lo = n;
    } else {
      hi = mid;
      n_hi = n;
    }
  }
  cut = least_of<T>(lo);
  last = C;
  if (n_lo != k) {  // the last are some of those equal to one another
    cut = value_of<T>(lo);
    last = first_class(C, [&](int c) {
      return n_hi + count_in_wave(tile, row, [&](float x, int j) { return (x == cut) & (j <= c); }) >= k;
    });
  }
}

// ------------------------------------------------------------------ selection
//
// The order of a row's classes is by value, largest first, equal values by class. A cut is the first place of the
// order at which the sum of the weights so far reaches a limit; the weights are integers, so that no order of
// summation changes it. It is found by value: a histogram of the keys in range over kBins equal parts, whose part
// with the limit becomes the next range, until it holds few elements (each then sums what is above it) or one value.

constexpr int kShort = 512;  // elements compared with one another

template <int NT>
struct SelectLds {
  static constexpr int kBins = NT == kWave ? 256 : 1024;  // 256: many one-wave blocks of a CU share its LDS
  uint64_t mass[kBins];
  uint32_t count[kBins];
  uint32_t list[kShort], weight[kShort];
  uint64_t red[NT / kWave];
  uint64_t before_mass;
  uint32_t before_count, part_count, part, n_list;
  uint32_t cut_key, cut_equal;
};

struct Cut {
  uint32_t key;          // value at the cut
  uint64_t above_mass;   // weights and number of the elements before it with a larger value
  uint32_t above_count;
  uint32_t equal;        // elements of that value
};

// weigh(x) gives an element's weight, 0 for one that is not in the order. by_mass: limit is a sum of weights (MASS
// then), else a number of elements. The keys of the elements lie in [lo, hi] and their sum or number reaches the
// limit >= 1.
template <class T, int NT, bool MASS, class W>
__device__ __forceinline__ Cut find_cut(const Row<T>& row, W weigh, uint32_t lo, uint32_t hi, uint64_t limit,
                                        bool by_mass, SelectLds<NT>& s) {
  constexpr int kVec = Row<T>::kVec;
  constexpr int kBins = SelectLds<NT>::kBins;
  const int tid = threadIdx.x;
  uint64_t above_mass = 0;
  uint32_t above_count = 0;
  bool listing = false;  // the range is short enough to be compared element by element
  for (;;) {
    int shift = 0;
    while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
    __syncthreads();
    for (int b = tid; b < kBins; b += NT) {
      s.mass[b] = 0;
      s.count[b] = 0;
    }
    if (tid == 0) s.n_list = 0;
    __syncthreads();
#pragma unroll 1
    for (int q = tid; q < row.Q; q += NT) {
      float x[kVec];
      row.load(q, x);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float y = no_nan(x[i]);
        const uint32_t k = key_of(y);
        const uint32_t w = k >= lo && k <= hi ? weigh(y) : 0;
        if (w) {
          if (listing) {
            s.list[atomicAdd(&s.n_list, 1u)] = k;
          } else {
            const uint32_t b = (hi - k) >> shift;
            atomicAdd(&s.count[b], 1u);
            if (MASS) atomicAdd((unsigned long long*)&s.mass[b], (unsigned long long)w);
          }
        }
      }
    }
    __syncthreads();
    if (listing) break;
    constexpr int kEach = kBins / NT;
    uint64_t m = 0, n = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      m += s.mass[tid * kEach + i];
      n += s.count[tid * kEach + i];
    }
    n = above_count + block_exclusive<NT>(n, s.red);
    m = MASS ? above_mass + block_exclusive<NT>(m, s.red) : 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t c = s.count[tid * kEach + i];
      const uint64_t w = s.mass[tid * kEach + i];
      const uint64_t at = by_mass ? m : n, to = by_mass ? m + w : n + c;
      if (at < limit && to >= limit) {
        s.part = tid * kEach + i;
        s.part_count = c;
        s.before_count = (uint32_t)n;
        s.before_mass = m;
      }
      n += c;
      m += w;
    }
    __syncthreads();
    above_count = s.before_count;
    above_mass = s.before_mass;
    hi -= s.part << shift;
    const uint32_t width = (1u << shift) - 1;
    lo = hi - lo > width ? hi - width : lo;
    if (lo == hi) return Cut{hi, above_mass, above_count, s.part_count};
    listing = s.part_count <= kShort;
  }
  const int n = (int)s.n_list;
  if (MASS) {
    for (int e = tid; e < n; e += NT) s.weight[e] = weigh(of_key(s.list[e]));
    __syncthreads();
  }
  for (int e = tid; e < n; e += NT) {
    const uint32_t k = s.list[e];
    uint64_t m = above_mass;
    uint32_t c = above_count, equal = 0;
#pragma unroll 4
    for (int o = 0; o < n; ++o) {
      const uint32_t ko = s.list[o];
      c += ko > k;
      equal += ko == k;
      if (MASS) m += ko > k ? s.weight[o] : 0;
    }
    const uint64_t at = by_mass ? m : c, to = by_mass ? m + (uint64_t)equal * s.weight[e] : (uint64_t)c + equal;
    if (at < limit && to >= limit) {  // every element of the value says the same
      s.cut_key = k;
      s.cut_equal = equal;
      s.before_count = c;
      s.before_mass = m;
    }
  }
  __syncthreads();
  return Cut{s.cut_key, s.before_mass, s.before_count, s.cut_equal};
}

// The first class in the vectors [lo, hi) whose sum of f over the classes from lo to it exceeds `target`, which their
// whole sum does. f(x, class) is a weight. The range is divided among the block's waves until one wave's share is a
// vector for each lane.
template <class T, int NT, class F>
__device__ __forceinline__ int find_in_order(const Row<T>& row, F f, uint64_t target, uint64_t* red, int lo, int hi) {
  constexpr int kVec = Row<T>::kVec;
  constexpr int kWaves = NT / kWave;
  const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
  auto sum_of = [&](int q) {
    float x[kVec];
    row.load(q, x);
    uint64_t v = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int j = row.first(q) + i;
      if (j >= 0 && j < row.C) v += f(no_nan(x[i]), j);
    }
    return v;
  };
  while (hi - lo > kWave) {
    int share = (hi - lo + kWaves - 1) / kWaves;
    share = kWaves == 1 ? kWave : share;
    int pick = -1;
    for (int from = lo; from < hi && pick < 0; from += share * kWaves) {
      const int a = from + w * share, b = min(hi, a + share);
      uint64_t v = 0;
      for (int q = a + l; q < b; q += kWave) v += sum_of(q);
      v = wave_sum64(v);
      __syncthreads();
      if (l == 0) red[w] = v;
      __syncthreads();
      for (int k = 0; k < kWaves; ++k) {
        const uint64_t r = red[k];
        if (target < r) {
          pick = from + k * share;
          break;
        }
        target -= r;
      }
    }
    lo = pick;
    hi = min(hi, lo + share);
  }
  // every wave does the last step
  const uint64_t v = lo + l < hi ? sum_of(lo + l) : 0, upto = wave_upto64(v);
  const int lane = (int)__builtin_ctzll(__ballot(upto > target));
  target -= lane_of64(upto - v, lane);
  const int q = lo + lane;
  float x[kVec];
  row.load(q, x);
  int found = -1;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int j = row.first(q) + i;
    if (found < 0 && j >= 0 && j < row.C) {
      const uint64_t u = f(no_nan(x[i]), j);
      if (target < u) found = j;
      else target -= u;
    }
  }
  return found;
}

// Runs f.template run<T>() for the type that dtype names.
template <class F>
inline snn_status for_type(int dtype, F f) {
  switch (dtype) {
    case SNN_F32: return f(float{});
    case SNN_BF16: return f(Bf16{});
    case SNN_F16: return f(F16{});
  }
  return SNN_ERR_INVALID_ARG;
}

// Vectors of a row at most, over the rows of a matrix.
template <class T>
inline int most_vectors(const void* p, int C, int64_t ld) {
  constexpr int kVec = 16 / (int)sizeof(T);
  const bool aligned = reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % kVec == 0;
  return aligned ? (C + kVec - 1) / kVec : (C + 2 * kVec - 2) / kVec;
}

inline int type_size(int dtype) { return dtype == SNN_F32 ? 4 : dtype == SNN_BF16 || dtype == SNN_F16 ? 2 : 0; }

// Rows of one launch. A dispatch counts its threads in 32 bits, and a row has up to 1024 of them; a call of more rows is
// several launches. (A multiple of the rows of a block.)
constexpr int64_t kRowsAtOnce = 1 << 21;
// f(first, number) for each launch's rows, until one fails.
template <class F>
inline snn_status in_launches(int64_t R, F f) {
  snn_status ok = SNN_OK;
  for (int64_t first = 0; first < R && ok == SNN_OK; first += kRowsAtOnce)
    ok = f(first, R - first < kRowsAtOnce ? R - first : kRowsAtOnce);
  return ok;
}
template <class T>
inline T* or_null(T* p, int64_t offset) {
  return p ? p + offset : nullptr;
}

// Arguments of a matrix of rows.
inline snn_status check_rows(const void* p, int dtype, int64_t R, int C, int64_t ld) {
  const int size = type_size(dtype);
  if (!p || size == 0 || R <= 0 || C <= 0 || ld < C) return SNN_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(p) % size != 0) return SNN_ERR_INVALID_ARG;
  if (R > INT32_MAX || C > kMaxClasses || ld > INT64_MAX / 4 / R) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

}  // namespace rows
}  // namespace snn
