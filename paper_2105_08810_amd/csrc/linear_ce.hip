// Softmax cross entropy of linear logits against one target a row, with the gradients of both factors.
//
//   z = x W  [R,C],  lse_r = log sum_c exp z_rc,  L_r = lse_r - z_r,target,  loss = sum_r w_r L_r
//   dz_rc = w_r (exp(z_rc - lse_r) - [c = target_r]),  dx = dz W^T,  dW = x^T dz
//
// With m_r the largest logit and o_r = sum over c != target of exp(z_rc - m_r), e_r = exp(z_r,target - m_r), s_r = o_r + e_r:
// dz_rc = w_r exp(z_rc - m_r) / s_r, dz_r,target = -w_r o_r / s_r, and L_r = log(1 + o_r) where the target is the largest. So
// nothing is rounded at the size of the logits, and no 1 is taken from a probability near 1: exp(z - lse) - 1 with lse in
// float32 was 0.07% off for rows of 99.96% at logits near 0, 76% at logits near 300.
//
// The classes are taken in pieces of a bounded number of logits: each piece's logits are formed, give their share of every
// row's sum of exponentials and are dropped; with the rows' sums known a piece's logits are formed again (in float32 unless
// there is one piece) and turned into its columns of dz, from which its share of dx and its columns of dW follow. Rows without a target (or of weight 0) take no part, whatever they hold.
#include <algorithm>

#include "gemm16.h"

namespace snn {
namespace {

using namespace vectors;

constexpr int kMaxRows = 1 << 24;
constexpr int kMaxHidden = 1 << 16;
// ------------------------------------------------------------------ float32

constexpr int64_t kPiece = (int64_t)1 << 27;  // logits of a piece
constexpr int kWaves = 4;                     // rows of a block in the kernels with a wavefront a row
constexpr int kCountParts = 256;

__device__ __forceinline__ bool takes_part(const int32_t* targets, const float* weight, int r, int C) {
  const int32_t t = targets[r];
  return t >= 0 && t < C && (!weight || weight[r] != 0.0f);
}

// Bit r of live: whether row r takes part (0 behind the last); parts[block]: how many of the block's rows do.
__global__ __launch_bounds__(256) void ce_live(const int32_t* __restrict__ targets, const float* __restrict__ weight, int R,
                                               int C, uint64_t* __restrict__ live, int32_t* __restrict__ parts) {
  int n = 0;
  for (int r0 = blockIdx.x * 256 + (threadIdx.x & ~(kWave - 1)); r0 < R; r0 += gridDim.x * 256) {
    const int r = r0 + lane_id();
    const uint64_t on = __ballot(r < R && takes_part(targets, weight, r, C));
    if (lane_id() == 0) live[r0 / 64] = on;
    n += __popcll(on);
  }
  __shared__ int all[256 / kWave];
  if (lane_id() == 0) all[threadIdx.x / kWave] = n;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.x] = all[0] + all[1] + all[2] + all[3];
}

__device__ __forceinline__ bool alive(const uint64_t* live, int r) { return live[r >> 6] >> (r & 63) & 1; }

// A row's weight where all that take part weigh the same: one over their number, from ce_live's n parts. A wavefront calls.
__device__ __forceinline__ float same_weight(const int32_t* __restrict__ parts, int n) {
  int s = 0;
  for (int k = lane_id(); k < n; k += kWave) s += parts[k];
  s = wave_sum_int(s);
  return s > 0 ? 1.0f / (float)s : 0.0f;
}

// A row's loss and 1 / s from its largest logit m, the sum o over the other classes and the target's logit.
__device__ __forceinline__ float finish_row(float m, float o, float zt, float& inv) {
  const float from = m > -INFINITY ? m : 0.0f;
  const float s = o + expf(zt - from);
  inv = 1.0f / s;
  // a row of infinities is NaN, as s is
  return zt == m && fabsf(m) < INFINITY ? log1pf(o) : (m - zt) + logf(s);
}

// A piece's share of every row's largest logit and sum of exponentials of classes that are not the target, and the target's
// logit.
__global__ __launch_bounds__(kWaves * kWave) void ce_sums(const float* __restrict__ z, int R, int n, int ld, int c0,
                                                          const int32_t* __restrict__ targets,
                                                          const uint64_t* __restrict__ live, float* __restrict__ top,
                                                          float* __restrict__ sum, float* __restrict__ at_target) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R || !alive(live, r)) return;
  const float* row = z + (size_t)r * ld;
  const int l = lane_id();
  float m = -INFINITY;
  for (int i = l; i < n; i += kWave) m = fmaxf(m, row[i]);  // a NaN is left to the sum
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
  const float ref = m > -INFINITY ? m : 0.0f;
  const int t = targets[r] - c0;
  float s = 0.0f;
  for (int i = l; i < n; i += kWave) s += i == t ? 0.0f : expf(row[i] - ref);
  s = wave_sum(s);
  if (l == 0) {
    if (c0 > 0) {
      const float m0 = top[r], s0 = sum[r];
      const float both = fmaxf(m0, m), from = both > -INFINITY ? both : 0.0f;
      s = s0 * expf(m0 - from) + s * expf(m - from);
      m = both;
    }
    top[r] = m;
    sum[r] = s;
    if (t >= 0 && t < n) at_target[r] = row[t];
  }
}

// Sum of a block's values in float64, in a fixed order; the first thread has it.
__device__ __forceinline__ double block_total(double s) {
  __shared__ double all[256];
  __syncthreads();
  all[threadIdx.x] = s;
  __syncthreads();
  for (int off = 128; off > 0; off >>= 1) {
    if ((int)threadIdx.x < off) all[threadIdx.x] += all[threadIdx.x + off];
    __syncthreads();
  }
  return all[0];
}

__device__ __forceinline__ void total_of(const double* __restrict__ parts, int n, float* __restrict__ loss) {
  double s = 0.0;
  for (int k = threadIdx.x; k < n; k += 256) s += parts[k];
  s = block_total(s);
  if (threadIdx.x == 0) *loss = (float)s;
}

__global__ __launch_bounds__(256) void ce_total(const double* __restrict__ parts, int n, float* __restrict__ loss) {
  total_of(parts, n, loss);
}

// Reduction over a wavefront or a block of L threads, the same in every one.
template <int L>
__device__ __forceinline__ float row_reduce(float v, bool sum, float* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const float o = __shfl_xor(v, off, kWave);
    v = sum ? v + o : fmaxf(v, o);
  }
  if constexpr (L > kWave) {
    __syncthreads();  // what was there has been read
    if (lane_id() == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int k = 1; k < L / kWave; ++k) v = sum ? v + red[k] : fmaxf(v, red[k]);
  }
  return v;
}

// A single piece's logits to dz (with GRAD) in one launch: log-sum-exp, loss and gradient of a row by L threads, a wavefront
// or a block of 1024 (7 rows of 9000: 8 us against 95 by wavefronts), its values in Q float4 of each (Q 0: rows beyond that
// are read for every pass). The logits are the sums of `slices` K slices, z_split apart; dz goes to the first. ld is a
// multiple of 4, and rows are read past n.
constexpr int kRowByBlock = 1024;    // classes from which a block takes a row
constexpr int kRowInRegs = 32768;    // classes up to which it keeps it
template <bool GRAD, int L, int Q>
__global__ __launch_bounds__(L > 256 ? L : 256) void ce_rows(float* __restrict__ z, int slices, size_t z_split, int R, int n,
                                                             int ld, const int32_t* __restrict__ targets,
                                                             const uint64_t* __restrict__ live,
                                                             const int32_t* __restrict__ counts, int n_counts,
                                                             const float* __restrict__ weight,
                                                             float* __restrict__ row_loss, double* __restrict__ parts) {
  constexpr int G = L > 256 ? 1 : 256 / L;
  __shared__ double all[G];
  __shared__ float red[L / kWave];
  const int w = threadIdx.x / L, l = threadIdx.x % L;
  const float same = weight ? 0.0f : same_weight(counts, n_counts);
  double weighted = 0.0;
  for (int r = blockIdx.x * G + w; r < R; r += gridDim.x * G) {  // with L > 64 a block is one row
    float* row = z + (size_t)r * ld;
    const bool on = alive(live, r);
    const float k = !on ? 0.0f : weight ? weight[r] : same;
    float loss = 0.0f, from = 0.0f, inv = 0.0f, rest = 0.0f;  // rest: the others' sum over all
    const int t = on ? targets[r] : -1;
    float4 held[Q > 0 ? Q : 1];
    const auto each = [&](auto f) {
      if constexpr (Q > 0) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
          if (4 * (q * L + l) < n) f(4 * (q * L + l), held[q]);
      } else {
#pragma unroll 4
        for (int i = 4 * l; i < n; i += 4 * L) {
          const float4 v = *reinterpret_cast<const float4*>(row + i);
          f(i, v);
        }
      }
    };
    if (on) {
      float zt = row[t];
      for (int p = 1; p < slices; ++p) zt += row[p * z_split + t];
      if constexpr (Q > 0) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
          if (4 * (q * L + l) < n) held[q] = *reinterpret_cast<const float4*>(row + 4 * (q * L + l));
        for (int p = 1; p < slices; ++p)
#pragma unroll
          for (int q = 0; q < Q; ++q)
            if (4 * (q * L + l) < n) {
              const float4 v = *reinterpret_cast<const float4*>(row + p * z_split + 4 * (q * L + l));
              held[q].x += v.x; held[q].y += v.y; held[q].z += v.z; held[q].w += v.w;
            }
      }
      float m = -INFINITY;
      each([&](int i, const float4& q) {  // a NaN is left to the sum
        m = fmaxf(m, q.x);
        if (i + 1 < n) m = fmaxf(m, q.y);
        if (i + 2 < n) m = fmaxf(m, q.z);
        if (i + 3 < n) m = fmaxf(m, q.w);
      });
      m = row_reduce<L>(m, false, red);
      from = m > -INFINITY ? m : 0.0f;
      float o = 0.0f;
      each([&](int i, const float4& q) {
        const float p[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (i + u < n && i + u != t) o += expf(p[u] - from);
      });
      o = row_reduce<L>(o, true, red);  // every thread has read row[t]
      loss = finish_row(m, o, zt, inv);
      rest = o * inv;
      weighted += (double)k * (double)loss;
    }
    if (l == 0 && row_loss) row_loss[r] = loss;
    if (GRAD) {
      if constexpr (L == kWave) __builtin_amdgcn_wave_barrier();
      const auto store = [&](int i, const float4& q) {
        const float p[4] = {q.x, q.y, q.z, q.w};
        float d[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) d[u] = on ? k * (i + u == t ? -rest : expf(p[u] - from) * inv) : 0.0f;
        *reinterpret_cast<float4*>(row + i) = make_float4(d[0], d[1], d[2], d[3]);  // the row's own padding past n
      };
      if (on) each(store);
      else
        for (int i = 4 * l; i < n; i += 4 * L) *reinterpret_cast<float4*>(row + i) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
  }
  if (l == 0) all[w] = weighted;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 1; q < G; ++q) weighted += all[q];
    parts[blockIdx.x] = weighted;
  }
}

// The last launch: block 0 adds up the loss, the others clear dx in the rows that take no part (dx NULL: none), a wavefront
// in those of 16 rows.
constexpr int kClearRows = 16;
__global__ __launch_bounds__(kWaves * kWave) void ce_finish(const double* __restrict__ parts, int n,
                                                            float* __restrict__ loss, const uint64_t* __restrict__ live,
                                                            int R, int H, float* __restrict__ dx, int64_t ld) {
  if (blockIdx.x == 0) {
    total_of(parts, n, loss);
    return;
  }
  const int r0 = (((int)blockIdx.x - 1) * kWaves + threadIdx.x / kWave) * kClearRows;
  if (r0 >= R) return;
  uint32_t dead = ~(uint32_t)(live[r0 >> 6] >> (r0 & 63)) & ((1u << min(R - r0, kClearRows)) - 1);
  const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  while (dead) {
    float* row = dx + (int64_t)(r0 + __builtin_ctz(dead)) * ld;
    dead &= dead - 1;
    for (int i = 4 * lane_id(); i < H; i += 4 * kWave) store_in<float, 4>(row, i, H, zero);
  }
}

// dx from its K slices, 0 in rows that take no part: a block takes 64 h of a row, its wavefronts a quarter of the slices each.
__global__ __launch_bounds__(kWaves * kWave) void ce_dx(const float* __restrict__ part, int slices,
                                                        const uint64_t* __restrict__ live, int R, int H,
                                                        float* __restrict__ dx, int64_t ld) {
  __shared__ float all[kWaves][kWave];
  const int w = threadIdx.x / kWave, l = lane_id();
  const int r = blockIdx.x, i = blockIdx.y * kWave + l;
  const int share = (slices + kWaves - 1) / kWaves;
  float s = 0.0f;
  if (i < H && alive(live, r)) {
#pragma unroll 4
    for (int k = w * share; k < min(slices, (w + 1) * share); ++k) s += part[((size_t)k * R + r) * H + i];
  }
  all[w][l] = s;
  __syncthreads();
  if (w == 0 && i < H) dx[(int64_t)r * ld + i] = (s + all[1][l]) + (all[2][l] + all[3][l]);
}

// Each row's 1 / s and loss; the weighted losses of a block in float64.
__global__ __launch_bounds__(256) void ce_losses(int R, const uint64_t* __restrict__ live, const int32_t* __restrict__ counts,
                                                 int n_counts, const float* __restrict__ weight,
                                                 const float* __restrict__ top, const float* __restrict__ sum,
                                                 const float* __restrict__ at_target, float* __restrict__ inv,
                                                 float* __restrict__ row_loss, double* __restrict__ parts) {
  const float same = weight ? 0.0f : same_weight(counts, n_counts);
  double s = 0.0;
  for (int r = blockIdx.x * 256 + threadIdx.x; r < R; r += gridDim.x * 256) {
    float loss = 0.0f;
    if (alive(live, r)) {
      loss = finish_row(top[r], sum[r], at_target[r], inv[r]);
      s += (double)(weight ? weight[r] : same) * (double)loss;
    }
    if (row_loss) row_loss[r] = loss;
  }
  s = block_total(s);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// z to dz in place; 0 in rows that take no part.
__global__ __launch_bounds__(kWaves * kWave) void ce_dz(float* __restrict__ z, int R, int n, int ld, int c0,
                                                        const int32_t* __restrict__ targets,
                                                        const uint64_t* __restrict__ live,
                                                        const int32_t* __restrict__ counts, int n_counts,
                                                        const float* __restrict__ weight, const float* __restrict__ top,
                                                        const float* __restrict__ sum, const float* __restrict__ inv) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R) return;
  float* row = z + (size_t)r * ld;
  const bool on = alive(live, r);
  const float k = weight ? weight[r] : same_weight(counts, n_counts);
  const float m = on ? top[r] : 0.0f, from = m > -INFINITY ? m : 0.0f, over = on ? inv[r] : 0.0f;
  const float rest = on ? sum[r] * over : 0.0f;
  const int t = targets[r] - c0;
  for (int i = lane_id(); i < n; i += kWave) row[i] = on ? k * (i == t ? -rest : expf(row[i] - from) * over) : 0.0f;
}

// A piece's columns of dW from its K slices, summed in order, 16 under way (64 slices of 1024 x 100: 21 us -> 7). With loss
// the first block also adds that up.
__global__ __launch_bounds__(256) void ce_dw(const float* __restrict__ part, int slices, int H, int n,
                                             float* __restrict__ dW, int64_t ld, const double* __restrict__ parts,
                                             int n_parts, float* __restrict__ loss) {
  if (loss && blockIdx.x == 0) total_of(parts, n_parts, loss);
  const size_t all = (size_t)H * n;
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (size_t)gridDim.x * 256) {
    double s = 0.0;
#pragma unroll 16
    for (int k = 0; k < slices; ++k) s += (double)part[k * all + e];
    dW[(int64_t)(e / n) * ld + e % n] = (float)s;
  }
}

// Few classes (up to kFew) of many float32 rows: everything of a row but dW in one launch. A block of four wavefronts takes
// 64 RT rows, a wavefront 16 RT of them and all classes, on the bf16 matrix cores with both operands in three parts (h + m + l, the six
// products down to 2^-16 of the leading one; values below 2^-110 lose some of their last bits, one of 2^128 - 2^119 and more
// counts as infinite). m is the class and n the row, so the accumulators hold every class of a row in four lanes:
// log-sum-exp, loss and dz are formed there, and, as a lane has four neighbouring classes of one row, its dz are the second
// product's operand as they stand: dx = dz W^T. So x is read and dx written once, and of the logits only dz leaves the
// registers (for dW). W's parts are made beforehand in the order of both products (ce_few_parts). Bound: the matrix cores
// (12 products of 128000 x 1024 x 112 in bf16 terms: 150 us at their nominal rate) beside reading x and writing dx (205 us);
// measured 320 to 365.
constexpr int kFew = 128;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ void split8(const float (&x)[8], uint4 (&part)[3]) {
  uint32_t w[3][4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float a = x[2 * q], b = x[2 * q + 1];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      w[p][q] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
      a -= __uint_as_float(w[p][q] << 16);
      b -= __uint_as_float(w[p][q] & 0xffff0000u);
    }
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) part[p] = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
}

// Term t of a product of parts: the five smaller ones, smallest first, then the leading one (to an accumulator of its own).
constexpr int kTerms = 6;
__device__ __forceinline__ void mfma_term(int t, const uint4 (&a)[3], const uint4 (&b)[3], f32x4& lead, f32x4& rest) {
  constexpr int kTerm[kTerms][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
  f32x4& c = t == kTerms - 1 ? lead : rest;
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[kTerm[t][0]]),
                                              __builtin_bit_cast(bf16x8, b[kTerm[t][1]]), c, 0, 0, 0);
}

// W's parts, zeros past its ends. For the first product [stage of 32 h][part][h / 8 % 4][class], 8 h of one class each; for
// the second [stage of 32 h][part][32-class step][g][h], of one h the 8 classes 32 step + 4 g + v and 16 more.
template <int NT>
__global__ __launch_bounds__(256) void ce_few_parts(const float* __restrict__ W, int64_t ld, int H, int C,
                                                    uint4* __restrict__ first, uint4* __restrict__ second) {
  constexpr int Cp = NT * 16, S = (NT + 1) / 2;
  const int stage = blockIdx.x;
  for (int q = threadIdx.x; q < 4 * Cp + 32 * 4 * S; q += 256) {
    float x[8];
    uint4 part[3];
    if (q < 4 * Cp) {
      const int kc = q / Cp, c = q % Cp;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int h = stage * 32 + 8 * kc + u;
        x[u] = h < H && c < C ? W[(int64_t)h * ld + c] : 0.0f;
      }
      split8(x, part);
#pragma unroll
      for (int p = 0; p < 3; ++p) first[((size_t)stage * 3 + p) * 4 * Cp + q] = part[p];
    } else {
      const int at = q - 4 * Cp, h = stage * 32 + at % 32, g = at / 32 % 4, step = at / 128;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int c = 32 * step + 16 * (u / 4) + 4 * g + u % 4;
        x[u] = h < H && c < C ? W[(int64_t)h * ld + c] : 0.0f;
      }
      split8(x, part);
#pragma unroll
      for (int p = 0; p < 3; ++p) second[((size_t)stage * 3 + p) * 128 * S + at] = part[p];
    }
  }
}

template <int NT, int RT, bool VEC>  // 16-class tiles, 16-row tiles of a wavefront; whether H is a multiple of 8
__global__ __launch_bounds__(256, 2) void ce_few(const float* __restrict__ x, int64_t ld_x, const uint4* __restrict__ first,
                                                 const uint4* __restrict__ second, int R, int H, int C,
                                                 const int32_t* __restrict__ targets, const float* __restrict__ weight,
                                                 const int32_t* __restrict__ counts, int n_counts,
                                                 float* __restrict__ row_loss, double* __restrict__ parts,
                                                 float* __restrict__ dx, int64_t ld_dx, float* __restrict__ dz, int ld_dz,
                                                 uint64_t* __restrict__ live) {
  constexpr int kRows = 64 * RT, Cp = NT * 16, S = (NT + 1) / 2;
  // pieces of a stage of W, two stages in LDS: lines [part][g] of its classes, or [part][step][g] of 32 h
  constexpr int kW1 = 12 * Cp, kW2 = 3 * 128 * S, kW = kW1 > kW2 ? kW1 : kW2;
  __shared__ __attribute__((aligned(1024))) uint4 Ws[2][kW];
  __shared__ int32_t on[kRows];
  const int w = threadIdx.x / kWave, l = lane_id(), i = l % 16, g = l / 16;
  const int r0 = blockIdx.x * kRows;
  const float same = weight ? 0.0f : same_weight(counts, n_counts);
  bool alive = false;
  if (threadIdx.x < kRows) {
    const int q = r0 + threadIdx.x;
    alive = q < R && takes_part(targets, weight, q, C);
    on[threadIdx.x] = alive;
    const uint64_t bits = __ballot(alive);
    if (live && l == 0 && q < R) live[q / 64] = bits;
  }
  const bool any = __syncthreads_or(alive);
  f32x4 lead[NT][RT], rest[NT][RT];
#pragma unroll
  for (int a = 0; a < NT; ++a)
#pragma unroll
    for (int b = 0; b < RT; ++b) lead[a][b] = rest[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int wave = __builtin_amdgcn_readfirstlane(w);
  const uint32_t lds = (uint32_t)(uintptr_t)(gemm16::LdsPtr)(char*)&Ws[0][0];
  const auto load_w = [&](const uint4* from, int n, int buf) {  // straight into LDS, 64 pieces at a time
    for (int q = wave; q < n / kWave; q += 4)
      gemm16::load_to_lds(from, (uint32_t)(q * kWave + l) * 16, __builtin_amdgcn_readfirstlane(lds + (buf * kW + q * kWave) * 16));
  };
  // A lane's part of a stage of x: 8 h of one row of each of its tiles, the second product operand as it stands. Past H
  // any of the row's values will do, since W is 0 there; rows that take no part have results that nothing uses.
  const float* px[RT];
#pragma unroll
  for (int b = 0; b < RT; ++b) px[b] = x + (int64_t)min(r0 + 16 * (RT * w + b) + i, R - 1) * ld_x;
  float xe[RT][8];
  const auto load_x = [&](int h0) {
#pragma unroll
    for (int b = 0; b < RT; ++b) {
      if constexpr (VEC) {
#pragma unroll
        for (int q = 0; q < 2; ++q) __builtin_memcpy(xe[b] + 4 * q, px[b] + min(h0 + 8 * g + 4 * q, H - 4), 16);
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) xe[b][u] = px[b][min(h0 + 8 * g + u, H - 1)];
      }
    }
  };
  // every block begins at another stage: rows are often a power of two apart, and blocks at the same h would meet in the
  // same memory channels
  const int stages = (H + 31) / 32, begin = (int)(blockIdx.x % stages);
  if (any) {
    load_w(first + (size_t)begin * kW1, kW1, 0);
    load_x(32 * begin);
    for (int n = 0, at = begin; n < stages; ++n) {
      at = at + 1 == stages ? 0 : at + 1;  // the stage after this one
      uint4 fb[RT][3];
#pragma unroll
      for (int b = 0; b < RT; ++b) split8(xe[b], fb[b]);
      gemm16::stage_barrier();  // this stage of W is there, the one before has been read
      if (n + 1 < stages) {
        load_w(first + (size_t)at * kW1, kW1, (n + 1) & 1);
        load_x(32 * at);
      }
      const uint4* W1 = Ws[n & 1];
#pragma unroll
      for (int a = 0; a < NT; a += 2) {  // neighbours in the issue order go to different accumulators
        uint4 fa[2][3];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int p = 0; p < 3; ++p)
            if (a + q < NT) fa[q][p] = W1[(4 * p + g) * Cp + 16 * (a + q) + i];
#pragma unroll
        for (int t = 0; t < kTerms; ++t)
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int b = 0; b < RT; ++b)
              if (a + q < NT) mfma_term(t, fa[q], fb[b], lead[a + q < NT ? a + q : 0][b], rest[a + q < NT ? a + q : 0][b]);
      }
    }
  }
  // lane (i, g) holds rows i of the wavefront's tiles, classes 16 a + 4 g + v
  double total = 0.0;
  // dz / w enters the second product raised by the power of two that brings the row's largest, the others' share, to [1, 2)
  // (of a share below 2^-126: to below 2): its parts keep their bits, and products overflow where dx would
  uint4 fz[RT][S][3];
  float k[RT], down[RT];
#pragma unroll
  for (int b = 0; b < RT; ++b) {
    const int at = 16 * (RT * w + b) + i, r = r0 + at;
    const bool mine = on[at];
    const int t = mine ? targets[r] : -1;
    float m = -INFINITY, zt = 0.0f;
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int c = 16 * a + 4 * g + v;
        lead[a][b][v] += rest[a][b][v];
        if (c < C) m = fmaxf(m, lead[a][b][v]);
        if (c == t) zt = lead[a][b][v];
      }
    m = fmaxf(m, __shfl_xor(m, 16, kWave));
    m = fmaxf(m, __shfl_xor(m, 32, kWave));
    zt += __shfl_xor(zt, 16, kWave);
    zt += __shfl_xor(zt, 32, kWave);
    const float from = m > -INFINITY ? m : 0.0f;
    float o = 0.0f;
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int c = 16 * a + 4 * g + v;
        o += c < C && c != t ? expf(lead[a][b][v] - from) : 0.0f;
      }
    o += __shfl_xor(o, 16, kWave);
    o += __shfl_xor(o, 32, kWave);
    float inv;
    const float of_row = finish_row(m, o, zt, inv), rest_of = o * inv;
    const float loss = mine ? of_row : 0.0f;
    k[b] = mine ? (weight ? weight[r] : same) : 0.0f;
    if (g == 0 && r < R && row_loss) row_loss[r] = loss;
    if (g == 0 && mine) total += (double)k[b] * (double)loss;
    if (!dx && !dz) continue;
    const uint32_t exponent = min(max(__float_as_uint(rest_of) >> 23 & 255u, 1u), 253u);
    const float up = __uint_as_float((254u - exponent) << 23);
    down[b] = __uint_as_float(exponent << 23);
#pragma unroll
    for (int step = 0; step < S; ++step) {
      float d[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int a = 2 * step + u / 4, c = 16 * a + 4 * g + u % 4;
        const float share = c == t ? -rest_of : expf(lead[a < NT ? a : 0][b][u % 4] - from) * inv;
        d[u] = a < NT && mine && c < C ? share : 0.0f;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int c = 16 * (2 * step + half) + 4 * g;
        if (dz && r < R && c < ld_dz)
          *reinterpret_cast<f32x4*>(dz + (size_t)r * ld_dz + c) =
              f32x4{k[b] * d[4 * half], k[b] * d[4 * half + 1], k[b] * d[4 * half + 2], k[b] * d[4 * half + 3]};
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) d[u] *= up;
      split8(d, fz[b][step]);
    }
  }
  total = block_total(total);
  if (threadIdx.x == 0) parts[blockIdx.x] = total;
  if (!dx) return;
  if (any) load_w(second + (size_t)begin * kW2, kW2, 0);  // (the losses' total has passed barriers since the last reads)
  for (int n = 0, at = begin; n < stages; ++n) {
    const int h0 = 32 * at;
    at = at + 1 == stages ? 0 : at + 1;
    f32x4 d[2][RT], e[2][RT];
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int b = 0; b < RT; ++b) d[half][b] = e[half][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (any) {
      gemm16::stage_barrier();
      if (n + 1 < stages) load_w(second + (size_t)at * kW2, kW2, (n + 1) & 1);
      const uint4* W2 = Ws[n & 1];
#pragma unroll
      for (int step = 0; step < S; ++step) {
        uint4 fa[2][3];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int p = 0; p < 3; ++p) fa[half][p] = W2[((p * S + step) * 4 + g) * 32 + 16 * half + i];
#pragma unroll
        for (int t = 0; t < kTerms; ++t)
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int b = 0; b < RT; ++b) mfma_term(t, fa[half], fz[b][step], d[half][b], e[half][b]);
      }
    }
#pragma unroll
    for (int b = 0; b < RT; ++b) {
      const int at = 16 * (RT * w + b) + i, r = r0 + at;
      if (r >= R) continue;
      const bool mine = on[at];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float o[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) o[v] = mine ? (d[half][b][v] + e[half][b][v]) * down[b] * k[b] : 0.0f;
        store_in<float, 4>(dx + (int64_t)r * ld_dx, min(h0 + 16 * half + 4 * g, H), H, o);
      }
    }
  }
}

// Few rows too (up to kFewDwRows): the float32 matrix cores, straight from memory, both products and all between in one
// launch. A block takes 16 rows; its 16 wavefronts every sixteenth run of 16 h of the first product (their sums are added in
// LDS, in order), a row each of what follows, and every sixteenth run of 16 h of dx. Bound: latency, and W read twice a block.
// A lane reads V = 1, 2 or 4 neighbouring classes at once, which are one element each of V tiles: class m of tile a is
// class_of(m) + a. The last lanes' begin early where the classes end, so that some classes are formed twice, alike.
// Few rows are 4096: us a call so and by the ways of more rows (rows x H x classes): float32 4096 x 200 x 10 40, 34; x 1024 x
// 10 51, 76; x 200 x 100 63, 62; x 1024 x 100 94, 117; 8192 x 200 x 10 75, 34; x 1024 x 10 92, 99; x 1024 x 100 182, 136;
// bfloat16 4096 x 200 x 10 40, 55; x 200 x 100 60, 56; x 1024 x 100 80, 78; 8192 x 1024 x 10 88, 92; x 200 x 100 117, 67.
constexpr int kFewDwRows = 4096;
template <int NT>
constexpr int kV = NT < 4 ? NT : 4;
template <int V>
__device__ __forceinline__ int class_of(int group, int m, int C) { return min(16 * V * group + V * m, max(C - V, 0)); }

template <class T, int NT>
__global__ __launch_bounds__(1024) void ce_small(const T* __restrict__ x, int64_t ld_x, const T* __restrict__ W, int64_t ld_w,
                                                 int R, int H, int C, const int32_t* __restrict__ targets,
                                                 const float* __restrict__ weight, float* __restrict__ row_loss,
                                                 double* __restrict__ parts, T* __restrict__ dx, int64_t ld_dx,
                                                 float* __restrict__ dz, int ld_dz, uint64_t* __restrict__ live) {
  constexpr int Cp = NT * 16;
  __shared__ float sum[16][Cp][17];  // of a wavefront: class, row
  __shared__ float d[16][Cp + 4];    // row, class
  __shared__ int count[16];
  __shared__ double losses[16];
  __shared__ bool on[16];
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), l = lane_id(), i = l % 16, g = l / 16;
  const int r0 = blockIdx.x * 16;
  int n = 0;
  if (!weight)
    for (int q = threadIdx.x; q < R; q += 1024) n += takes_part(targets, weight, q, C);
  n = wave_sum_int(n);
  if (l == 0) count[w] = n;
  // lane (i, g) multiplies h0 + 4 g + s in step s: of row i of x, of its classes of W
  constexpr int V = kV<NT>;
  int at[NT / V];
#pragma unroll
  for (int q = 0; q < NT / V; ++q) at[q] = class_of<V>(q, i, C);
  const T* px = x + (int64_t)min(r0 + i, R - 1) * ld_x;
  f32x4 acc[NT];
#pragma unroll
  for (int a = 0; a < NT; ++a) acc[a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int h0 = 16 * w; h0 < H; h0 += 256) {
    float xv[4], wv[4][NT / V][V];
    if (h0 + 16 <= H) {
      load<T, 4>(px + h0 + 4 * g, xv);
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) xv[s] = h0 + 4 * g + s < H ? to_float(px[h0 + 4 * g + s]) : 0.0f;
    }
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int q = 0; q < NT / V; ++q) load<T, V>(W + (int64_t)min(h0 + 4 * g + s, H - 1) * ld_w + at[q], wv[s][q]);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int a = 0; a < NT; ++a)
        acc[a] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[s][a / V][a % V], xv[s], acc[a], 0, 0, 0);
  }
#pragma unroll
  for (int a = 0; a < NT; ++a)
#pragma unroll
    for (int v = 0; v < 4; ++v) sum[w][class_of<V>(a / V, 4 * g + v, C) + a % V][i] = acc[a][v];
  __syncthreads();
  {  // row r0 + w, classes l and l + 64
    const int r = r0 + w;
    const bool mine = r < R && takes_part(targets, weight, r, C);
    const int t = mine ? targets[r] : -1;
    int takes = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) takes += count[q];
    const float k = !mine ? 0.0f : weight ? weight[r] : 1.0f / (float)takes;
    constexpr int Q = (Cp + kWave - 1) / kWave;
    float z[Q], m = -INFINITY, zt = 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = q * kWave + l;
      z[q] = 0.0f;
      if (c < C) {
#pragma unroll
        for (int p = 0; p < 16; ++p) z[q] += sum[p][c][w];
        m = fmaxf(m, z[q]);  // a NaN is left to the sum
      }
      if (c == t) zt = z[q];
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
    zt = wave_sum(zt);
    const float from = m > -INFINITY ? m : 0.0f;
    float o = 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q) o += q * kWave + l < C && q * kWave + l != t ? expf(z[q] - from) : 0.0f;
    o = wave_sum(o);
    float inv;
    const float of_row = finish_row(m, o, zt, inv), rest = o * inv;
    const float loss = mine ? of_row : 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int c = q * kWave + l;
      const float v = mine && c < C ? k * (c == t ? -rest : expf(z[q] - from) * inv) : 0.0f;
      if (c < Cp) d[w][c] = v;
      if (dz && r < R && c < ld_dz) dz[(size_t)r * ld_dz + c] = v;
    }
    if (l == 0) {
      on[w] = mine;
      losses[w] = mine ? (double)k * (double)loss : 0.0;
      if (r < R && row_loss) row_loss[r] = loss;
    }
  }
  __syncthreads();
  if (w == 0) {
    const uint64_t bits = __ballot(l < 16 && on[i]);
    if (l == 0) {
      reinterpret_cast<uint16_t*>(live)[blockIdx.x] = (uint16_t)bits;
      double s = 0.0;
      for (int q = 0; q < 16; ++q) s += losses[q];
      parts[blockIdx.x] = s;
    }
  }
  if (!dx) return;
  for (int h0 = 16 * w; h0 < H; h0 += 256) {  // lane (i, g): W's row h0 + i, dz of row i; then h0 + 4 g + v of row i
    const T* pw = W + (int64_t)min(h0 + i, H - 1) * ld_w;
    float wv[NT][4];
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      if (16 * a >= C) break;
      if (16 * a + 16 <= C) {
        load<T, 4>(pw + 16 * a + 4 * g, wv[a]);
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) wv[a][s] = to_float(pw[min(16 * a + 4 * g + s, C - 1)]);
      }
    }
    f32x4 o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      if (16 * a >= C) break;
#pragma unroll
      for (int s = 0; s < 4; ++s)
        o = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[a][s], d[i][16 * a + 4 * g + s], o, 0, 0, 0);
    }
    float v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = on[i] ? o[u] : 0.0f;
    if (r0 + i < R) store_in<T, 4>(dx + (int64_t)(r0 + i) * ld_dx, min(h0 + 4 * g, H), H, v);
  }
}

// dW of few rows and classes: a block 16 h and V tiles of classes, its 16 wavefronts every sixteenth run of 16 rows, straight
// from memory on the float32 matrix cores; their sums are added in LDS, in order. Of more rows a block takes a slice, to
// slices[slice][H][C]; else the first block also adds up the loss. dz's rows end in zeros at a multiple of 4.
template <class T, int V>
__global__ __launch_bounds__(1024) void ce_few_dw(const T* __restrict__ x, int64_t ld_x, const float* __restrict__ dz,
                                                  int ld_dz, const uint64_t* __restrict__ live, int R, int H, int C,
                                                  T* __restrict__ dW, int64_t ld_dw, float* __restrict__ slices,
                                                  const double* __restrict__ parts, int n_parts, float* __restrict__ loss) {
  __shared__ float sum[16][V * 16][17];  // of a wavefront: class, h
  const int w = threadIdx.x / kWave, l = lane_id(), i = l % 16, g = l / 16;
  const int h = blockIdx.x * 16 + i;
  const int base = blockIdx.y * V * 16;
  const int at = class_of<V>(blockIdx.y, i, ld_dz);
  f32x4 acc[V];
#pragma unroll
  for (int a = 0; a < V; ++a) acc[a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int per = ((R + 15) / 16 + gridDim.z - 1) / gridDim.z * 16, hi = min(R, ((int)blockIdx.z + 1) * per);
  for (int r0 = blockIdx.z * per + 16 * w; r0 < hi; r0 += 256) {
    float b[4], d[4][V];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = min(r0 + 4 * j + g, R - 1);  // slices end at multiples of 16, or with the rows
      const bool on = r0 + 4 * j + g < R && alive(live, r);
      b[j] = to_float(x[(int64_t)r * ld_x + min(h, H - 1)]);
      if (!on) b[j] = 0.0f;
      load<float, V>(dz + (size_t)r * ld_dz + at, d[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int a = 0; a < V; ++a) acc[a] = __builtin_amdgcn_mfma_f32_16x16x4f32(d[j][a], b[j], acc[a], 0, 0, 0);
  }
#pragma unroll
  for (int a = 0; a < V; ++a)
#pragma unroll
    for (int v = 0; v < 4; ++v) sum[w][class_of<V>(blockIdx.y, 4 * g + v, ld_dz) + a - base][i] = acc[a][v];
  __syncthreads();
  for (int q = threadIdx.x; q < 16 * V * 16; q += 1024) {
    const int c = q % (V * 16), n = q / (V * 16);
    if (base + c >= C || blockIdx.x * 16 + n >= H) continue;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += sum[k][c][n];
    const int at_h = blockIdx.x * 16 + n;
    if (slices) slices[((size_t)blockIdx.z * H + at_h) * C + base + c] = s;
    else dW[(int64_t)at_h * ld_dw + base + c] = from_float<T>(s);
  }
  if (!slices && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < kWave) {
    double s = 0.0;
    for (int k = l; k < n_parts; k += kWave) s += parts[k];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, kWave);
    if (l == 0) *loss = (float)s;
  }
}

// Whether a call takes a way of few classes: in 16 bits only that of few rows, which multiplies in float32.
bool few_of(int dtype, int R, int C) { return C <= kFew && (dtype == SNN_F32 || R <= kFewDwRows); }

// Whether it also has few rows.
bool few_rows(int R, int C) { return C <= kFew && R <= kFewDwRows; }

// Whether dW of more rows is formed like that of few, a block a slice of them, and not as a product in tiles of 128 x 128, most
// of which would lie past the classes. us a call, in tiles and so (rows x H x classes): 52460 x 681 x 9 187, 160; 13635 x
// 261 x 39 64, 52; 130000 x 16 x 30 185, 49; 128000 x 1024 x 10 480, 469; but x 32 475, 499; 14649 x 2027 x 34 191, 207.
constexpr int kSkinny = 64;
bool skinny_of(int H, int C) { return C <= kSkinny && (int64_t)C * H < 32768; }

struct Plan {
  int width, pieces;          // classes of a piece
  int z_slices, dw_slices, dx_slices;   // K slices of the products
  int ld;                     // of a piece's logits
};

Plan plan_of(int R, int H, int C) {
  Plan p;
  p.width = (int)std::min<int64_t>(C, std::max<int64_t>(256, kPiece / R / 128 * 128));
  p.pieces = (C + p.width - 1) / p.width;
  p.ld = (p.width + 3) / 4 * 4;
  p.z_slices = p.pieces == 1 && p.width <= kRowInRegs ? plan_splits(R, p.width, H, 88e12).splits : 1;
  p.dw_slices = few_rows(R, C)    ? 1
                : skinny_of(H, C) ? std::max(2, std::min(64, 4 * cu_count() / ((H + 15) / 16)))
                                  : plan_splits(H, p.width, R, 88e12).splits;
  p.dx_slices = plan_splits(R, H, p.width, 88e12).splits;
  return p;
}

constexpr int kLossParts = 256;

struct Workspace {
  uint64_t* live;
  int32_t* counts;
  uint4 *first, *second;
  float *z, *dX, *dW, *top, *sum, *at_target, *inv;
  double* parts;
  size_t bytes;
};

Workspace carve(void* ws, int R, int H, bool few, bool grad, const Plan& p) {
  Carve c(ws);
  Workspace g;
  g.live = c.take<uint64_t>(((size_t)R + 63) / 64);
  g.counts = c.take<int32_t>(kCountParts);
  const size_t stages = few && R > kFewDwRows ? (H + 31) / 32 : 0;
  g.first = c.take<uint4>(stages * 12 * kFew);
  g.second = c.take<uint4>(stages * 12 * kFew);
  const size_t rows = few || p.pieces == 1 ? 0 : (size_t)R;
  g.top = c.take<float>(rows);
  g.sum = c.take<float>(rows);
  g.at_target = c.take<float>(rows);
  g.inv = c.take<float>(rows);
  g.parts = c.take<double>(few ? (R + 15) / 16 : p.pieces == 1 ? R : kLossParts);
  g.z = c.take<float>(few && !grad ? 0 : (size_t)R * p.ld * (few ? 1 : p.z_slices));
  g.dX = c.take<float>(!few && grad && p.dx_slices > 1 ? (size_t)p.dx_slices * R * H : 0);
  g.dW = c.take<float>(grad && p.dw_slices > 1 ? (size_t)p.dw_slices * H * p.width : 0);
  g.bytes = c.off;
  return g;
}

// n columns of dW from their K slices. With loss also that, from n_parts parts.
void enqueue_dw_sum(int n, int H, float* dW, int64_t ld_dw, const Plan& p, const Workspace& g, hipStream_t s, int n_parts,
                    float* loss) {
  hipLaunchKernelGGL(ce_dw, dim3((unsigned)std::min<int64_t>(((int64_t)H * n + 255) / 256, 8 * cu_count())), dim3(256), 0, s,
                     g.dW, p.dw_slices, H, n, dW, ld_dw, g.parts, n_parts, loss);
}

// A piece's columns of dW (n of them) from its dz, in K slices where the product alone has few tiles. With loss also that,
// from n_parts parts.
void enqueue_dw(const float* x, int64_t ld_x, const float* dz, int ld_dz, int R, int H, int n, float* dW, int64_t ld_dw,
                const Plan& p, const Workspace& g, hipStream_t s, int n_parts = 0, float* loss = nullptr) {
  const uint32_t* live = reinterpret_cast<const uint32_t*>(g.live);  // the words' halves in order
  if (p.dw_slices == 1) {
    gemm_split_km(H, n, R, x, (int)ld_x, dz, ld_dz, dW, (int)ld_dw, 1, 0, s, live);
    if (loss) hipLaunchKernelGGL(ce_total, dim3(1), dim3(256), 0, s, g.parts, n_parts, loss);
    return;
  }
  gemm_split_km(H, n, R, x, (int)ld_x, dz, ld_dz, g.dW, n, p.dw_slices, (size_t)H * n, s, live);
  enqueue_dw_sum(n, H, dW, ld_dw, p, g, s, n_parts, loss);
}

template <class T, int NT>
void run_few(const T* x, int64_t ld_x, const T* W, int64_t ld_w, int R, int H, int C, const int32_t* targets,
             const float* weight, float* loss, float* row_loss, T* dx, int64_t ld_dx, T* dW, int64_t ld_dw, const Plan& p,
             const Workspace& g, hipStream_t s) {
  if (few_rows(R, C)) {
    const int blocks = (R + 15) / 16;
    constexpr int N = NT == 7 ? 8 : NT, V = kV<N>;
    hipLaunchKernelGGL((ce_small<T, N>), dim3((unsigned)blocks), dim3(1024), 0, s, x, ld_x, W, ld_w, R, H, C, targets, weight,
                       row_loss, g.parts, dx, ld_dx, dW ? g.z : nullptr, p.ld, g.live);
    if (dW)
      hipLaunchKernelGGL((ce_few_dw<T, V>), dim3((unsigned)((H + 15) / 16), N / V), dim3(1024), 0, s, x, ld_x, g.z, p.ld,
                         g.live, R, H, C, dW, ld_dw, nullptr, g.parts, blocks, loss);
    else
      hipLaunchKernelGGL(ce_total, dim3(1), dim3(256), 0, s, g.parts, blocks, loss);
    return;
  }
  if constexpr (sizeof(T) == 4) {
    // 32 rows a wavefront read W's parts half as often; 16 where 32 would leave compute units without a block
    const bool wide = (R + 127) / 128 >= 2 * cu_count(), vec = H % 8 == 0;
    const int blocks = wide ? (R + 127) / 128 : (R + 63) / 64;
    // without weights a launch of its own counts the rows that take part (6000 x 512 x 100: 80 us, with a count in every
    // block 100; 6000 x 200 x 10: 33, 38)
    const int counted = weight ? 0 : std::min(kCountParts, (R + 1023) / 1024);
    if (counted)
      hipLaunchKernelGGL(ce_live, dim3((unsigned)counted), dim3(256), 0, s, targets, weight, R, C, g.live, g.counts);
    hipLaunchKernelGGL((ce_few_parts<NT>), dim3((unsigned)((H + 31) / 32)), dim3(256), 0, s, W, ld_w, H, C, g.first,
                       g.second);
    const auto few = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, x, ld_x, g.first, g.second, R, H, C, targets,
                         weight, g.counts, counted, row_loss, g.parts, dx, ld_dx, dW ? g.z : nullptr,
                         p.ld, counted ? nullptr : g.live);
    };
    if (wide) few(vec ? ce_few<NT, 2, true> : ce_few<NT, 2, false>);
    else few(vec ? ce_few<NT, 1, true> : ce_few<NT, 1, false>);
    if constexpr (NT <= kSkinny / 16) {
      if (dW && skinny_of(H, C)) {
        hipLaunchKernelGGL((ce_few_dw<T, NT>), dim3((unsigned)((H + 15) / 16), 1, (unsigned)p.dw_slices), dim3(1024), 0, s, x,
                           ld_x, g.z, p.ld, g.live, R, H, C, dW, ld_dw, g.dW, g.parts, blocks, loss);
        enqueue_dw_sum(C, H, dW, ld_dw, p, g, s, blocks, loss);
        return;
      }
    }
    if (dW) enqueue_dw(x, ld_x, g.z, p.ld, R, H, C, dW, ld_dw, p, g, s, blocks, loss);
    else hipLaunchKernelGGL(ce_total, dim3(1), dim3(256), 0, s, g.parts, blocks, loss);
  }
}

template <class T>
void run_few(const T* x, int64_t ld_x, const T* W, int64_t ld_w, int R, int H, int C, const int32_t* targets,
             const float* weight, float* loss, float* row_loss, T* dx, int64_t ld_dx, T* dW, int64_t ld_dw, const Plan& p,
             const Workspace& g, hipStream_t s) {
#define SNN_FEW(NT)                                                                                                       \
  run_few<T, NT>(x, ld_x, W, ld_w, R, H, C, targets, weight, loss, row_loss, dx, ld_dx, dW, ld_dw, p, g, s)
  if (C <= 16) SNN_FEW(1);
  else if (C <= 32) SNN_FEW(2);
  else if (C <= 64) SNN_FEW(4);
  else if (C <= 112) SNN_FEW(7);
  else SNN_FEW(8);
#undef SNN_FEW
}

void run(const float* x, int64_t ld_x, const float* W, int64_t ld_w, int R, int H, int C, const int32_t* targets,
         const float* weight, float* loss, float* row_loss, float* dx, int64_t ld_dx, float* dW, int64_t ld_dw,
         const Plan& p, const Workspace& g, hipStream_t s) {
  const dim3 rows((unsigned)((R + kWaves - 1) / kWaves)), waves(kWaves * kWave);
  const int counted = std::min(kCountParts, (R + 1023) / 1024);
  const bool grad = dx || dW;
  hipLaunchKernelGGL(ce_live, dim3((unsigned)counted), dim3(256), 0, s, targets, weight, R, C, g.live, g.counts);
  int n_parts = 0;
  if (p.pieces == 1) {
    const size_t z_split = (size_t)R * p.ld;
    gemm_split_kr(R, C, H, x, (int)ld_x, W, (int)ld_w, g.z, p.ld, s, p.z_slices, z_split);
    const bool by_block = C >= kRowByBlock;
    n_parts = by_block ? std::min(R, 2 * cu_count()) : std::min((int)rows.x, 8 * cu_count());
    const auto of_rows = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)n_parts), dim3(by_block ? 1024 : 256), 0, s, g.z, p.z_slices, z_split, R, C,
                         p.ld, targets, g.live, g.counts, counted, weight, row_loss, g.parts);
    };
#define SNN_ROWS(L, Q) of_rows(grad ? ce_rows<true, L, Q> : ce_rows<false, L, Q>)
    if (C <= 256) SNN_ROWS(kWave, 1);
    else if (C <= 512) SNN_ROWS(kWave, 2);
    else if (!by_block) SNN_ROWS(kWave, 4);
    else if (C <= 4096) SNN_ROWS(1024, 1);
    else if (C <= 8192) SNN_ROWS(1024, 2);
    else if (C <= 16384) SNN_ROWS(1024, 4);
    else if (C <= kRowInRegs) SNN_ROWS(1024, 8);
    else SNN_ROWS(1024, 0);
#undef SNN_ROWS
  } else {
    for (int c0 = 0; c0 < C; c0 += p.width) {
      const int n = std::min(p.width, C - c0);
      gemm_split_kr(R, n, H, x, (int)ld_x, W + c0, (int)ld_w, g.z, p.ld, s);
      hipLaunchKernelGGL(ce_sums, rows, waves, 0, s, g.z, R, n, p.ld, c0, targets, g.live, g.top, g.sum, g.at_target);
    }
    n_parts = std::min(kLossParts, (R + 255) / 256);
    hipLaunchKernelGGL(ce_losses, dim3((unsigned)n_parts), dim3(256), 0, s, R, g.live, g.counts, counted, weight, g.top,
                       g.sum, g.at_target, g.inv, row_loss, g.parts);
  }
  float* to = p.dx_slices > 1 ? g.dX : dx;
  const int ld_to = p.dx_slices > 1 ? H : (int)ld_dx;
  for (int c0 = 0; grad && c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0);
    if (p.pieces > 1) {
      gemm_split_kr(R, n, H, x, (int)ld_x, W + c0, (int)ld_w, g.z, p.ld, s);
      hipLaunchKernelGGL(ce_dz, rows, waves, 0, s, g.z, R, n, p.ld, c0, targets, g.live, g.counts, counted, weight, g.top,
                         g.sum, g.inv);
    }
    if (dx) gemm_split_kc(R, H, n, g.z, p.ld, W + c0, (int)ld_w, to, ld_to, s, c0 > 0, p.dx_slices, (size_t)R * H);
    if (dW) enqueue_dw(x, ld_x, g.z, p.ld, R, H, n, dW + c0, ld_dw, p, g, s);
  }
  if (dx && p.dx_slices > 1)
    hipLaunchKernelGGL(ce_dx, dim3((unsigned)R, (unsigned)((H + kWave - 1) / kWave)), waves, 0, s, g.dX, p.dx_slices, g.live,
                       R, H, dx, ld_dx);
  const bool clear = dx && p.dx_slices == 1;
  hipLaunchKernelGGL(ce_finish, dim3(1 + (clear ? (R + kWaves * kClearRows - 1) / (kWaves * kClearRows) : 0)), waves, 0, s, g.parts,
                     n_parts, loss, g.live, R, H, dx, ld_dx);
}

// ------------------------------------------------------------------ 16-bit operands

// x and dz of 16-bit calls are multiplied in that type. dz enters as ref times (w / ref)(softmax - onehot), ref the
// largest weight, so that one weight for all rows costs no rounding; float16's numbers are also raised by 2^15, since
// those below 2^-14 have few bits. Both come off the float32 sums. Bound: the matrix cores, with four products of R H C
// where the gradients alone have three. 8192 x 1024 x 32003 bfloat16: sums of exponentials 482 us (1.06 PFLOP/s with 5% of
// the rows left out), dz 585, dx 429, dW 424 (1.2). The rounding of dz makes dx's error against 64 bits 1.00 (there) to 1.25
// times that of rounding the result alone.
template <class T>
constexpr float kRaise = std::is_same<T, F16>::value ? 32768.0f : 1.0f;

// Classes of a partial sum of exponentials: a wavefront's.
template <int TILE>
constexpr int kPart = gemm16::Shape<TILE>::kWaveM;

// pos[r]: rows before r that take part, pos[R]: their number; ref: the largest weight. Blocks of 1024 threads: one takes up
// to kOneBlock rows, a run of them a thread; beyond, the flags' prefix is formed by the scan and ref by a launch of its own
// (rows x 128 x 300 bfloat16, us a call by one block and by the scan: 4096 58, 65; 8192 69, 71; 16384 92, 87; 32768 129, 106).
constexpr int kOneBlock = 8192;
static_assert(kOneBlock <= 32 * 1024, "a thread's rows have a bit each");
__global__ __launch_bounds__(1024) void ce_places(const int32_t* __restrict__ targets, const float* __restrict__ weight,
                                                  int R, int C, int32_t* __restrict__ pos, float* __restrict__ ref) {
  __shared__ int count[1024 / kWave];
  __shared__ float top[1024 / kWave];
  const int per = (R + 1023) / 1024, lo = min(R, (int)threadIdx.x * per), hi = min(R, lo + per);
  const int w = threadIdx.x / kWave;
  int n = 0;
  uint32_t on = 0;  // of the thread's at most 32 rows
  float m = 0.0f;
  for (int r = lo; r < hi; ++r)
    if (takes_part(targets, weight, r, C)) {
      on |= 1u << (r - lo);
      ++n;
      if (weight) m = fmaxf(m, fabsf(weight[r]));
    }
  const int upto = wave_incl_scan(n);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
  if (lane_id() == kWave - 1) {
    count[w] = upto;
    top[w] = m;
  }
  __syncthreads();
  int p = upto - n, all = 0;
  for (int k = 0; k < 1024 / kWave; ++k) {
    if (k < w) p += count[k];
    all += count[k];
    m = fmaxf(m, top[k]);
  }
  for (int r = lo; r < hi; ++r) {
    pos[r] = p;
    p += on >> (r - lo) & 1;
  }
  if (threadIdx.x == 0) {
    pos[R] = all;
    *ref = weight ? m : (all > 0 ? 1.0f / (float)all : 0.0f);
  }
}

__global__ __launch_bounds__(256) void ce_flags(const int32_t* __restrict__ targets, const float* __restrict__ weight, int R,
                                                int C, int32_t* __restrict__ flags) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < R) flags[r] = takes_part(targets, weight, r, C);
}

__global__ __launch_bounds__(1024) void ce_ref(const float* __restrict__ weight, const int32_t* __restrict__ pos, int R,
                                               float* __restrict__ ref) {
  __shared__ float top[1024 / kWave];
  float m = 0.0f;
  if (weight) {
    for (int r = threadIdx.x; r < R; r += 1024)
      if (pos[r + 1] > pos[r]) m = fmaxf(m, fabsf(weight[r]));
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
    if (lane_id() == 0) top[threadIdx.x / kWave] = m;
    __syncthreads();
    for (int k = 0; k < 1024 / kWave; ++k) m = fmaxf(m, top[k]);
  } else if (pos[R] > 0) {
    m = 1.0f / (float)pos[R];
  }
  if (threadIdx.x == 0) *ref = m;
}

// Rows to their packed places, row_of[place] = row: lines of Hp, zeros behind H and in the lines behind the rows that take
// part up to a whole tile. The others' loss is 0, and their dx where the product writes dx itself (dx NULL: it does not).
template <class T>
__global__ __launch_bounds__(kWaves * kWave) void ce_pack16(const T* __restrict__ x, int64_t ld, int R, int Rp, int H,
                                                            int Hp, const int32_t* __restrict__ targets,
                                                            const float* __restrict__ weight,
                                                            const int32_t* __restrict__ pos, T* __restrict__ X,
                                                            int32_t* __restrict__ target, float* __restrict__ w,
                                                            int32_t* __restrict__ row_of, float* __restrict__ row_loss,
                                                            int tile, T* __restrict__ dx, int64_t ld_dx) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= Rp) return;
  const int n = pos[R], p0 = r < R ? pos[r] : n;
  const bool live = r < R && pos[r + 1] > p0;
  const int p = live ? p0 : n + (r - p0);
  if (!live && r < R) {
    if (row_loss && lane_id() == 0) row_loss[r] = 0.0f;
    if (dx)
      for (int i = lane_id(); i < H; i += kWave) dx[(int64_t)r * ld_dx + i] = T{0};
  }
  if (p >= (n + tile - 1) / tile * tile) return;
  for (int i = lane_id() * 8; i < Hp; i += kWave * 8) {
    T v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = T{0};
    if (live) {
      const T* s = x + (int64_t)r * ld + i;
      if (i + 8 <= H) {
        __builtin_memcpy(v, s, 16);
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (i + u < H) v[u] = s[u];
      }
    }
    *reinterpret_cast<uint4*>(X + (size_t)p * Hp + i) = __builtin_bit_cast(uint4, v);
  }
  if (lane_id() == 0) {
    target[p] = live ? targets[r] : -1;
    w[p] = !live ? 0.0f : weight ? weight[r] : 1.0f / (float)n;
    row_of[p] = r;
  }
}

// n columns of W in lines of `width`, zeros behind them and in the lines from H on.
template <class T>
__global__ __launch_bounds__(256) void ce_weights16(const T* __restrict__ W, int64_t ld, int H, int n, int width,
                                                    T* __restrict__ out) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8, h = blockIdx.y;
  if (c >= width) return;
  T v[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) v[u] = T{0};
  if (h < H) {
    const T* s = W + (int64_t)h * ld + c;
    if (c + 8 <= n) {
      __builtin_memcpy(v, s, 16);
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c + u < n) v[u] = s[u];
    }
  }
  *reinterpret_cast<uint4*>(out + (size_t)h * width + c) = __builtin_bit_cast(uint4, v);
}

// Logits of a tile of classes (m) and rows (n). GRAD false: every row's largest logit and sum of exponentials over the
// classes of a wavefront but the target, to part[class / kPart][row], and the target's logit. GRAD true: dz to
// G[row][class], from every row's largest logit, 1 / s and o / s.
template <class T, bool GRAD, int TILE>
__global__ __launch_bounds__(gemm16::Shape<TILE>::kThreads, 2) void ce_logits16(
    const T* __restrict__ W, int64_t ldw, const T* __restrict__ X, int Hp, int stages, int c0, int C, int R, int Rp,
    int tiles_m, int tiles_n, const int32_t* __restrict__ pos, const int32_t* __restrict__ target,
    float2* __restrict__ part, float* __restrict__ at_target, const float* __restrict__ tops,
    const float* __restrict__ inv, const float* __restrict__ rest, const float* __restrict__ w,
    const float* __restrict__ ref, T* __restrict__ G, int64_t ldg) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const gemm16::Tiles t = gemm16::tile_of(tiles_m, tiles_n, 1);
  if (!t.ok || t.n * TILE >= pos[R]) return;
  using S = gemm16::Shape<TILE>;
  gemm16::Product<T, true, false, TILE> z;
  const int l = lane_id(), g = l / 16;
  const int m0 = t.m * TILE + z.m_of_wave();
  const int first = c0 + m0;  // class of the wavefront's first m
  const int n0 = t.n * TILE + z.n_of_wave() + l % 16;
  // what the rows need at the end is asked for now
  int32_t tgt[S::kB];
  float top[S::kB], k[S::kB], kt[S::kB];  // factors of the exponentials, the target's dz
#pragma unroll
  for (int b = 0; b < S::kB; ++b) {
    tgt[b] = target[n0 + 16 * b];
    if (GRAD) {
      top[b] = k[b] = kt[b] = 0.0f;
      if (tgt[b] >= 0) {
        const float all = w[n0 + 16 * b] / *ref * kRaise<T>;
        top[b] = tops[n0 + 16 * b];
        k[b] = all * inv[n0 + 16 * b];
        kt[b] = -all * rest[n0 + 16 * b];
      }
    }
  }
  z.run(W, ldw, t.m * TILE, X, Hp, t.n * TILE, 0, stages, smem);
  constexpr float kLog2e = 1.44269504088896340736f;
  const bool ragged = first + kPart<TILE> > C;
#pragma unroll
  for (int b = 0; b < S::kB; ++b) {
    const int n = n0 + 16 * b;
    const int at = tgt[b] - first;  // the target among this wavefront's classes
    const bool here = tgt[b] >= 0 && (unsigned)at < (unsigned)kPart<TILE>;
    if (ragged) {
#pragma unroll
      for (int a = 0; a < S::kA; ++a)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (first + 16 * a + 4 * g + v >= C) z.acc[a][b][v] = -INFINITY;
    }
    if constexpr (!GRAD) {
      if (here && (at / 4) % 4 == g) {
#pragma unroll
        for (int a = 0; a < S::kA; ++a)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (at == 16 * a + 4 * g + v) {
              at_target[n] = z.acc[a][b][v];
              z.acc[a][b][v] = -INFINITY;
            }
      }
      float m = -INFINITY;
#pragma unroll
      for (int a = 0; a < S::kA; ++a)
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, z.acc[a][b][v]);
      m = fmaxf(m, __shfl_xor(m, 16, kWave));
      m = fmaxf(m, __shfl_xor(m, 32, kWave));
      const float from = m > -INFINITY ? m : 0.0f;
      float s = 0.0f;
#pragma unroll
      for (int a = 0; a < S::kA; ++a)
#pragma unroll
        for (int v = 0; v < 4; ++v) s += __builtin_amdgcn_exp2f((z.acc[a][b][v] - from) * kLog2e);
      s += __shfl_xor(s, 16, kWave);
      s += __shfl_xor(s, 32, kWave);
      if (g == 0) part[(size_t)(first / kPart<TILE>) * Rp + n] = make_float2(m, s);
    } else {
      const bool live = tgt[b] >= 0;
#pragma unroll
      for (int a = 0; a < S::kA; ++a) {
        T d[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float p = __builtin_amdgcn_exp2f((z.acc[a][b][v] - top[b]) * kLog2e) * k[b];
          d[v] = from_float<T>(!live ? 0.0f : here && at == 16 * a + 4 * g + v ? kt[b] : p);
        }
        *reinterpret_cast<uint2*>(G + (size_t)n * ldg + m0 + 16 * a + 4 * g) = __builtin_bit_cast(uint2, d);
      }
    }
  }
}

// Every row's largest logit, 1 / s, o / s and loss from the parts of its classes; the weighted losses of a block in
// float64. A block takes 32 rows, 32 threads share a row's parts.
__global__ __launch_bounds__(1024) void ce_join16(const float2* __restrict__ part, int parts, int R, int Rp,
                                                  const int32_t* __restrict__ pos, const int32_t* __restrict__ row_of,
                                                  const float* __restrict__ at_target, const float* __restrict__ w,
                                                  float* __restrict__ top, float* __restrict__ inv,
                                                  float* __restrict__ rest, float* __restrict__ row_loss,
                                                  double* __restrict__ losses) {
  __shared__ float2 all[32][33];
  const int x = threadIdx.x % 32, y = threadIdx.x / 32;
  const int r = blockIdx.x * 32 + x;
  if ((int)blockIdx.x * 32 >= pos[R]) {
    if (threadIdx.x == 0) losses[blockIdx.x] = 0.0;
    return;
  }
  float m = -INFINITY, s = 0.0f;
  const auto add = [&](float m1, float s1) {
    const float both = fmaxf(m, m1), from = both > -INFINITY ? both : 0.0f;
    s = s * expf(m - from) + s1 * expf(m1 - from);
    m = both;
  };
#pragma unroll 4
  for (int p = y; p < parts; p += 32) {
    const float2 q = part[(size_t)p * Rp + r];
    add(q.x, q.y);
  }
  all[y][x] = make_float2(m, s);
  __syncthreads();
  if (y == 0) {
    for (int k = 1; k < 32; ++k) add(all[k][x].x, all[k][x].y);
    double weighted = 0.0;
    if (r < pos[R]) {
      const float zt = at_target[r];
      float over;
      const float others = m;
      m = fmaxf(m, zt);
      const float from = m > -INFINITY ? m : 0.0f;
      s *= expf(others - from);
      const float loss = finish_row(m, s, zt, over);
      top[r] = from;
      inv[r] = over;
      rest[r] = s * over;
      if (row_loss) row_loss[row_of[r]] = loss;
      weighted = (double)w[r] * (double)loss;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) weighted += __shfl_xor(weighted, off, kWave);
    if (x == 0) losses[blockIdx.x] = weighted;
  }
}

// A K slice's dx of a piece: dX[slice][row][h] (+)= sum over its classes of G W; with dx the whole of it, to the rows' places.
template <class T, int TILE>
__global__ __launch_bounds__(gemm16::Shape<TILE>::kThreads, 2) void ce_dx16(
    const T* __restrict__ W, int64_t ldw, const T* __restrict__ G, int64_t ldg, int stages, int per, int R, int Rp, int H,
    int Hp, int tiles_m, int tiles_n, int slices, const int32_t* __restrict__ pos, int accumulate, float* __restrict__ dX,
    const int32_t* __restrict__ row_of, const float* __restrict__ ref, T* __restrict__ dx, int64_t ld) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const gemm16::Tiles t = gemm16::tile_of(tiles_m, tiles_n, slices);
  if (!t.ok || t.n * TILE >= pos[R]) return;
  using S = gemm16::Shape<TILE>;
  gemm16::Product<T, false, false, TILE> d;
  const int from = t.slice * per;
  d.run(W, ldw, t.m * TILE, G, ldg, t.n * TILE, (int64_t)from * gemm16::kK, max(0, min(per, stages - from)), smem);
  const int l = lane_id();
  const int n0 = t.n * TILE + d.n_of_wave() + l % 16, m0 = t.m * TILE + d.m_of_wave() + l / 16 * 4;
  if (dx) {
    const float k = *ref / kRaise<T>;
#pragma unroll
    for (int b = 0; b < S::kB; ++b) {
      const int n = n0 + 16 * b;
      if (n >= pos[R]) continue;
      T* row = dx + (int64_t)row_of[n] * ld;
#pragma unroll
      for (int a = 0; a < S::kA; ++a) {
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = d.acc[a][b][u] * k;
        store_in<T, 4>(row, min(m0 + 16 * a, H), H, v);
      }
    }
    return;
  }
  float* out = dX + ((size_t)t.slice * Rp + n0) * Hp + m0;
#pragma unroll
  for (int b = 0; b < S::kB; ++b)
#pragma unroll
    for (int a = 0; a < S::kA; ++a) {
      gemm16::f32x4* o = reinterpret_cast<gemm16::f32x4*>(out + (size_t)16 * b * Hp + 16 * a);
      *o = accumulate ? *o + d.acc[a][b] : d.acc[a][b];
    }
}

// dx from its K slices: a block takes 256 h of a row, its wavefronts a quarter of the slices each. The first
// row's first block also adds up the loss.
template <class T>
__global__ __launch_bounds__(kWaves * kWave) void ce_dx_out16(const float* __restrict__ dX, int slices, int R, int Rp, int H,
                                                              int Hp, const int32_t* __restrict__ pos,
                                                              const float* __restrict__ ref, T* __restrict__ dx,
                                                              int64_t ld, const double* __restrict__ parts, int n_parts,
                                                              float* __restrict__ loss, int r0) {
  __shared__ float4 all[kWaves][kWave];
  if (r0 + (int)blockIdx.x == 0 && blockIdx.y == 0) total_of(parts, n_parts, loss);
  const int w = threadIdx.x / kWave, l = lane_id();
  const int r = r0 + blockIdx.x, i = (blockIdx.y * kWave + l) * 4;
  const int p = pos[r];
  const bool live = pos[r + 1] > p;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (live && i < Hp) {
    const int share = (slices + kWaves - 1) / kWaves;
#pragma unroll 4
    for (int q = w * share; q < min(slices, (w + 1) * share); ++q) {
      const float4 v = *reinterpret_cast<const float4*>(dX + ((size_t)q * Rp + p) * Hp + i);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  all[w][l] = s;
  __syncthreads();
  if (w > 0 || i >= H) return;
  float o[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int q = 1; q < kWaves; ++q) {
    o[0] += all[q][l].x; o[1] += all[q][l].y; o[2] += all[q][l].z; o[3] += all[q][l].w;
  }
  const float k = *ref / kRaise<T>;
#pragma unroll
  for (int u = 0; u < 4; ++u) o[u] *= k;
  store_in<T, 4>(dx + (int64_t)r * ld, i, H, o);
}

// dW of a piece's n columns: the tile itself with one slice, else its share to part[slice][h][width].
template <class T, int TILE>
__global__ __launch_bounds__(gemm16::Shape<TILE>::kThreads, 2) void ce_dw16(const T* __restrict__ G, int64_t ldg, const T* __restrict__ X,
                                                               int Hp, int R, int H, int n, int width, int tiles_m,
                                                               int tiles_n, int slices, const int32_t* __restrict__ pos,
                                                               const float* __restrict__ ref, T* __restrict__ dW,
                                                               int64_t ld, float* __restrict__ part) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const gemm16::Tiles t = gemm16::tile_of(tiles_m, tiles_n, slices);
  if (!t.ok) return;
  const int stages = (pos[R] + gemm16::kK - 1) / gemm16::kK;
  const int per = (stages + slices - 1) / slices, from = t.slice * per;
  using S = gemm16::Shape<TILE>;
  gemm16::Product<T, true, true, TILE> d;
  d.run(G, ldg, t.m * TILE, X, Hp, t.n * TILE, (int64_t)from * gemm16::kK, max(0, min(per, stages - from)), smem);
  const int l = lane_id();
  const int m0 = t.m * TILE + d.m_of_wave() + l / 16 * 4, n0 = t.n * TILE + d.n_of_wave() + l % 16;
  const float k = *ref / kRaise<T>;
#pragma unroll
  for (int b = 0; b < S::kB; ++b) {
    const int h = n0 + 16 * b;
    if (h >= H) continue;
#pragma unroll
    for (int a = 0; a < S::kA; ++a) {
      const int c = m0 + 16 * a;
      if (slices > 1) {
        *reinterpret_cast<gemm16::f32x4*>(part + ((size_t)t.slice * H + h) * width + c) = d.acc[a][b];
      } else if (c < n) {
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = d.acc[a][b][u] * k;
        store_in<T, 4>(dW + (int64_t)h * ld, c, n, v);
      }
    }
  }
}

template <class T>
__global__ void ce_dw_out16(const float* __restrict__ part, int slices, int H, int n, int width,
                            const float* __restrict__ ref, T* __restrict__ dW, int64_t ld) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= n) return;
  const float k = *ref / kRaise<T>;
  for (int h = blockIdx.y; h < H; h += gridDim.y) {
    float s = 0.0f;
    for (int q = 0; q < slices; ++q) s += part[((size_t)q * H + h) * width + c];
    dW[(int64_t)h * ld + c] = from_float<T>(s * k);
  }
}

constexpr int64_t kPiece16 = (int64_t)1 << 28;  // dz values of a piece

// K slices of a product of `tiles` tiles and `stages` stages: blocks go in rounds over the compute units (two at a time of
// the small tile, at half the speed each), a stage takes a microsecond, a slice's share of a tile (written and read) a
// quarter of one.
int slices_of(int64_t tiles, int stages, int tile) {
  const int64_t at_once = cu_count() * (tile == 128 ? 2 : 1);
  int best = 1;
  double least = 0.0;
  for (int s = 1; s <= 64 && (s == 1 || s * 4 <= stages); ++s) {
    const double rounds = (double)((tiles * s + at_once - 1) / at_once);
    const double t = rounds * ((stages + s - 1) / s + 3) + (s > 1 ? 0.25 * rounds + 0.1 * s * tiles / at_once : 0.0);
    if (s == 1 || t < least) {
      best = s;
      least = t;
    }
  }
  return best;
}

int padded(int n, int to) { return (n + to - 1) / to * to; }

struct Plan16 {
  int tile, Rp, Hp, width, pieces, dx_slices, dw_slices;
  bool direct;   // dx from the product itself
  size_t parts;  // partial sums of exponentials a row
};

// The large tile where its blocks fill the card twice over and a product has stages enough to cover its end. Small against
// large tile, bfloat16, us a call (rows x H x classes): 360 x 128 x 512 47, 72; 3000 x 1000 x 8000 (384 large tiles) 285, 295;
// 2048 x 1024 x 16384 (512) 334, 303; 8192 x 1024 x 32003 2408, 2059; 4926 x 128 x 71434 1024, 1063; x 200 1417, 1254.
int tile_of(int R, int H, int C) {
  return H > 128 && (int64_t)((R + 255) / 256) * ((C + 255) / 256) >= 2 * cu_count() ? 256 : 128;
}

Plan16 plan16_of(int R, int H, int C) {
  Plan16 p;
  p.tile = tile_of(R, H, C);
  p.Rp = padded(R, p.tile);
  p.Hp = padded(H, p.tile);
  const int most = (int)std::min<int64_t>(padded(C, p.tile), std::max<int64_t>(p.tile, kPiece16 / p.Rp / p.tile * p.tile));
  p.pieces = (C + most - 1) / most;
  p.width = padded((C + p.pieces - 1) / p.pieces, p.tile);
  p.pieces = (C + p.width - 1) / p.width;
  p.dx_slices = slices_of((int64_t)(p.Hp / p.tile) * (p.Rp / p.tile), p.width / gemm16::kK, p.tile);
  p.dw_slices = slices_of((int64_t)(p.width / p.tile) * (p.Hp / p.tile), p.Rp / gemm16::kK, p.tile);
  p.direct = p.pieces == 1 && p.dx_slices == 1;
  p.parts = (size_t)p.pieces * p.width / (p.tile / 2);
  return p;
}

struct Workspace16 {
  int32_t *flags, *pos, *temp, *target, *row_of;
  int64_t* total;
  uint16_t *X, *W, *G;
  float *w, *at_target, *top, *inv, *rest, *ref, *dX, *dW;
  float2* part;
  double* parts;
  size_t bytes;
};

// W is always given room, so that the size does not depend on its address.
Workspace16 carve16(void* ws, int R, int H, int C, bool grad, const Plan16& p) {
  Carve c(ws);
  Workspace16 g;
  const size_t flags = R > kOneBlock ? (size_t)R : 0;
  g.flags = c.take<int32_t>(flags);
  g.pos = c.take<int32_t>((size_t)R + 1);
  g.temp = c.take<int32_t>(scan_temp_elems(R));
  g.total = c.take<int64_t>(1);
  g.target = c.take<int32_t>(p.Rp);
  g.row_of = c.take<int32_t>(p.Rp);
  g.w = c.take<float>(p.Rp);
  g.at_target = c.take<float>(p.Rp);
  g.top = c.take<float>(p.Rp);
  g.inv = c.take<float>(p.Rp);
  g.rest = c.take<float>(p.Rp);
  g.ref = c.take<float>(1);
  g.parts = c.take<double>(p.Rp / 32);
  g.part = c.take<float2>(p.parts * p.Rp);
  g.X = c.take<uint16_t>((size_t)p.Rp * p.Hp);
  g.W = c.take<uint16_t>((size_t)p.Hp * p.width);
  g.G = c.take<uint16_t>(grad ? (size_t)p.Rp * p.width : 0);
  g.dX = c.take<float>(grad && !p.direct ? (size_t)p.dx_slices * p.Rp * p.Hp : 0);
  g.dW = c.take<float>(grad && p.dw_slices > 1 ? (size_t)p.dw_slices * H * p.width : 0);
  g.bytes = c.off;
  return g;
}

template <class T, int TILE>
void run16(const T* x, int64_t ld_x, const T* W, int64_t ld_w, int R, int H, int C, const int32_t* targets,
           const float* weight, float* loss, float* row_loss, T* dx, int64_t ld_dx, T* dW, int64_t ld_dw,
           const Plan16& p, const Workspace16& g, hipStream_t s) {
  T *X = reinterpret_cast<T*>(g.X), *Wp = reinterpret_cast<T*>(g.W), *G = reinterpret_cast<T*>(g.G);
  using S = gemm16::Shape<TILE>;
  const dim3 waves(kWaves * kWave), block(S::kThreads);
  const auto rows_of = [](int n) { return dim3((unsigned)((n + kWaves - 1) / kWaves)); };
  for (const void* f : {(const void*)ce_logits16<T, false, TILE>, (const void*)ce_logits16<T, true, TILE>,
                        (const void*)ce_dx16<T, TILE>, (const void*)ce_dw16<T, TILE>})
    ensure_dynamic_lds(f, S::kLds);
  if (R <= kOneBlock) {
    hipLaunchKernelGGL(ce_places, dim3(1), dim3(1024), 0, s, targets, weight, R, C, g.pos, g.ref);
  } else {
    hipLaunchKernelGGL(ce_flags, dim3((unsigned)((R + 255) / 256)), dim3(256), 0, s, targets, weight, R, C, g.flags);
    launch_exclusive_scan(g.flags, R, g.pos, g.total, g.temp, s);
    hipLaunchKernelGGL(ce_ref, dim3(1), dim3(1024), 0, s, weight, g.pos, R, g.ref);
  }
  hipLaunchKernelGGL(ce_pack16<T>, rows_of(p.Rp), waves, 0, s, x, ld_x, R, p.Rp, H, p.Hp, targets, weight, g.pos, X,
                     g.target, g.w, g.row_of, row_loss, TILE, p.direct ? dx : nullptr, ld_dx);
  // W in place where its rows are whole tiles at 16-byte addresses
  const bool whole = H % TILE == 0 && C % TILE == 0 && ld_w % 8 == 0 && ld_w < (1 << 22) &&
                     reinterpret_cast<uintptr_t>(W) % 16 == 0;
  const T* w = nullptr;
  int64_t ldw = 0;
  const auto weights = [&](int c0, int n) {
    if (whole) {
      w = W + c0;
      ldw = ld_w;
    } else {
      hipLaunchKernelGGL(ce_weights16<T>, dim3((unsigned)((p.width / 8 + 255) / 256), (unsigned)p.Hp), dim3(256), 0, s,
                         W + c0, ld_w, H, n, p.width, Wp);
      w = Wp;
      ldw = p.width;
    }
  };
  const int tiles_n = p.Rp / TILE, tiles_h = p.Hp / TILE, stages_h = padded(H, gemm16::kK) / gemm16::kK;
  for (int c0 = 0; c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0), tiles_m = (n + TILE - 1) / TILE;
    weights(c0, n);
    hipLaunchKernelGGL((ce_logits16<T, false, TILE>), dim3(gemm16::grid_of(tiles_m, tiles_n, 1)), block, S::kLds, s, w, ldw,
                       X, p.Hp, stages_h, c0, C, R, p.Rp, tiles_m, tiles_n, g.pos, g.target, g.part, g.at_target, nullptr,
                       nullptr, nullptr, nullptr, nullptr, (T*)nullptr, 0);
  }
  hipLaunchKernelGGL(ce_join16, dim3((unsigned)(p.Rp / 32)), dim3(1024), 0, s, g.part, padded(C, TILE) / kPart<TILE>, R, p.Rp,
                     g.pos, g.row_of, g.at_target, g.w, g.top, g.inv, g.rest, row_loss,
                     g.parts);
  if (!dx || p.direct) hipLaunchKernelGGL(ce_total, dim3(1), dim3(256), 0, s, g.parts, p.Rp / 32, loss);
  if (!dx && !dW) return;
  for (int c0 = 0; c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0), tiles_m = (n + TILE - 1) / TILE;
    if (p.pieces > 1) weights(c0, n);
    hipLaunchKernelGGL((ce_logits16<T, true, TILE>), dim3(gemm16::grid_of(tiles_m, tiles_n, 1)), block, S::kLds, s, w, ldw,
                       X, p.Hp, stages_h, c0, C, R, p.Rp, tiles_m, tiles_n, g.pos, g.target, nullptr, nullptr, g.top, g.inv,
                       g.rest, g.w, g.ref, G, (int64_t)p.width);
    if (dx) {
      const int stages = tiles_m * (TILE / gemm16::kK), per = (stages + p.dx_slices - 1) / p.dx_slices;
      hipLaunchKernelGGL((ce_dx16<T, TILE>), dim3(gemm16::grid_of(tiles_h, tiles_n, p.dx_slices)), block, S::kLds, s, w, ldw,
                         G, (int64_t)p.width, stages, per, R, p.Rp, H, p.Hp, tiles_h, tiles_n, p.dx_slices, g.pos, c0 > 0,
                         g.dX, g.row_of, g.ref, p.direct ? dx : nullptr, ld_dx);
    }
    if (dW) {
      hipLaunchKernelGGL((ce_dw16<T, TILE>), dim3(gemm16::grid_of(tiles_m, tiles_h, p.dw_slices)), block, S::kLds, s, G,
                         (int64_t)p.width, X, p.Hp, R, H, n, p.width, tiles_m, tiles_h, p.dw_slices, g.pos, g.ref, dW + c0,
                         ld_dw, g.dW);
      if (p.dw_slices > 1)
        hipLaunchKernelGGL(ce_dw_out16<T>, dim3((unsigned)((n + 255) / 256), (unsigned)std::min(H, 1024)), dim3(256), 0, s,
                           g.dW, p.dw_slices, H, n, p.width, g.ref, dW + c0, ld_dw);
    }
  }
  const int step = 1 << 22;  // rows of a launch: a dispatch counts threads in 32 bits
  for (int r0 = 0; dx && !p.direct && r0 < R; r0 += step)
    hipLaunchKernelGGL(ce_dx_out16<T>, dim3((unsigned)std::min(step, R - r0), (unsigned)((H + 255) / 256)), waves, 0, s, g.dX,
                       p.dx_slices, R, p.Rp, H, p.Hp, g.pos, g.ref, dx, ld_dx, g.parts, p.Rp / 32, loss, r0);
}

template <class T>
void run16(const T* x, int64_t ld_x, const T* W, int64_t ld_w, int R, int H, int C, const int32_t* targets,
           const float* weight, float* loss, float* row_loss, T* dx, int64_t ld_dx, T* dW, int64_t ld_dw,
           const Plan16& p, const Workspace16& g, hipStream_t s) {
  if (p.tile == 256)
    run16<T, 256>(x, ld_x, W, ld_w, R, H, C, targets, weight, loss, row_loss, dx, ld_dx, dW, ld_dw, p, g, s);
  else
    run16<T, 128>(x, ld_x, W, ld_w, R, H, C, targets, weight, loss, row_loss, dx, ld_dx, dW, ld_dw, p, g, s);
}

snn_status check_sizes(int dtype, int64_t R, int H, int C) {
  if (!dtype_size(dtype) || R <= 0 || H <= 0 || C <= 0) return SNN_ERR_INVALID_ARG;
  if (R > kMaxRows || H > kMaxHidden || C > rows::kMaxClasses) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" size_t snn_linear_ce_workspace(int dtype, int64_t R, int H, int C, int grad) {
  if (check_sizes(dtype, R, H, C) != SNN_OK) return 0;
  const bool few = few_of(dtype, (int)R, C);
  if (few || dtype == SNN_F32) return carve(nullptr, (int)R, H, few, grad != 0, plan_of((int)R, H, C)).bytes;
  return carve16(nullptr, (int)R, H, C, grad != 0, plan16_of((int)R, H, C)).bytes;
}

extern "C" snn_status snn_linear_ce(const void* x, const void* W, int dtype, int64_t R, int H, int C, int64_t ld_x,
                                    int64_t ld_w, const int32_t* targets, const float* weight, float* loss,
                                    float* row_loss, void* dx, int64_t ld_dx, void* dW, int64_t ld_dw, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  if (!x || !W || !targets || !loss || !workspace) return SNN_ERR_INVALID_ARG;
  if (const snn_status st = check_sizes(dtype, R, H, C)) return st;
  if (ld_x < H || ld_w < C || (dx && ld_dx < H) || (dW && ld_dw < C)) return SNN_ERR_INVALID_ARG;
  if (misaligned(x, dtype) || misaligned(W, dtype) || misaligned(dx, dtype) || misaligned(dW, dtype))
    return SNN_ERR_INVALID_ARG;
  if (ld_w > INT32_MAX || ld_x > INT32_MAX || (dx && ld_dx > INT32_MAX) || (dW && ld_dw > INT32_MAX)) return SNN_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool few = few_of(dtype, (int)R, C);
  if (few || dtype == SNN_F32) {
    const Plan p = plan_of((int)R, H, C);
    const Workspace g = carve(workspace, (int)R, H, few, dx || dW, p);
    if (workspace_bytes < g.bytes) return SNN_ERR_INVALID_ARG;
#define SNN_CE(RUN, T)                                                                                                \
  RUN(static_cast<const T*>(x), ld_x, static_cast<const T*>(W), ld_w, (int)R, H, C, targets, weight, loss, row_loss,  \
      static_cast<T*>(dx), ld_dx, static_cast<T*>(dW), ld_dw, p, g, s)
    if (!few) SNN_CE(run, float);
    else if (dtype == SNN_F32) SNN_CE(run_few<float>, float);
    else if (dtype == SNN_BF16) SNN_CE(run_few<Bf16>, Bf16);
    else SNN_CE(run_few<F16>, F16);
    return launch_status();
  }
  const Plan16 p = plan16_of((int)R, H, C);
  const Workspace16 g = carve16(workspace, (int)R, H, C, dx || dW, p);
  if (workspace_bytes < g.bytes) return SNN_ERR_INVALID_ARG;
  if (dtype == SNN_BF16) SNN_CE(run16<Bf16>, Bf16);
  else SNN_CE(run16<F16>, F16);
#undef SNN_CE
  return launch_status();
}
