// Distillation of a student's rows of logits z against a teacher's records (K classes with their logits v, and the
// teacher's log-sum-exp L at the same temperature tau), with the gradient:
//   p_k = exp(v_k/tau - L), p_t = max(0, 1 - sum p) for the classes not listed; without L, p = softmax(v/tau) and
//   p_t = 0; mass = sum p + p_t; q = softmax(z/tau), q_t = its sum over the classes not listed
//   loss of a row = sum_k p_k (log p_k - log q_k) + p_t (log p_t - log q_t)
//   d loss / d z_j = (mass q_j - p_j) / tau for a listed class, (mass q_t - p_t) (q_j / q_t) / tau for another
// The classes not listed are summed by themselves, not as 1 - sum q_k: the difference of two sums of the whole row
// would leave nothing of a small q_t. All sums and the gradient are float32, the loss over the rows float64.
//
// A row is read once and its gradient written once where it fits a block's registers. The exponentials
// are kept there, each thread's relative to its own largest logit, so that the only barrier between reading and writing
// is the one that joins the threads' sums; a factor per thread then makes them gradients. The K listed classes have
// their bit in LDS, count as -inf in that pass, and get their own gradient after it. The teacher's side (K values) is
// formed by every wave for itself, which needs no barrier.
//   distill_small  16 lanes a row (up to 8 values each), four rows a wave: rows of up to 128 values
//   distill_tile   a block a row, in registers
//   distill_rows   a block a row, read twice: rows beyond the registers
//
// Measured: 128000 x 100 float32, K 8: 34.6 us (3.1 TB/s, vector instructions issued 98% of the time); 2048 x 32003
// bfloat16, K 64: 72 us (3.6 TB/s, 59%); 512 x 131072 float32, K 32: 139 us (3.9 TB/s of one read and the write; the
// second read passes the L2 caches but for a tenth; 41%).
#include "rows.h"

namespace snn {
namespace {

using namespace rows;

constexpr float kLog2e = 1.44269504088896340736f;

// A sum of exp(x / tau) over some logits x: the largest of them, and the sum relative to it. Logits are subtracted before
// they are scaled by c = log2(e) / tau: the product of one could overflow (masks of the type's lowest value), and its
// rounding be more than a row's logits span.
struct Sum2 {
  float max, total;
};
__device__ __forceinline__ float or_zero(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ float power(float x, float from, float c) { return exp2_fast((x - from) * c); }
__device__ __forceinline__ Sum2 join(Sum2 a, Sum2 b, float c) {
  const float m = fmaxf(a.max, b.max);
  const float safe = or_zero(m);
  return Sum2{m, a.total * power(a.max, safe, c) + b.total * power(b.max, safe, c)};
}
__device__ __forceinline__ bool empty(Sum2 a) { return a.max == -INFINITY && a.total == 0.0f; }

// One maximum and one rescaled sum for the wave (a join at each step would form two exponentials).
__device__ __forceinline__ Sum2 wave_join(Sum2 v, float c) {
  const float m = wave_reduce(v.max, Larger());
  return Sum2{m, wave_reduce(v.total * power(v.max, or_zero(m), c), Plus())};
}

template <int NT>
__device__ __forceinline__ Sum2 block_join(Sum2 v, float c, Sum2* red) {
  v = wave_join(v, c);
  if (NT == kWave) return v;
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = v;
  __syncthreads();
  float m = red[0].max;
#pragma unroll
  for (int k = 1; k < NT / kWave; ++k) m = fmaxf(m, red[k].max);
  float total = 0.0f;
#pragma unroll
  for (int k = 0; k < NT / kWave; ++k) total += red[k].total * power(red[k].max, or_zero(m), c);
  return Sum2{m, total};
}

struct Distill {
  const void* logits;
  int C;
  int64_t ld;
  const int32_t* ids;
  const float* vals;
  const float* lse;
  int K;
  float tau;
  const float* weight;
  float mean;  // every row's weight where there is no array of them
  int64_t R;   // rows of this launch
  float* row_loss;
  void* grad;
  int64_t ld_grad;
  int accumulate;
  double* part;  // a block's sum of weight * loss; NULL where there is one block, which writes the loss
  float* loss;
  __device__ __forceinline__ void add(int64_t block, double v) const {
    if (!part) *loss = (float)v;
    else part[block] = v;
  }
  __device__ __forceinline__ float weight_of(int64_t r) const { return weight ? weight[r] : mean; }
};

// (x - from) / tau, rounded by itself: not contracted with what it is added to.
__device__ __forceinline__ float over_tau(float x, float from, float inv_tau) {
#pragma clang fp contract(off)
  return (x - from) * inv_tau;
}
// What logarithms are relative to where the largest value is `top`: beside a number far from 0 float32 keeps too little of
// a sum's logarithm, and beside a type's lowest value nothing.
__device__ __forceinline__ float far_from_zero(float top, float inv_tau) {
  return fabsf(top * inv_tau) < 1024.0f || isinf(top) ? 0.0f : top;
}

// What a row's loss and gradient need of its sums.
struct RowSums {
  float loss;
  float from, lse;   // log q_j = (z_j - from) / tau - lse; 0 for a row with nothing in it, whose z are all -inf
  float max, per;    // q_j = 2^((z_j - max) c) per
  float mass;
  float factor;      // of 2^((z_j - rest.max) c) for a class that is not listed, without weight / tau
};
// The loss is that of the classes not listed; the caller adds the others' terms. Logarithms are differences of float32
// log-sum-exps, so a loss is exact to about 2^-23 |lse|; the gradient takes ratios of sums.
__device__ __forceinline__ RowSums row_sums(Sum2 rest, Sum2 own, float listed_p, float p_t, float c, float inv_tau) {
  RowSums s;
  const Sum2 all = join(rest, own, c);
  const bool none = empty(all);  // q = 0
  s.max = or_zero(all.max);
  s.per = none ? 0.0f : 1.0f / all.total;
  s.mass = listed_p + p_t;
  const float q_t = empty(rest) ? 0.0f : rest.total * power(rest.max, s.max, c) * s.per;
  s.factor = empty(rest) ? 0.0f * s.per : (s.mass * q_t - p_t) * (1.0f / rest.total);  // NaN with a NaN in either
  s.from = far_from_zero(all.max, inv_tau);
  const float lse_t = over_tau(rest.max, s.from, inv_tau) + logf(rest.total);  // -inf where there is nothing
  const float own_max = over_tau(own.max, s.from, inv_tau), top = or_zero(fmaxf(own_max, lse_t));
  s.lse = none ? 0.0f : top + logf(expf(lse_t - top) + own.total * expf(own_max - top));
  s.loss = p_t > 0.0f ? p_t * (logf(p_t) - (lse_t - s.lse)) : s.lse == s.lse ? 0.0f : s.lse;
  return s;
}
__device__ __forceinline__ float left_of(float listed_p) {  // max(0, 1 - p); a NaN stays one
  return listed_p < 1.0f ? 1.0f - listed_p : listed_p >= 1.0f ? 0.0f : listed_p;
}

// ------------------------------------------------------------------ 16 lanes a row

// A lane's vectors are next to one another: value i of lane l is number l * kEach + i from the row's aligned address.
template <class T>
struct Small {
  static constexpr int kVec = Row<T>::kVec;
  static constexpr int kEach = 8;
  static constexpr int NV = kEach / kVec;
  static constexpr int kValues = 16 * kEach;
};

constexpr int kNotListed = 0x7fffffff;  // a NaN that no listed value has
__device__ __forceinline__ int listed_bits(float v) { return __float_as_int(v == v ? v : NAN); }

template <class T, int ROWS>
__global__ __launch_bounds__(16 * ROWS) void distill_small(Distill a) {
  using S = Small<T>;
  constexpr int kVec = S::kVec, kEach = S::kEach, NV = S::NV;
  __shared__ __attribute__((aligned(16))) int table[ROWS][S::kValues];  // the listed values
  __shared__ double part[ROWS];
  const int slot = threadIdx.x / 16, l = threadIdx.x % 16;
  const int64_t r = (int64_t)blockIdx.x * ROWS + slot;
  const int C = a.C, K = a.K;
  // what does not wait for the weight is fetched beside it: the lane's first entry, the teacher's log-sum-exp
  const int64_t at = min(r, a.R - 1);
  const Row<T> row(a.logits, at, a.ld, C);
  const float w = r < a.R ? a.weight_of(r) : 0.0f;
  const int id0 = l < K ? a.ids[at * K + l] : -1;
  const float v0 = l < K ? a.vals[at * K + l] : 0.0f;
  const float lse = a.lse ? a.lse[at] : 0.0f;
  int4* mine = reinterpret_cast<int4*>(&table[slot][l * kEach]);
  mine[0] = mine[1] = make_int4(kNotListed, kNotListed, kNotListed, kNotListed);
  const bool live = w != 0.0f;
  uint4 raw[NV];
  if (live) {
    const int from = row.lead ? 1 : 0, to = (row.lead + C) / kVec;  // whole vectors
    if (to > from) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        raw[i] = *reinterpret_cast<const uint4*>(row.base + min(max(l * NV + i, from), to - 1) * kVec);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (l * NV + i < from || l * NV + i >= to) raw[i] = load_raw(row, l * NV + i);
  }
  __syncthreads();
  const float inv_tau = 1.0f / a.tau;
  if (live) {
    if (id0 >= 0 && id0 < C) table[slot][row.lead + id0] = listed_bits(v0);
    for (int k = l + 16; k < K; k += 16) {
      const int id = a.ids[r * K + k];
      if (id >= 0 && id < C) table[slot][row.lead + id] = listed_bits(a.vals[r * K + k]);
    }
  }
  __syncthreads();
  float loss = 0.0f;
  if (live) {
    float x[kEach], lp[kEach];
    bool listed[kEach];
    const int4 t[2] = {mine[0], mine[1]};
    __builtin_memcpy(lp, t, sizeof(lp));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float y[kVec];
      unpack<T>(raw[i], y);
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[i * kVec + e] = y[e];
    }
    float count = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      listed[i] = __float_as_int(lp[i]) != kNotListed;
      lp[i] = listed[i] ? lp[i] : -INFINITY;
      count += listed[i] ? 1.0f : 0.0f;
    }
    // the teacher: log p, and the sum of p
    float shift;
    if (a.lse) {
      shift = lse;
#pragma unroll
      for (int i = 0; i < kEach; ++i) lp[i] = over_tau(lp[i], 0.0f, inv_tau);
    } else {
      float top = lp[0], z = 0.0f;
#pragma unroll
      for (int i = 1; i < kEach; ++i) top = fmaxf(top, lp[i]);
      top = row16_reduce(top, Larger());
      const float from = far_from_zero(top, inv_tau);
      top = or_zero(over_tau(top, from, inv_tau));
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        lp[i] = over_tau(lp[i], from, inv_tau);
        z += exp2_fast((lp[i] - top) * kLog2e);
      }
      z = row16_reduce(z, Plus());
      shift = z == 0.0f ? 0.0f : top + logf(z);
    }
    float p[kEach], listed_p = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      lp[i] -= shift;
      p[i] = listed[i] ? exp2_fast(lp[i] * kLog2e) : 0.0f;
      listed_p += p[i];
    }
    listed_p = row16_reduce(listed_p, Plus());
    count = row16_reduce(count, Plus());
    const float p_t = a.lse && count < (float)C ? left_of(listed_p) : 0.0f;
    // the student
    const float c = kLog2e * inv_tau;
    Sum2 rest{-INFINITY, 0.0f}, own{-INFINITY, 0.0f};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      rest.max = fmaxf(rest.max, listed[i] ? -INFINITY : x[i]);
      own.max = fmaxf(own.max, listed[i] ? x[i] : -INFINITY);
    }
    rest.max = row16_reduce(rest.max, Larger());
    own.max = row16_reduce(own.max, Larger());
    float e[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      e[i] = power(x[i], or_zero(listed[i] ? own.max : rest.max), c);
      rest.total += listed[i] ? 0.0f : e[i];
      own.total += listed[i] ? e[i] : 0.0f;
    }
    rest.total = row16_reduce(rest.total, Plus());
    own.total = row16_reduce(own.total, Plus());
    const RowSums s = row_sums(rest, own, listed_p, p_t, c, inv_tau);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (listed[i] && !(p[i] <= 0.0f)) loss += p[i] * (lp[i] - (over_tau(x[i], s.from, inv_tau) - s.lse));
    loss = row16_reduce(loss, Plus()) + s.loss;
    if (a.grad) {
      const Row<T> out(a.grad, r, a.ld_grad, C);
      const float scale = w * inv_tau;
      const float own_per = scale * s.mass * power(own.max, s.max, c) * s.per;  // 0 where all of them are -inf
      const float rest_per = scale * s.factor;
      float g[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) g[i] = listed[i] ? fmaf(e[i], own_per, -scale * p[i]) : e[i] * rest_per;
      if (out.lead == row.lead) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float y[kVec];
          if (a.accumulate) out.load(l * NV + i, y);
#pragma unroll
          for (int v = 0; v < kVec; ++v) y[v] = a.accumulate ? y[v] + g[i * kVec + v] : g[i * kVec + v];
          store_vec(out, l * NV + i, y);
        }
      } else {
        T* to = const_cast<T*>(out.base) + out.lead;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int j = l * kEach + i - row.lead;
          if (j >= 0 && j < C) to[j] = from_float<T>(a.accumulate ? to_float(to[j]) + g[i] : g[i]);
        }
      }
    }
  } else if (r < a.R && a.grad && !a.accumulate) {
    T* to = static_cast<T*>(a.grad) + r * a.ld_grad;
    for (int j = l; j < C; j += 16) to[j] = from_float<T>(0.0f);
  }
  if (l == 0) {
    part[slot] = live ? (double)w * (double)loss : 0.0;
    if (r < a.R && a.row_loss) a.row_loss[r] = loss;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double v = 0.0;
    for (int k = 0; k < ROWS; ++k) v += part[k];
    a.add(blockIdx.x, v);
  }
}

// ------------------------------------------------------------------ a block a row

// The row's entries as every wave holds them, entry k at lane k % 64: the first kHeld of a lane with their student's
// logit in registers, fetched before anything waits for the row; the others are read where they are needed.
constexpr int kHeld = 2;
template <class T>
struct Entries {
  const int32_t* ids;
  const float* vals;
  int K, C;
  float held_v[kHeld];
  float x[kHeld];
  int id[kHeld];            // -1: no entry
  float inv_tau;
  const Row<T>& row;

  __device__ __forceinline__ Entries(const Distill& a, int64_t r, const Row<T>& row_)
      : ids(a.ids + r * a.K), vals(a.vals + r * a.K), K(a.K), C(a.C), inv_tau(1.0f / a.tau), row(row_) {
#pragma unroll
    for (int e = 0; e < kHeld; ++e) {
      const int k = threadIdx.x % kWave + e * kWave;
      id[e] = k < K ? ids[k] : -1;
      held_v[e] = k < K ? vals[k] : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < kHeld; ++e) {
      if (id[e] >= C) id[e] = -1;
      x[e] = id[e] >= 0 ? row.at(id[e]) : 0.0f;
    }
  }
  // f(id, v, student's logit) of the lane's entries
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
      if (id[e] >= 0) f(id[e], held_v[e], x[e]);
    for (int k = threadIdx.x % kWave + kHeld * kWave; k < K; k += kWave) {
      const int j = ids[k];
      if (j >= 0 && j < C) f(j, vals[k], row.at(j));
    }
  }
};

struct Teacher {
  float from, shift, inv_tau;
  float listed_p, p_t;
  __device__ __forceinline__ float log_p(float v) const { return over_tau(v, from, inv_tau) - shift; }
};
// Also sets the listed classes' bits (by the first wave).
template <class T>
__device__ __forceinline__ Teacher teacher_of(const Distill& a, int64_t r, const Entries<T>& entries, uint32_t* bits) {
  if (threadIdx.x < kWave)
    entries.each([&](int id, float, float) {
      const int v = entries.row.lead + id;
      atomicOr(&bits[v >> 5], 1u << (v & 31));
    });
  Teacher t;
  t.from = 0.0f;
  t.inv_tau = entries.inv_tau;
  if (a.lse) {
    t.shift = a.lse[r];
  } else {
    float top = -INFINITY, z = 0.0f;
    entries.each([&](int, float v, float) { top = fmaxf(top, v); });
    top = wave_reduce(top, Larger());
    t.from = far_from_zero(top, t.inv_tau);
    top = or_zero(over_tau(top, t.from, t.inv_tau));
    entries.each([&](int, float v, float) { z += expf(over_tau(v, t.from, t.inv_tau) - top); });
    z = wave_reduce(z, Plus());
    t.shift = z == 0.0f ? 0.0f : top + logf(z);
  }
  float p = 0.0f, n = 0.0f;
  entries.each([&](int, float v, float) {
    p += expf(t.log_p(v));
    n += 1.0f;
  });
  t.listed_p = wave_reduce(p, Plus());
  n = wave_reduce(n, Plus());
  t.p_t = a.lse && n < (float)a.C ? left_of(t.listed_p) : 0.0f;
  return t;
}

// Joins the listed classes to the others' sum, forms the row's loss (every wave for itself).
template <class T>
__device__ __forceinline__ RowSums finish_row(const Entries<T>& entries, const Teacher& t, Sum2 rest, float c) {
  float top = -INFINITY, z = 0.0f;
  entries.each([&](int, float, float x) { top = fmaxf(top, x); });
  top = wave_reduce(top, Larger());
  entries.each([&](int, float, float x) { z += power(x, or_zero(top), c); });
  RowSums s = row_sums(rest, Sum2{top, wave_reduce(z, Plus())}, t.listed_p, t.p_t, c, t.inv_tau);
  float loss = 0.0f;
  entries.each([&](int, float v, float x) {
    const float lp = t.log_p(v), p = expf(lp);
    if (!(p <= 0.0f)) loss += p * (lp - (over_tau(x, s.from, t.inv_tau) - s.lse));
  });
  s.loss += wave_reduce(loss, Plus());
  return s;
}

// The listed classes' gradients by the first wave, over what the pass over the row left there (nothing added to it).
template <class T>
__device__ __forceinline__ void listed_grads(const Distill& a, int64_t r, const Entries<T>& entries, const Teacher& t,
                                             const RowSums& s, float c, float scale) {
  T* grad = static_cast<T*>(a.grad) + r * a.ld_grad;
  __syncthreads();
  if (threadIdx.x < kWave)
    entries.each([&](int id, float v, float x) {
      const float q = power(x, s.max, c) * s.per;
      const float g = scale * (s.mass * q - expf(t.log_p(v)));
      grad[id] = from_float<T>(a.accumulate ? to_float(grad[id]) + g : g);
    });
}

// Vector q of the gradient.
template <class T>
__device__ __forceinline__ void put(const Distill& a, const Row<T>& row, const Row<T>& out, int q,
                                    const float (&x)[16 / sizeof(T)]) {
  constexpr int kVec = Row<T>::kVec;
  if (out.lead == row.lead) {
    float y[kVec];
    if (a.accumulate) {
      out.load(q, y);
#pragma unroll
      for (int i = 0; i < kVec; ++i) y[i] += x[i];
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i) y[i] = x[i];
    }
    store_vec(out, q, y);
  } else {
    T* to = const_cast<T*>(out.base) + out.lead;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int j = row.first(q) + i;
      if (j >= 0 && j < a.C) to[j] = from_float<T>(a.accumulate ? to_float(to[j]) + x[i] : x[i]);
    }
  }
}

// Has the compiler unpack a vector anew where it is used next, instead of keeping its values from the last time: 32
// registers instead of 64 for a thread's 64 16-bit values.
__device__ __forceinline__ void forget(uint4& u) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));
#endif
}

// A vector with -inf for the values whose bits are on.
template <class T>
__device__ __forceinline__ uint4 without(const uint4& u, uint32_t on) {
  constexpr int kVec = Row<T>::kVec;
  T v[kVec];
  __builtin_memcpy(v, &u, 16);
#pragma unroll
  for (int k = 0; k < kVec; ++k) v[k] = on >> k & 1 ? lowest<T>() : v[k];
  uint4 w;
  __builtin_memcpy(&w, v, 16);
  return w;
}

template <class T, int NT>
__device__ __forceinline__ void row_without_weight(const Distill& a, int64_t r) {
  if (threadIdx.x == 0) {
    if (a.row_loss) a.row_loss[r] = 0.0f;
    a.add(r, 0.0);
  }
  if (a.grad && !a.accumulate) {
    const Row<T> out(a.grad, r, a.ld_grad, a.C);
    const float zero[Row<T>::kVec] = {};
    for (int q = threadIdx.x; q < out.Q; q += NT) store_vec(out, q, zero);
  }
}

template <class T, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void distill_tile(Distill a) {
  constexpr int kVec = Row<T>::kVec;
  constexpr bool kKeep = sizeof(T) == 4;  // the exponentials in the logits' place; 16-bit rows form them twice
  __shared__ uint32_t bits[NT * NV * kVec / 32];
  __shared__ Sum2 red[NT / kWave];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const float w = a.weight_of(r);
  if (w == 0.0f) return row_without_weight<T, NT>(a, r);  // not read: what is there may be anything
  const Row<T> row(a.logits, r, a.ld, a.C);
  const Entries<T> entries(a, r, row);
  uint4 raw[NV];
  load_vectors<T, NT>(row, raw, 0, row.Q);
  for (int k = tid; k < (row.Q * kVec + 31) / 32; k += NT) bits[k] = 0;
  __syncthreads();
  const Teacher t = teacher_of<T>(a, r, entries, bits);
  __syncthreads();
  const float c = kLog2e / a.tau;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int q = i * NT + tid, v = q * kVec;
    const uint32_t on = q < row.Q ? bits[v >> 5] >> (v & 31) & ((1u << kVec) - 1) : 0;
    if (on) raw[i] = without<T>(raw[i], on);  // few vectors hold a listed class
    float x[kVec];
    unpack<T>(raw[i], x);
#pragma unroll
    for (int k = 0; k < kVec; ++k) top = fmaxf(top, x[k]);
    if (!kKeep) forget(raw[i]);
  }
  // one multiply-add a value, and the rounding of what the exponents are relative to as a factor of the thread's sum
  const Exponent at = exponent_of(top, c);
  const float exact = top == -INFINITY ? 1.0f : exp2_fast(-fmaf(top, at.c, -at.mc));
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float x[kVec];
    unpack<T>(raw[i], x);
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      x[k] = exp2_fast(fmaf(x[k], at.c, -at.mc));
      sum += x[k];
    }
    if (kKeep) __builtin_memcpy(&raw[i], x, 16);
    else forget(raw[i]);
  }
  const Sum2 rest = block_join<NT>(Sum2{top, sum * exact}, c, red);
  const RowSums s = finish_row<T>(entries, t, rest, c);
  if (tid == 0) {
    if (a.row_loss) a.row_loss[r] = s.loss;
    a.add(r, (double)w * (double)s.loss);
  }
  if (!a.grad) return;
  const Row<T> out(a.grad, r, a.ld_grad, a.C);
  const float scale = w / a.tau;
  const float per = scale * s.factor * (top == -INFINITY ? 0.0f : exact * power(top, rest.max, c));
  const auto gradient = [&](const uint4& u, float (&x)[kVec]) {
    if (kKeep) __builtin_memcpy(x, &u, 16);
    else unpack<T>(u, x);
#pragma unroll
    for (int k = 0; k < kVec; ++k) x[k] = kKeep ? x[k] * per : exp2_fast(fmaf(x[k], at.c, -at.mc)) * per;
  };
  const bool alike = out.lead == row.lead && !a.accumulate;
  const int from = out.lead ? 1 : 0, to = (out.lead + a.C) / kVec;  // whole vectors
  uint4 last = raw[0];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int q = i * NT + tid;
    if (i > 0 && q == to) last = raw[i];
    if (alike) {
      float x[kVec];
      T v[kVec];
      gradient(raw[i], x);
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] = from_float<T>(x[k]);
      uint4 u;
      __builtin_memcpy(&u, v, 16);
      if (q >= from && q < to) store_past(const_cast<T*>(out.base) + (size_t)q * kVec, u);
    }
  }
  if (alike) {  // the ends of the row
#pragma unroll 1
    for (int end = 0; end < 2; ++end) {
      const int q = end ? to : 0;
      if (end ? to < out.Q && to >= from && tid == to % NT : tid < from) {
        float x[kVec];
        gradient(end ? last : raw[0], x);
        store_vec(out, q, x);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i * NT + tid < row.Q) {
        float x[kVec];
        gradient(raw[i], x);
        put(a, row, out, i * NT + tid, x);
      }
  }
  listed_grads<T>(a, r, entries, t, s, c, scale);
}

template <class T, int NT>
__global__ __launch_bounds__(NT) void distill_rows(Distill a) {
  constexpr int kVec = Row<T>::kVec;
  extern __shared__ uint32_t bits[];
  __shared__ Sum2 red[NT / kWave];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const float w = a.weight_of(r);
  if (w == 0.0f) return row_without_weight<T, NT>(a, r);
  const Row<T> row(a.logits, r, a.ld, a.C);
  const Entries<T> entries(a, r, row);
  for (int k = tid; k < (row.Q * kVec + 31) / 32; k += NT) bits[k] = 0;
  __syncthreads();
  const Teacher t = teacher_of<T>(a, r, entries, bits);
  __syncthreads();
  const float c = kLog2e / a.tau;
  constexpr int kAhead = 4;  // vectors of a thread in flight
  const int steps = (row.Q + kAhead * NT - 1) / (kAhead * NT);
  auto pass = [&](bool back, auto f) {
    for (int step = 0; step < steps; ++step) {
      const int q0 = (back ? steps - 1 - step : step) * kAhead * NT + tid;
      uint4 raw[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (q0 + u * NT < row.Q) raw[u] = load_raw(row, q0 + u * NT);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int q = q0 + u * NT;
        if (q < row.Q) {
          float x[kVec];
          unpack<T>(raw[u], x);
          const int v = q * kVec;
          const uint32_t on = bits[v >> 5] >> (v & 31);
#pragma unroll
          for (int k = 0; k < kVec; ++k)
            if (on >> k & 1) x[k] = -INFINITY;
          f(x, q);
        }
      }
    }
  };
  Sum2 rest{-INFINITY, 0.0f};
  pass(false, [&](float (&x)[kVec], int) {
    float m = x[0];
#pragma unroll
    for (int k = 1; k < kVec; ++k) m = fmaxf(m, x[k]);
    m = fmaxf(rest.max, m);
    const float safe = or_zero(m);
    float v = rest.total * power(rest.max, safe, c);
#pragma unroll
    for (int k = 0; k < kVec; ++k) v += power(x[k], safe, c);
    rest = Sum2{m, v};
  });
  rest = block_join<NT>(rest, c, red);
  const RowSums s = finish_row<T>(entries, t, rest, c);
  if (tid == 0) {
    if (a.row_loss) a.row_loss[r] = s.loss;
    a.add(r, (double)w * (double)s.loss);
  }
  if (!a.grad) return;
  const Row<T> out(a.grad, r, a.ld_grad, a.C);
  const float scale = w / a.tau;
  const float per = scale * s.factor, safe = or_zero(rest.max);
  pass(true, [&](float (&x)[kVec], int q) {  // from the end, which was read last
#pragma unroll
    for (int k = 0; k < kVec; ++k) x[k] = power(x[k], safe, c) * per;
    put(a, row, out, q, x);
  });
  listed_grads<T>(a, r, entries, t, s, c, scale);
}

// Sums of `each` parts in a fixed order: one block writes the loss itself.
__global__ __launch_bounds__(1024) void distill_total(const double* __restrict__ part, int64_t n, int64_t each,
                                                      double* __restrict__ sums, float* __restrict__ loss) {
  __shared__ double red[1024 / kWave];
  const int64_t from = blockIdx.x * each, to = min(n, from + each);
  double v = 0.0;
#pragma unroll 4
  for (int64_t k = from + threadIdx.x; k < to; k += 1024) v += part[k];
  v = block_reduce<1024>(v, [](double a, double b) { return a + b; }, red);
  if (threadIdx.x == 0) {
    if (gridDim.x == 1) *loss = (float)v;
    else sums[blockIdx.x] = v;
  }
}

constexpr int64_t kTotalEach = 16384;  // parts of a block of the loss's sum

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" size_t snn_readout_distill_workspace(int64_t R, int C, int dtype) {
  if (R <= 0 || R > INT32_MAX || bad_dim(C) || C > rows::kMaxClasses || rows::type_size(dtype) == 0) return 0;
  Carve c(nullptr);
  c.take<double>((size_t)R);  // weighted losses of the rows or of groups of them
  c.take<double>((size_t)((R + kTotalEach - 1) / kTotalEach));
  return c.off;
}

extern "C" snn_status snn_readout_distill(const void* logits, int dtype, int64_t R, int C, int64_t ld,
                                          const int32_t* ids, const float* vals, const float* lse, int K, float tau,
                                          const float* weight, float* loss, float* row_loss, void* grad,
                                          int64_t ld_grad, int accumulate, void* workspace, size_t workspace_bytes,
                                          void* stream) {
  snn_status ok = rows::check_rows(logits, dtype, R, C, ld);
  if (ok != SNN_OK) return ok;
  if (grad) {
    ok = rows::check_rows(grad, dtype, R, C, ld_grad);
    if (ok != SNN_OK) return ok;
  }
  if (!ids || !vals || !loss || !workspace || K <= 0 || K > C || !(tau > 0.0f) || isinf(tau))
    return SNN_ERR_INVALID_ARG;
  if (workspace_bytes < snn_readout_distill_workspace(R, C, dtype)) return SNN_ERR_INVALID_ARG;
  if (K > rows::kMaxListed) return SNN_ERR_UNSUPPORTED;
  Carve ws(workspace);
  double* part = ws.take<double>((size_t)R);
  double* sums = ws.take<double>((size_t)((R + kTotalEach - 1) / kTotalEach));
  hipStream_t s = static_cast<hipStream_t>(stream);
  int64_t n = R;  // blocks, each with a part of the loss
  const snn_status launched = rows::for_type(dtype, [&](auto type) {
    using T = decltype(type);
    constexpr int kWide = sizeof(T) == 4 ? 16 : 8;  // 64 values of a thread in registers
    const int Q = rows::most_vectors<T>(logits, C, ld);
    const bool small = Q <= 16 * Small<T>::NV;
    // one block of all rows, which needs no launch for the loss (17 x 20 float32 5.6 us, 7.5 in blocks of 16 rows; 64 x 100
    // 7.4 and 7.8, kernels alone)
    if (small) n = R <= 64 ? 1 : (R + 15) / 16;
    // Rows of more vectors than 1024 threads hold four of, 16-bit rows and rows that fill the chip take narrow blocks with
    // kWide vectors a thread: 1 x 20000 float32 12.5 us in 1024 threads and 8.6 so, 1 x 10000 bfloat16 8.9 and 7.1, 300 x
    // 12000 float32 16.7 and 12.3; but 1 x 12000 float32 7.2 and 7.6, 256 x 16384 float32 11.8 and 12.8.
    const bool narrow = sizeof(T) == 2 || Q > 4 * 1024 || R > cu_count();
    return rows::in_launches(R, [&](int64_t first, int64_t count) {
      using rows::or_null;
      const Distill a{static_cast<const T*>(logits) + first * ld, C, ld, ids + first * K, vals + first * K,
                      or_null(lse, first), K, tau, or_null(weight, first), 1.0f / (float)R, count, or_null(row_loss, first),
                      or_null(static_cast<T*>(grad), first * ld_grad), ld_grad, accumulate,
                      n == 1 ? nullptr : part + (small ? first / 16 : first), loss};
      const dim3 grid((unsigned)count);
      if (small) {
        if (n == 1)  // and no launch for the loss
          hipLaunchKernelGGL((distill_small<T, 64>), dim3(1), dim3(1024), 0, s, a);
        else
          hipLaunchKernelGGL((distill_small<T, 16>), dim3((unsigned)((count + 15) / 16)), dim3(256), 0, s, a);
      } else if (Q <= 4 * 64) {
        hipLaunchKernelGGL((distill_tile<T, 64, 4>), grid, dim3(64), 0, s, a);
      } else if (Q <= 4 * 256) {
        hipLaunchKernelGGL((distill_tile<T, 256, 4>), grid, dim3(256), 0, s, a);
      } else if (Q <= kWide * 256 && narrow) {
        hipLaunchKernelGGL((distill_tile<T, 256, kWide>), grid, dim3(256), 0, s, a);
      } else if (Q <= kWide * 512 && narrow) {
        hipLaunchKernelGGL((distill_tile<T, 512, kWide>), grid, dim3(512), 0, s, a);
      } else if (sizeof(T) == 4 && Q <= 4 * 1024) {
        if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((distill_tile<T, 1024, 4>), grid, dim3(1024), 0, s, a);
      } else if (Q <= kWide * 1024) {
        hipLaunchKernelGGL((distill_tile<T, 1024, kWide>), grid, dim3(1024), 0, s, a);
      } else {
        const size_t lds = ((size_t)Q * Row<T>::kVec + 31) / 32 * 4;
        ensure_dynamic_lds((const void*)distill_rows<T, 1024>, (int)lds);
        hipLaunchKernelGGL((distill_rows<T, 1024>), grid, dim3(1024), lds, s, a);
      }
      return launch_status();
    });
  });
  if (launched != SNN_OK || n == 1) return launched;
  if (n > kTotalEach) {
    const int64_t blocks = (n + kTotalEach - 1) / kTotalEach;
    hipLaunchKernelGGL(distill_total, dim3((unsigned)blocks), dim3(1024), 0, s, part, n, kTotalEach, sums, loss);
    hipLaunchKernelGGL(distill_total, dim3(1), dim3(1024), 0, s, sums, blocks, blocks, sums, loss);
  } else {
    hipLaunchKernelGGL(distill_total, dim3(1), dim3(1024), 0, s, part, n, n, sums, loss);
  }
  return launch_status();
}
