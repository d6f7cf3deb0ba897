// Distillation of a student's rows of logits z against a teacher's records (K classes with their logits v, and the
// teacher's log-sum-exp L at the same temperature tau), with the gradient:
//   p_k = exp(v_k/tau - L), p_t = max(0, 1 - sum p) for the classes not listed; without L, p = softmax(v/tau) and
//   p_t = 0; mass = sum p + p_t; q = softmax(z/tau), q_t = its sum over the classes not listed
//   loss of a row = sum_k p_k (log p_k - log q_k) + p_t (log p_t - log q_t)
//   d loss / d z_j = (mass q_j - p_j) / tau for a listed class, (mass q_t - p_t) (q_j / q_t) / tau for another
// The classes not listed are summed by themselves, not as 1 - sum q_k: the difference of two sums of the whole row
// would leave nothing of a small q_t.
#include "rows.h"

namespace snn {
namespace {

using namespace rows;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// A sum of 2^x kept as total * 2^max.
struct Sum2 {
  float max, total;
};
__device__ __forceinline__ Sum2 join(Sum2 a, Sum2 b) {
  const float m = fmaxf(a.max, b.max);
  const float safe = m == -INFINITY ? 0.0f : m;
  return Sum2{m, a.total * exp2_fast(a.max - safe) + b.total * exp2_fast(b.max - safe)};
}

template <int NT>
struct DistillLds {
  Sum2 red[NT / kWave];
  float fred[NT / kWave];
  int ired[NT / kWave];
};

template <int NT>
__device__ __forceinline__ Sum2 block_join(Sum2 v, Sum2* red) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1)
    v = join(v, Sum2{__shfl_xor(v.max, off, kWave), __shfl_xor(v.total, off, kWave)});
  if (NT == kWave) return v;
  __syncthreads();
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = v;
  __syncthreads();
  Sum2 r = red[0];
#pragma unroll
  for (int k = 1; k < NT / kWave; ++k) r = join(r, red[k]);
  return r;
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
  int64_t R;
  float* row_loss;
  void* grad;
  int64_t ld_grad;
  int accumulate;
};

template <class T, int NT>
__global__ __launch_bounds__(NT) void distill_rows(Distill a) {
  extern __shared__ uint32_t listed[];  // a bit per class
  __shared__ DistillLds<NT> s;
  constexpr int kVec = Row<T>::kVec;
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const int C = a.C, K = a.K;
  T* grad = a.grad ? static_cast<T*>(a.grad) + r * a.ld_grad : nullptr;
  const float w = a.weight ? a.weight[r] : 1.0f / (float)a.R;
  if (w == 0.0f) {  // not read: what is there may be anything
    if (tid == 0) a.row_loss[r] = 0.0f;
    if (grad && !a.accumulate)
      for (int j = tid; j < C; j += NT) grad[j] = from_float<T>(0.0f);
    return;
  }
  const Row<T> row(a.logits, r, a.ld, C);
  const int32_t* ids = a.ids + r * K;
  const float* vals = a.vals + r * K;
  for (int k = tid; k < (C + 31) / 32; k += NT) listed[k] = 0;
  __syncthreads();
  const auto larger = [](float x, float y) { return fmaxf(x, y); };
  const auto add = [](auto x, auto y) { return x + y; };
  const float c = kLog2e / a.tau;
  // the teacher
  float top = -INFINITY;
  int n = 0;
  for (int k = tid; k < K; k += NT) {
    const int id = ids[k];
    if (id >= 0 && id < C) {
      atomicOr(&listed[id >> 5], 1u << (id & 31));
      top = fmaxf(top, vals[k]);
      ++n;
    }
  }
  n = block_reduce<NT>(n, add, s.ired);
  float shift;  // p_k = exp(v_k / tau - shift)
  if (a.lse) {
    shift = a.lse[r];
  } else {
    top = block_reduce<NT>(top, larger, s.fred) / a.tau;
    float z = 0.0f;
    for (int k = tid; k < K; k += NT)
      if (ids[k] >= 0 && ids[k] < C) z += expf(vals[k] / a.tau - top);
    z = block_reduce<NT>(z, add, s.fred);
    shift = top == -INFINITY ? 0.0f : top + logf(z);
  }
  float listed_p = 0.0f;
  for (int k = tid; k < K; k += NT)
    if (ids[k] >= 0 && ids[k] < C) listed_p += expf(vals[k] / a.tau - shift);
  listed_p = block_reduce<NT>(listed_p, add, s.fred);
  const float p_t = a.lse && n < C ? (listed_p < 1.0f ? 1.0f - listed_p : listed_p >= 1.0f ? 0.0f : listed_p) : 0.0f;
  const float mass = listed_p + p_t;
  __syncthreads();  // the bits
  // the student: the classes not listed, then the listed ones
  Sum2 rest{-INFINITY, 0.0f};
  for (int q = tid; q < row.Q; q += NT) {
    float x[kVec];
    row.load(q, x);
    float m = rest.max;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int j = row.first(q) + i;
      if (j < 0 || j >= C || (listed[j >> 5] >> (j & 31) & 1)) x[i] = -INFINITY;
      m = fmaxf(m, x[i] * c);
    }
    const float safe = m == -INFINITY ? 0.0f : m;
    float v = rest.total * exp2_fast(rest.max - safe);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v += exp2_fast(fmaf(x[i], c, -safe));
    rest = Sum2{m, v};
  }
  rest = block_join<NT>(rest, s.red);
  Sum2 all{-INFINITY, 0.0f};
  for (int k = tid; k < K; k += NT)
    if (ids[k] >= 0 && ids[k] < C) {
      const float x = row.at(ids[k]);
      const float m = x * c;
      all = join(all, Sum2{m, x == -INFINITY ? 0.0f : exp2_fast(fmaf(x, c, -m))});
    }
  all = join(block_join<NT>(all, s.red), rest);
  const bool none = all.max == -INFINITY && all.total == 0.0f;  // a row with nothing in it: q = 0
  const float base = none ? 0.0f : all.max;
  const float log_total = none ? 0.0f : logf(all.total);
  const float per = none ? 0.0f : 1.0f / all.total;
  const float rest_base = rest.max == -INFINITY ? 0.0f : rest.max;
  float loss = 0.0f;
  for (int k = tid; k < K; k += NT)
    if (ids[k] >= 0 && ids[k] < C) {
      const float lp = vals[k] / a.tau - shift, p = expf(lp);
      const float lq = fmaf(row.at(ids[k]), c, -base) * kLn2 - log_total;
      if (!(p <= 0.0f)) loss += p * (lp - lq);
    }
  loss = block_reduce<NT>(loss, add, s.fred);
  const float lq_t = (rest.max - base) * kLn2 + logf(rest.total) - log_total;  // -inf where there is nothing
  if (p_t > 0.0f) loss += p_t * (logf(p_t) - lq_t);
  if (tid == 0) a.row_loss[r] = loss;
  if (!grad) return;
  const float scale = w / a.tau;
  const float q_t = none ? 0.0f : rest.total * exp2_fast(rest_base - base) * per;
  const bool no_rest = rest.max == -INFINITY && rest.total == 0.0f;
  const float factor = no_rest ? 0.0f : scale * (mass * q_t - p_t) / rest.total;
  // the gradients of listed classes: read before the others are written, written after them
  constexpr int kEach = (kMaxListed + NT - 1) / NT;
  float mine[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int k = tid + e * NT;
    mine[e] = 0.0f;
    if (k < K && ids[k] >= 0 && ids[k] < C) {
      const float q = exp2_fast(fmaf(row.at(ids[k]), c, -base)) * per;
      mine[e] = scale * (mass * q - expf(vals[k] / a.tau - shift));
      if (a.accumulate) mine[e] += to_float(grad[ids[k]]);
    }
  }
  __syncthreads();
  for (int q = tid; q < row.Q; q += NT) {
    float x[kVec];
    row.load(q, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int j = row.first(q) + i;
      if (j >= 0 && j < C && !(listed[j >> 5] >> (j & 31) & 1)) {
        float g = exp2_fast(fmaf(x[i], c, -rest_base)) * factor;
        if (a.accumulate) g += to_float(grad[j]);
        grad[j] = from_float<T>(g);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int k = tid + e * NT;
    if (k < K && ids[k] >= 0 && ids[k] < C) grad[ids[k]] = from_float<T>(mine[e]);
  }
}

// loss = sum of w_r row_loss_r over the rows with a weight, in float64 and a fixed order.
__global__ __launch_bounds__(1024) void distill_total(const float* __restrict__ row_loss,
                                                      const float* __restrict__ weight, int64_t R,
                                                      float* __restrict__ loss) {
  __shared__ double red[1024 / kWave];
  double v = 0.0;
  for (int64_t r = threadIdx.x; r < R; r += 1024)
    v += weight ? (weight[r] != 0.0f ? (double)weight[r] * (double)row_loss[r] : 0.0) : (double)row_loss[r];
  v = block_reduce<1024>(v, [](double a, double b) { return a + b; }, red);
  if (threadIdx.x == 0) *loss = (float)(weight ? v : v / (double)R);
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" size_t snn_readout_distill_workspace(int64_t R, int C, int dtype) {
  if (R <= 0 || R > INT32_MAX || bad_dim(C) || C > rows::kMaxClasses || rows::type_size(dtype) == 0) return 0;
  Carve c(nullptr);
  c.take<float>((size_t)R);  // losses of the rows
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
  float* losses = ws.take<float>((size_t)R);
  if (row_loss) losses = row_loss;
  const Distill a{logits, C, ld, ids, vals, lse, K, tau, weight, R, losses, grad, ld_grad, accumulate};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const size_t lds = (size_t)(C + 31) / 32 * 4;
  return rows::for_type(dtype, [&](auto type) {
    using T = decltype(type);
    if (C <= 1024) {
      hipLaunchKernelGGL((distill_rows<T, 64>), dim3((unsigned)R), dim3(64), lds, s, a);
    } else if (C <= 16384) {
      hipLaunchKernelGGL((distill_rows<T, 256>), dim3((unsigned)R), dim3(256), lds, s, a);
    } else {
      ensure_dynamic_lds((const void*)distill_rows<T, 1024>, (int)lds);
      hipLaunchKernelGGL((distill_rows<T, 1024>), dim3((unsigned)R), dim3(1024), lds, s, a);
    }
    hipLaunchKernelGGL(distill_total, dim3(1), dim3(1024), 0, s, losses, weight, R, loss);
    return launch_status();
  });
}
