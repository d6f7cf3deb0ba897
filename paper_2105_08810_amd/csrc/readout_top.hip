// A teacher's record of its answers: the K largest logits of every row with their classes, largest first and equal
// ones by class, and the row's log-sum-exp at a temperature, which gives the listed classes' probabilities and what
// is left for the others.
#include "rows.h"

namespace snn {
namespace {

using namespace rows;

template <int NT>
struct TopLds {
  SelectLds<NT> select;
  uint64_t taken[kMaxListed];
  float fred[NT / kWave];
  uint32_t n_taken;
};

template <class T, int NT>
__global__ __launch_bounds__(NT) void top_rows(const void* __restrict__ logits, int C, int64_t ld, int K, float inv,
                                               int32_t* __restrict__ ids, float* __restrict__ vals,
                                               float* __restrict__ lse) {
  __shared__ TopLds<NT> s;
  constexpr int kVec = Row<T>::kVec;
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const Row<T> row(logits, r, ld, C);
  float m = -INFINITY, least = INFINITY;
  uint64_t count = 0;
  for (int q = tid; q < row.Q; q += NT) {
    float x[kVec];
    row.load(q, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const float y = no_nan(x[i]);
      m = fmaxf(m, y);
      if (y > -INFINITY) {
        least = fminf(least, y);
        ++count;
      }
    }
  }
  const auto larger = [](float a, float b) { return fmaxf(a, b); };
  const auto smaller = [](float a, float b) { return fminf(a, b); };
  const auto add = [](auto a, auto b) { return a + b; };
  m = block_reduce<NT>(m, larger, s.fred);
  least = block_reduce<NT>(least, smaller, s.fred);
  count = block_reduce<NT>(count, add, s.select.red);
  if (lse) {
    float sum = 0.0f;
    const float safe = isinf(m) ? 0.0f : m;
    for (int q = tid; q < row.Q; q += NT) {
      float x[kVec];
      row.load(q, x);
#pragma unroll
      for (int i = 0; i < kVec; ++i) sum += expf((no_nan(x[i]) - safe) * inv);
    }
    sum = block_reduce<NT>(sum, add, s.fred);
    if (tid == 0) lse[r] = isinf(m) ? m : m * inv + logf(sum);
  }
  uint32_t cut_key = 0;
  int last = C;  // class of the last listed element at the cut
  if (count > (uint64_t)K) {
    const auto one = [](float x) { return (uint32_t)(x > -INFINITY); };
    const Cut c = find_cut<T, NT, false>(row, one, key_of(least), key_of(m), (uint64_t)K, s.select);
    cut_key = c.key;
    const uint32_t ties = K - c.above_count;
    if (ties < c.equal)
      last = find_in_order<T, NT>(row, [&](float x, int) { return (uint64_t)(key_of(x) == cut_key); }, ties - 1,
                                  s.select.red);
  }
  __syncthreads();
  if (tid == 0) s.n_taken = 0;
  __syncthreads();
  for (int q = tid; q < row.Q; q += NT) {
    float x[kVec];
    row.load(q, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const float y = no_nan(x[i]);
      const int j = row.first(q) + i;
      const uint32_t k = key_of(y);
      if (y > -INFINITY && (k > cut_key || (k == cut_key && j <= last)))
        s.taken[atomicAdd(&s.n_taken, 1u)] = (uint64_t)~k << 32 | (uint32_t)j;
    }
  }
  __syncthreads();
  const int n = (int)s.n_taken;
  for (int e = tid; e < K; e += NT) {
    int place = e, id = -1;
    float v = -INFINITY;
    if (e < n) {
      const uint64_t mine = s.taken[e];
      place = 0;
      for (int o = 0; o < n; ++o) place += s.taken[o] < mine;
      id = (int)(uint32_t)mine;
      v = row.at(id);
    }
    ids[r * K + place] = id;
    vals[r * K + place] = v;
  }
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" snn_status snn_readout_top(const void* logits, int dtype, int64_t R, int C, int64_t ld, int K, float tau,
                                      int32_t* ids, float* vals, float* lse, void* stream) {
  const snn_status ok = rows::check_rows(logits, dtype, R, C, ld);
  if (ok != SNN_OK) return ok;
  if (!ids || !vals || K <= 0 || K > C || !(tau > 0.0f) || isinf(tau)) return SNN_ERR_INVALID_ARG;
  if (K > rows::kMaxListed) return SNN_ERR_UNSUPPORTED;
  const float inv = 1.0f / tau;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return rows::for_type(dtype, [&](auto type) {
    using T = decltype(type);
    if (C <= 1024)
      hipLaunchKernelGGL((top_rows<T, 64>), dim3((unsigned)R), dim3(64), 0, s, logits, C, ld, K, inv, ids, vals, lse);
    else if (C <= 16384)
      hipLaunchKernelGGL((top_rows<T, 256>), dim3((unsigned)R), dim3(256), 0, s, logits, C, ld, K, inv, ids, vals, lse);
    else
      hipLaunchKernelGGL((top_rows<T, 1024>), dim3((unsigned)R), dim3(1024), 0, s, logits, C, ld, K, inv, ids, vals,
                         lse);
    return launch_status();
  });
}
