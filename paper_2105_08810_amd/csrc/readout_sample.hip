// One class per row drawn from its logits with temperature, top-k, top-p and min-p, from a given uniform number.
//   t_j = (z_j - max z) / temperature, e_j = exp(t_j), weight n_j = round(2^31 e_j)
//   kept: of the order by value (ties by class) the first top_k, of these the shortest prefix with a weight of at
//   least top_p of theirs, of these the classes with e_j >= min_p
//   drawn: the first class whose kept weights up to it, in the order of the classes, exceed floor(u * their sum)
// The weights are whole numbers, so every sum is exact and the answer does not depend on how it was summed.
#include "rows.h"

namespace snn {
namespace {

using namespace rows;

constexpr float kUnit = 2147483648.0f;   // 2^31
constexpr float kFaintest = 23.0f;       // exp(-23) 2^31 < 1/2: beyond it a weight is 0

// Settings of one row; a pointer that is NULL leaves its filter out.
struct Settings {
  const float* u;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
};

struct Weigh {
  float max, inv;
  __device__ __forceinline__ float e(float x) const {  // in this order of operations, each rounded
    return x == max ? 1.0f : expf((x - max) * inv);
  }
  __device__ __forceinline__ uint32_t operator()(float x) const {
    return x == -INFINITY ? 0u : (uint32_t)rintf(e(x) * kUnit);
  }
};

template <int NT>
struct SampleLds {
  SelectLds<NT> select;
  float fred[NT / kWave];
  int ired[NT / kWave];
};

template <class T, int NT>
__global__ __launch_bounds__(NT) void sample_rows(const void* __restrict__ logits, int C, int64_t ld, Settings set,
                                                  int32_t* __restrict__ cls, float* __restrict__ logp,
                                                  int32_t* __restrict__ kept) {
  __shared__ SampleLds<NT> s;
  constexpr int kVec = Row<T>::kVec;
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const Row<T> row(logits, r, ld, C);
  float m = -INFINITY;
  for (int q = tid; q < row.Q; q += NT) {
    float x[kVec];
    row.load(q, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) m = fmaxf(m, x[i]);
  }
  m = block_reduce<NT>(m, [](float a, float b) { return fmaxf(a, b); }, s.fred);
  auto answer = [&](int j, float lp, int n) {
    if (tid == 0) {
      cls[r] = j;
      if (logp) logp[r] = lp;
      if (kept) kept[r] = n;
    }
  };
  if (m == -INFINITY) return answer(-1, -INFINITY, 0);
  // beyond 1e30 every finite logit has the same weight
  float temperature = set.temperature ? set.temperature[r] : 1.0f;
  temperature = temperature > 1e30f ? 1e30f : temperature;
  int k = set.top_k ? set.top_k[r] : 0;
  if (k <= 0 || k > C) k = C;
  if (!(temperature > 0.0f)) k = 1;
  const Weigh weigh{m, 1.0f / temperature};
  if (k == 1) {  // the first of the largest
    int at = INT32_MAX;
    for (int q = tid; q < row.Q; q += NT) {
      float x[kVec];
      row.load(q, x);
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (x[i] == m) at = min(at, row.first(q) + i);
    }
    at = block_reduce<NT>(at, [](int a, int b) { return min(a, b); }, s.ired);
    return answer(at, 0.0f, 1);
  }
  // the weights of all and how many there are
  uint64_t sum = 0;
  uint64_t count = 0;
  for (int q = tid; q < row.Q; q += NT) {
    float x[kVec];
    row.load(q, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const uint32_t n = weigh(no_nan(x[i]));
      sum += n;
      count += n != 0;
    }
  }
  const auto add = [](uint64_t a, uint64_t b) { return a + b; };
  sum = block_reduce<NT>(sum, add, s.select.red);
  count = block_reduce<NT>(count, add, s.select.red);
  const uint32_t hi = key_of(m);
  const uint32_t lo = key_of(m - kFaintest * temperature);
  if ((uint64_t)k < count) {
    const Cut c = find_cut<T, NT, false>(row, weigh, lo, hi, (uint64_t)k, s.select);
    // the elements above the cut weigh what they weigh; those at it weigh the same each
    uint64_t above = 0;
    for (int q = tid; q < row.Q; q += NT) {
      float x[kVec];
      row.load(q, x);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float y = no_nan(x[i]);
        if (key_of(y) > c.key) above += weigh(y);
      }
    }
    sum = block_reduce<NT>(above, add, s.select.red) + (uint64_t)(k - c.above_count) * weigh(of_key(c.key));
  }
  uint64_t limit = sum;
  if (set.top_p) {
    const float p = set.top_p[r];
    if (!(p >= 1.0f)) limit = p > 0.0f ? (uint64_t)ceil((double)p * (double)sum) : 1;
    limit = limit < 1 ? 1 : limit;
  }
  const Cut c = find_cut<T, NT, true>(row, weigh, lo, hi, limit, s.select);
  const uint32_t each = weigh(of_key(c.key));
  const uint32_t ties = (uint32_t)((limit - c.above_mass + each - 1) / each);
  float least = set.min_p ? set.min_p[r] : 0.0f;
  least = least > 0.0f ? fminf(least, 1.0f) : 0.0f;
  int last = C;  // class of the last kept element at the cut
  if (ties < c.equal)
    last = find_in_order<T, NT>(row, [&](float x, int) { return (uint64_t)(key_of(x) == c.key); }, ties - 1,
                                s.select.red);
  auto share = [&](float x, int j) -> uint64_t {
    const uint32_t key = key_of(x);
    if (key < c.key || (key == c.key && j > last)) return 0;
    return weigh.e(x) >= least ? weigh(x) : 0;
  };
  uint64_t total = 0;
  count = 0;
  for (int q = tid; q < row.Q; q += NT) {
    float x[kVec];
    row.load(q, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const uint64_t n = share(no_nan(x[i]), row.first(q) + i);
      total += n;
      count += n != 0;
    }
  }
  total = block_reduce<NT>(total, add, s.select.red);
  count = block_reduce<NT>(count, add, s.select.red);
  const double at = floor((double)set.u[r] * (double)total);
  const uint64_t point = at > 0.0 ? (at < (double)total ? (uint64_t)at : total - 1) : 0;
  const int j = find_in_order<T, NT>(row, share, point, s.select.red);
  const float x = no_nan(row.at(j));
  const float t = x == m ? 0.0f : (x - m) * weigh.inv;
  answer(j, t - (float)log((double)total * (1.0 / kUnit)), (int)count);
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" snn_status snn_readout_sample(const void* logits, int dtype, int64_t R, int C, int64_t ld, const float* u,
                                         const float* temperature, const int32_t* top_k, const float* top_p,
                                         const float* min_p, int32_t* cls, float* logp, int32_t* kept, void* stream) {
  const snn_status ok = rows::check_rows(logits, dtype, R, C, ld);
  if (ok != SNN_OK) return ok;
  if (!u || !cls) return SNN_ERR_INVALID_ARG;
  const Settings set{u, temperature, top_k, top_p, min_p};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return rows::for_type(dtype, [&](auto type) {
    using T = decltype(type);
    if (C <= 1024)
      hipLaunchKernelGGL((sample_rows<T, 64>), dim3((unsigned)R), dim3(64), 0, s, logits, C, ld, set, cls, logp, kept);
    else if (C <= 16384)
      hipLaunchKernelGGL((sample_rows<T, 256>), dim3((unsigned)R), dim3(256), 0, s, logits, C, ld, set, cls, logp, kept);
    else
      hipLaunchKernelGGL((sample_rows<T, 1024>), dim3((unsigned)R), dim3(1024), 0, s, logits, C, ld, set, cls, logp,
                         kept);
    return launch_status();
  });
}
