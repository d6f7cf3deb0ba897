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

// exp(t) for t <= 0 (from -64 on; -64 for less): 2^(t log2 e) with the product in two parts, the whole of it apart. Within
// an ulp of the correctly rounded value; no test for what overflows.
__device__ __forceinline__ float exp_down(float t) {
#pragma clang fp contract(off)
  constexpr double kFull = 1.44269504088896340736;
  constexpr float kHigh = (float)kFull, kLow = (float)(kFull - (double)kHigh);
  t = fmaxf(t, -64.0f);
  const float h = t * kHigh, n = rintf(h);
  const float low = fmaf(t, kLow, fmaf(t, kHigh, -h));
  return ldexpf(exp2_fast((h - n) + low), (int)n);
}

struct Weigh {
  float max, inv;
  // In this order of operations, each rounded. Of infinities the largest is at 0 and others at -inf; any other row's
  // largest is at 0 by itself.
  __device__ __forceinline__ float t(float x) const { return x == max ? 0.0f : (x - max) * inv; }
  __device__ __forceinline__ float e(float x) const { return exp_down(t(x)); }
  __device__ __forceinline__ uint32_t of(float x, float e) const {
    return x == -INFINITY ? 0u : (uint32_t)rintf(e * kUnit);
  }
  __device__ __forceinline__ uint32_t operator()(float x) const { return of(x, e(x)); }
  // For a finite max and inv, where -inf has weight 0 by itself.
  __device__ __forceinline__ float plain_t(float x) const { return (x - max) * inv; }
};

struct Sample {
  const void* logits;
  int64_t R;
  int C;
  int64_t ld;
  Settings set;
  int32_t* cls;
  float* logp;
  int32_t* kept;
  __device__ __forceinline__ void answer(int64_t r, int j, float lp, int n) const {
    cls[r] = j;
    if (logp) logp[r] = lp;
    if (kept) kept[r] = n;
  }
};

// A row's settings with what leaves a filter out made plain.
struct RowSettings {
  float u, temperature, top_p, min_p;
  int k;  // 1 also where the largest logit is asked for
  __device__ __forceinline__ RowSettings(const Settings& set, int64_t r, int C) {
    u = set.u[r];
    temperature = set.temperature ? set.temperature[r] : 1.0f;
    temperature = temperature > 1e30f ? 1e30f : temperature;  // beyond it every finite logit has the same weight
    k = set.top_k ? set.top_k[r] : 0;
    if (k <= 0 || k > C) k = C;
    if (!(temperature > 0.0f)) k = 1;
    top_p = set.top_p ? set.top_p[r] : 1.0f;
    top_p = top_p > 0.0f ? fminf(top_p, 1.0f) : 0.0f;
    min_p = set.min_p ? set.min_p[r] : 0.0f;
    min_p = min_p > 0.0f ? fminf(min_p, 1.0f) : 0.0f;
  }
  // The weight that a prefix of the order has to reach, of `sum`.
  __device__ __forceinline__ uint64_t limit(uint64_t sum) const {
    if (top_p >= 1.0f) return sum;
    const uint64_t l = (uint64_t)ceil((double)top_p * (double)sum);
    return l < 1 ? 1 : l;
  }
  __device__ __forceinline__ uint64_t point(uint64_t total) const {
    const double at = floor((double)u * (double)total);
    return at > 0.0 ? (at < (double)total ? (uint64_t)at : total - 1) : 0;
  }
};

// log of a drawn class's share of the kept weights
__device__ __forceinline__ float log_share(const Weigh& weigh, float x, uint64_t total) {
  return weigh.t(x) - (float)log((double)total * (1.0 / kUnit));
}

// ------------------------------------------------------------------ short rows, 16 lanes each

template <class T>
__global__ __launch_bounds__(256) void sample_short(Sample a) {
  __shared__ uint64_t list[kShortRows][kShortRow];
  __shared__ uint32_t weight[kShortRows][kShortRow];
  const int slot = threadIdx.x / 16, l = threadIdx.x % 16;
  const int64_t r = (int64_t)blockIdx.x * kShortRows + slot;
  const bool live = r < a.R;
  const Row<T> row(a.logits, min(r, a.R - 1), a.ld, a.C);
  const RowSettings set(a.set, min(r, a.R - 1), a.C);
  float x[kShortEach];
  load_short(row, x);
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kShortEach; ++i) {
    x[i] = no_nan(x[i]);
    m = fmaxf(m, x[i]);
  }
  m = row16_reduce(m, Larger());
  const Weigh weigh{m, set.temperature > 0.0f ? 1.0f / set.temperature : INFINITY};
  const bool ordered = set.k < a.C || set.top_p < 1.0f;
  // Elements of these arrays are set by selects, never in a branch that only some lanes take: there the compiler kept
  // the arrays as vectors and lost a store.
  uint32_t w[kShortEach];
  uint64_t mine[kShortEach];
  float e[kShortEach];
  int n = 0;
#pragma unroll
  for (int i = 0; i < kShortEach; ++i) {
    w[i] = 0;
    mine[i] = 0;
    e[i] = 0.0f;
    if (16 * i < a.C) {
      e[i] = weigh.e(x[i]);
      w[i] = weigh.of(x[i], e[i]);
      mine[i] = (uint64_t)~key_of(x[i]) << 32 | (uint32_t)(16 * i + l);
      int count;
      const int at = n + row16_place(w[i] != 0, count);
      if (w[i]) {
        list[slot][at] = mine[i];
        weight[slot][at] = w[i];
      }
      n += count;
    }
  }
  __syncthreads();
  uint64_t limit = UINT64_MAX;
  uint64_t before[kShortEach] = {};
  if (ordered) {
    int rank[kShortEach] = {};
    for (int o = 0; o < n; ++o) {
      const uint64_t other = list[slot][o];
      const uint32_t its = weight[slot][o];
#pragma unroll
      for (int i = 0; i < kShortEach; ++i)
        if (16 * i < a.C) {
          const bool ahead = other < mine[i];
          rank[i] += ahead;
          before[i] += ahead ? its : 0;
        }
    }
    uint64_t sum = 0;
#pragma unroll
    for (int i = 0; i < kShortEach; ++i) {
      w[i] = rank[i] < set.k ? w[i] : 0;
      sum += w[i];
    }
    limit = set.limit(lane_of_row16(row16_upto64(sum)));
  }
  // the kept weights up to each class, in the order of the classes
  uint64_t upto[kShortEach], total = 0;
  int count = 0;
#pragma unroll
  for (int i = 0; i < kShortEach; ++i) {
    upto[i] = 0;
    w[i] = (before[i] < limit) & (e[i] >= set.min_p) ? w[i] : 0;
    if (16 * i < a.C) {
      upto[i] = total + row16_upto64(w[i]);
      total = lane_of_row16(upto[i]);
      int kept;
      row16_place(w[i] != 0, kept);
      count += kept;
    }
  }
  if (!live) return;
  if (total == 0) {
    if (l == 0) a.answer(r, -1, -INFINITY, 0);
    return;
  }
  const uint64_t point = set.point(total);
#pragma unroll
  for (int i = 0; i < kShortEach; ++i)
    if (w[i] && upto[i] > point && upto[i] - w[i] <= point) a.answer(r, 16 * i + l, log_share(weigh, x[i], total), count);
}

// ------------------------------------------------------------------ any row, read in passes

template <int NT>
struct GeneralLds {
  SelectLds<NT> select;
  float fred[NT / kWave];
  int ired[NT / kWave];
};

template <class T, int NT>
__device__ __forceinline__ void sample_general(const Sample& a, int64_t r, const Row<T>& row, const RowSettings& set,
                                               GeneralLds<NT>& s) {
  constexpr int kVec = Row<T>::kVec;
  const int tid = threadIdx.x;
  const int C = a.C;
  float m = -INFINITY;
  for (int q = tid; q < row.Q; q += NT) {
    float x[kVec];
    row.load(q, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) m = fmaxf(m, x[i]);
  }
  m = block_reduce<NT>(m, Larger(), s.fred);
  if (m == -INFINITY) {
    if (tid == 0) a.answer(r, -1, -INFINITY, 0);
    return;
  }
  if (set.k == 1) {  // the first of the largest
    int at = INT32_MAX;
    for (int q = tid; q < row.Q; q += NT) {
      float x[kVec];
      row.load(q, x);
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (x[i] == m) at = min(at, row.first(q) + i);
    }
    at = block_reduce<NT>(at, [](int x, int y) { return min(x, y); }, s.ired);
    if (tid == 0) a.answer(r, at, 0.0f, 1);
    return;
  }
  const Weigh weigh{m, 1.0f / set.temperature};
  // Passes over the row: the weights of all and how many there are; then, the cut known, of the kept.
  Cut cut{0, 0, 0, 0};
  int last = C;  // class of the last kept element at the cut
  uint64_t ties = 0;
  bool by_share = false;
  const auto part_of = [&](float x, int j) -> uint64_t {
    const uint32_t key = key_of(x);
    if (!by_share) return key == cut.key;
    if (key < cut.key || (key == cut.key && j > last)) return 0;
    const float e = weigh.e(x);
    return e >= set.min_p ? weigh.of(x, e) : 0;
  };
  uint64_t sum = 0, count = 0, target = 0;
#pragma unroll 1
  for (int round = 0; round < 2; ++round) {
    by_share = true;  // round 0: with no cut, and any e
    sum = count = 0;
#pragma unroll 1
    for (int q = tid; q < row.Q; q += NT) {
      float x[kVec];
      row.load(q, x);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float y = no_nan(x[i]);
        const uint64_t n = round == 0 ? weigh(y) : part_of(y, row.first(q) + i);
        sum += n;
        count += n != 0;
      }
    }
    sum = block_sum64<NT>(sum, s.select.red);
    count = block_sum64<NT>(count, s.select.red);
    if (round == 0) {
      const uint32_t hi = key_of(m), lo = key_of(m - kFaintest * set.temperature);
      uint64_t limit = (uint64_t)set.k;
#pragma unroll 1
      for (int by_mass = (uint64_t)set.k < count ? 0 : 1; by_mass < 2; ++by_mass) {
        if (by_mass) limit = set.limit(sum);
        cut = find_cut<T, NT, true>(row, weigh, lo, hi, limit, by_mass != 0, s.select);
        // what lies at the cut weighs the same each
        const uint64_t each = weigh(of_key(cut.key));
        ties = by_mass ? (limit - cut.above_mass + each - 1) / each : limit - cut.above_count;
        sum = cut.above_mass + ties * each;
      }
      by_share = false;
      target = ties - 1;
    } else {
      target = set.point(sum);
    }
    if (round == 1 || ties < cut.equal) {
      const int j = find_in_order<T, NT>(row, part_of, target, s.select.red, 0, row.Q);
      if (round == 0) last = j;
      else if (tid == 0) a.answer(r, j, log_share(weigh, no_nan(row.at(j)), sum), (int)count);
    }
  }
}

template <class T, int NT>
__global__ __launch_bounds__(NT) void sample_rows(Sample a) {
  __shared__ GeneralLds<NT> s;
  const int64_t r = blockIdx.x;
  sample_general<T, NT>(a, r, Row<T>(a.logits, r, a.ld, a.C), RowSettings(a.set, r, a.C), s);
}

// ------------------------------------------------------------------ rows in registers

constexpr int kBins = 1024;
constexpr float kBinsPer = (kBins - 1) / kFaintest;  // bins of equal width in t
// Lanes of each wave that the bound is taken from, at most: with n of 64 lanes -64 log(1 - n/64) of its values reach it.
template <int NT>
constexpr int kNthMost = NT == kWave ? 56 : 24;

template <int NT, int NV>
struct TileLds {
  static constexpr int kList = NT == kWave ? 256 : NT == 256 ? 512 : 1024;
  static constexpr int kChunks = NV * NT / kWave;
  union {
    GeneralLds<NT> general;
    uint64_t mass[kBins];
    struct {
      uint64_t list[kList];  // key (inverted) and class: in the order when ascending
      uint64_t before[kList];
      uint32_t weight[kList], rank[kList];
    };
  };
  uint64_t chunk[kChunks];
  uint64_t red[NT / kWave];
  uint64_t above;
  float fred[NT / kWave];
  uint32_t ured[NT / kWave];
  int ired[NT / kWave];
  uint32_t n_list, part;
};

// 0, which the compiler does not know.
__device__ __forceinline__ int opaque_zero() {
  int v = 0;
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
  return v;
}

__device__ __forceinline__ uint64_t entry(uint32_t key, int j) { return (uint64_t)~key << 32 | (uint32_t)j; }
__device__ __forceinline__ float logit_of(uint64_t e) { return of_key(~(uint32_t)(e >> 32)); }

// Draws from the n collected elements, which hold all that can be kept. sum: the weight that top-p is a part of; 0:
// that of the first k elements. Each element is compared with all others by several threads, a share of them each.
template <class T, int NT, int NV>
__device__ __forceinline__ void draw_from_list(const Sample& a, int64_t r, const RowSettings& set, const Weigh& weigh,
                                               int n, uint64_t sum, TileLds<NT, NV>& s) {
  constexpr int kList = TileLds<NT, NV>::kList;
  const int tid = threadIdx.x;
  int width = kWave;  // entries side by side
  while (width < n && width < NT) width <<= 1;
  const int each = (n + NT / width - 1) / (NT / width);  // others of a thread
  const int from = tid / width * each, to = min(n, from + each);
  for (int e = tid; e < n; e += NT) {
    s.weight[e] = weigh(logit_of(s.list[e]));
    s.rank[e] = 0;
    s.before[e] = 0;
  }
  __syncthreads();
  for (int e = tid % width; e < n; e += width) {
    const uint64_t mine = s.list[e];
    uint64_t b = 0;
    uint32_t rank = 0;
#pragma unroll 4
    for (int o = from; o < to; ++o) {
      const bool ahead = s.list[o] < mine;
      rank += ahead;
      b += ahead ? s.weight[o] : 0;
    }
    if (rank) {
      atomicAdd(&s.rank[e], rank);
      atomicAdd((unsigned long long*)&s.before[e], (unsigned long long)b);
    }
  }
  __syncthreads();
  if (sum == 0) {
    for (int e = tid; e < n; e += NT) sum += s.rank[e] < (uint32_t)set.k ? s.weight[e] : 0;
    sum = block_sum64<NT>(sum, s.red);
  }
  const uint64_t limit = set.limit(sum);
  uint64_t total = 0;  // and the number kept, above bit 48
  for (int e = tid; e < n; e += NT) {
    const bool in = (s.rank[e] < (uint32_t)set.k) & (s.before[e] < limit) & (weigh.e(logit_of(s.list[e])) >= set.min_p);
    const uint32_t w = in ? s.weight[e] : 0;
    s.weight[e] = w;
    total += w + ((uint64_t)(w != 0) << 48);
  }
  static_assert(kList < (1 << 15), "sums of 2^31 each stay below bit 48");
  total = block_sum64<NT>(total, s.red);
  const int count = (int)(total >> 48);
  total &= ((uint64_t)1 << 48) - 1;
  const uint64_t point = set.point(total);
  for (int e = tid; e < n; e += NT) s.before[e] = 0;
  __syncthreads();
  for (int e = tid % width; e < n; e += width) {
    const uint32_t j = (uint32_t)s.list[e];
    uint64_t b = 0;
#pragma unroll 4
    for (int o = from; o < to; ++o) b += (uint32_t)s.list[o] < j ? s.weight[o] : 0;
    if (b) atomicAdd((unsigned long long*)&s.before[e], (unsigned long long)b);
  }
  __syncthreads();
  for (int e = tid; e < n; e += NT) {
    const uint32_t w = s.weight[e];
    const uint64_t b = s.before[e];
    if (w && b <= point && point < b + w)
      a.answer(r, (int)(uint32_t)s.list[e], log_share(weigh, logit_of(s.list[e]), total), count);
  }
}

// False where the row takes the general way.
template <class T, int NT, int NV>
__device__ __forceinline__ bool sample_in_registers(const Sample& a, int64_t r, const Row<T>& row,
                                                    const RowSettings& set, TileLds<NT, NV>& s) {
  constexpr int kVec = Row<T>::kVec;
  constexpr int kWaves = NT / kWave;
  constexpr int kList = TileLds<NT, NV>::kList;
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  Tile<T, NT, NV> tile;
  tile.load(row);
  // the largest value and a bound that at least `want` values reach
  const bool few = set.k <= kNthMost<NT> * kWaves;  // what top-k keeps can be collected
  const int nth = few ? (set.k + kWaves - 1) / kWaves : max(4, 16 / kWaves);
  float most = -INFINITY;
  bool nan = false;
  tile.each_unrolled(row, [&](const float (&x)[kVec], int, int) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      most = fmaxf(most, x[i]);
      nan |= x[i] != x[i];
    }
  });
  const uint32_t own = nan ? 0u : key_of(most);  // 0 is no value's key
  uint32_t high = wave_max_u32(own);
  uint32_t bound = wave_nth(own, nth);
  bool odd = __ballot(nan) != 0;
  if (tid == 0) s.n_list = 0;
  if (NT > kWave) {
    if (lane == 0) {
      s.ured[wave] = odd ? 0u : bound;
      s.fred[wave] = of_key(high);
    }
    __syncthreads();
    float m = s.fred[0];
    bound = s.ured[0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) {
      bound = min(bound, s.ured[k]);
      m = fmaxf(m, s.fred[k]);
    }
    odd = bound == 0;
    high = key_of(m);
  }
  __syncthreads();
  const float m = of_key(high);
  const Weigh weigh{m, 1.0f / set.temperature};
  if (odd || isinf(m) || (!few && set.k < a.C) || (isinf(weigh.inv) && set.k != 1)) return false;
  if (set.k == 1) {  // the first of the largest
    int at = INT32_MAX;
    tile.each(row, [&](const float (&x)[kVec], int q, int) {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (x[i] == m) at = min(at, row.first(q) + i);
    });
    at = block_reduce<NT>(at, [](int x, int y) { return min(x, y); }, s.ired);
    if (tid == 0) a.answer(r, at, 0.0f, 1);
    return true;
  }
  const float least = of_key(bound);
  int last = a.C;  // class of the last kept element at the cut
  const auto bin_of = [&](float t) { return min(kBins - 1, (int)(t * -kBinsPer)); };
  // One loop over the row for all passes: the exponential's code is there once.
  //   kCollect  the elements that reach the bound (all that top-k keeps)
  //   kSum      the same, and the sum of all weights: perhaps the elements reach top-p of it
  //   kBin      else the weights by t
  //   kPart     and the elements of the part with the cut
  //   kShare    the kept weights of runs of 64 vectors, which follow one another in the order of the classes
  enum { kCollect, kSum, kBin, kPart, kShare };
  int mode = few ? kCollect : set.top_p < 1.0f ? kSum : kShare;
  uint64_t sum = 0, limit = 0, above = 0;
  uint32_t count = 0;
  float cut = -INFINITY;
  int part = 0, n = 0;
  for (;;) {
    count = 0;
    uint64_t own_sum = 0;
    tile.each(row, [&](const float (&x)[kVec], int q, int) {
      // hidden from the compiler, which would make a loop of its own for every mode
      const int mode_here = __builtin_amdgcn_readfirstlane(mode + opaque_zero());
      uint32_t take = 0;
      if (mode_here == kCollect) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) take |= (uint32_t)((x[i] >= least) & (x[i] > -INFINITY)) << i;
      } else {
        float e[kVec];
        uint32_t w[kVec];
        uint64_t v = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          e[i] = exp_down(weigh.plain_t(x[i]));
          w[i] = (uint32_t)rintf(e[i] * kUnit);
        }
        if (mode_here == kShare) {
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            const bool in = ((x[i] > cut) | ((x[i] == cut) & (row.first(q) + i <= last))) & (e[i] >= set.min_p);
            w[i] = in ? w[i] : 0;
            v += w[i];
            count += w[i] != 0;
          }
          v = wave_sum64(v);
          if (lane == 0) s.chunk[q / kWave] = v;
        } else if (mode_here == kBin) {
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (w[i]) atomicAdd((unsigned long long*)&s.mass[bin_of(weigh.plain_t(x[i]))], (unsigned long long)w[i]);
        } else if (mode_here == kSum) {
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            v += w[i];
            take |= (uint32_t)((x[i] >= least) & (x[i] > -INFINITY)) << i;
          }
          own_sum += v;
        } else {
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            take |= (uint32_t)((w[i] != 0) & (bin_of(weigh.plain_t(x[i])) == part)) << i;
        }
      }
      if (take) {
        uint32_t at = atomicAdd(&s.n_list, (uint32_t)__popc(take));
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          if ((take >> i & 1) && at < (uint32_t)kList) s.list[at] = entry(key_of(x[i]), row.first(q) + i);
          at += take >> i & 1;
        }
      }
    });
    if (mode == kShare) break;
    __syncthreads();
    n = (int)s.n_list;
    if (mode == kCollect || mode == kPart) {
      if (n > kList) return false;
    }
    bool draw = mode == kCollect;
    if (mode == kSum) {
      sum = block_sum64<NT>(own_sum, s.red);
      limit = set.limit(sum);
      if (n <= kList) {
        uint64_t listed = 0;
        for (int e = tid; e < n; e += NT) listed += weigh(logit_of(s.list[e]));
        draw = block_sum64<NT>(listed, s.red) >= limit;
      }
    }
    if (draw) {
      __syncthreads();
      draw_from_list<T, NT, NV>(a, r, set, weigh, n, sum, s);
      return true;
    }
    if (mode == kSum) {
      __syncthreads();
      for (int b = tid; b < kBins; b += NT) s.mass[b] = 0;
      if (tid == 0) s.n_list = 0;
      __syncthreads();
      mode = kBin;
    } else if (mode == kBin) {
      constexpr int kEach = kBins / NT;
      uint64_t b = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) b += s.mass[tid * kEach + i];
      b = block_exclusive<NT>(b, s.red);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const uint64_t w = s.mass[tid * kEach + i];
        if (b < limit && b + w >= limit) {
          s.part = tid * kEach + i;
          s.above = b;
        }
        b += w;
      }
      __syncthreads();
      part = (int)s.part;
      above = s.above;
      mode = kPart;
    } else {
      for (int e = tid; e < n; e += NT) s.weight[e] = weigh(logit_of(s.list[e]));
      __syncthreads();
      for (int e = tid; e < n; e += NT) {
        const uint64_t mine = s.list[e];
        uint64_t before = above;
#pragma unroll 4
        for (int o = 0; o < n; ++o) before += s.list[o] < mine ? s.weight[o] : 0;
        if (before < limit && before + s.weight[e] >= limit) {  // the last kept
          s.ured[0] = ~(uint32_t)(mine >> 32);  // (a key of 0's either sign stands for both)
          s.ired[0] = (int)(uint32_t)mine;
        }
      }
      __syncthreads();
      cut = of_key(s.ured[0]);
      last = s.ired[0];
      mode = kShare;
    }
  }
  const int runs = (row.Q + NT - 1) / NT * kWaves;
  for (int c = runs + tid; c < TileLds<NT, NV>::kChunks; c += NT) s.chunk[c] = 0;
  const uint64_t counted = block_sum64<NT>(count, s.red);
  __syncthreads();
  // every wave for itself: the run of the point
  constexpr int kChunks = TileLds<NT, NV>::kChunks;
  constexpr int kOwn = (kChunks + kWave - 1) / kWave;
  uint64_t v = 0;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) v += lane * kOwn + i < kChunks ? s.chunk[lane * kOwn + i] : 0;
  const uint64_t upto = wave_upto64(v), total = lane_of64(upto, kWave - 1);
  const uint64_t point = set.point(total);
  const int at = (int)__builtin_ctzll(__ballot(upto > point));
  uint64_t target = point - lane_of64(upto - v, at);
  int run = at * kOwn;
#pragma unroll
  for (int i = 0; i < kOwn - 1; ++i) {
    const uint64_t w = s.chunk[run];
    if (target >= w) {
      target -= w;
      ++run;
    }
  }
  if (wave != 0) return true;
  const auto share = [&](float x, int j) -> uint64_t {
    const float e = weigh.e(x);
    return ((x > cut) | ((x == cut) & (j <= last))) & (e >= set.min_p) ? weigh.of(x, e) : 0;
  };
  const int j = find_in_order<T, kWave>(row, share, target, nullptr, run * kWave, min(row.Q, (run + 1) * kWave));
  if (lane == 0) a.answer(r, j, log_share(weigh, row.at(j), total), (int)counted);
  return true;
}

template <class T, int NT, int NV>
__global__ __launch_bounds__(NT) void sample_tile(Sample a) {
  __shared__ TileLds<NT, NV> s;
  const int64_t r = blockIdx.x;
  const Row<T> row(a.logits, r, a.ld, a.C);
  const RowSettings set(a.set, r, a.C);
  if (!sample_in_registers<T, NT, NV>(a, r, row, set, s)) sample_general<T, NT>(a, r, row, set, s.general);
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
  const Sample a{logits, R, C, ld, Settings{u, temperature, top_k, top_p, min_p}, cls, logp, kept};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)R);
  return rows::for_type(dtype, [&](auto type) {
    using T = decltype(type);
    const int Q = rows::most_vectors<T>(logits, C, ld);
    if (C <= rows::kShortRow)
      hipLaunchKernelGGL((sample_short<T>), dim3((unsigned)((R + rows::kShortRows - 1) / rows::kShortRows)), dim3(256),
                         0, s, a);
    else if (Q <= 4 * 64)
      hipLaunchKernelGGL((sample_tile<T, 64, 4>), grid, dim3(64), 0, s, a);
    else if (Q <= 4 * 256)
      hipLaunchKernelGGL((sample_tile<T, 256, 4>), grid, dim3(256), 0, s, a);
    else if (Q <= 4 * 1024)
      hipLaunchKernelGGL((sample_tile<T, 1024, 4>), grid, dim3(1024), 0, s, a);
    else if (Q <= 16 * 1024)
      hipLaunchKernelGGL((sample_tile<T, 1024, 16>), grid, dim3(1024), 0, s, a);
    else
      hipLaunchKernelGGL((sample_rows<T, 1024>), grid, dim3(1024), 0, s, a);
    return launch_status();
  });
}
