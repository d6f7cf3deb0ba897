// One class per row drawn from its logits with temperature, top-k, top-p and min-p, from a given uniform number.
//   t_j = (z_j - max z) / temperature, e_j = exp(t_j), weight n_j = round(2^31 e_j)
//   kept: of the order by value (ties by class) the first top_k, of these the shortest prefix with a weight of at
//   least top_p of theirs, of these the classes with e_j >= min_p
//   drawn: the first class whose kept weights up to it, in the order of the classes, exceed floor(u * their sum)
// The weights are whole numbers, so every sum is exact and the answer does not depend on how it was summed.
//
// A row is held in registers. What top-k keeps is collected by the waves' n-th largest lanes, as a teacher's record is;
// what top-p keeps is either among those or found by a histogram of t and an order within one of its bins; without
// either filter the weights are summed in runs along the row and the drawn class is sought in one run.
//   sample_short   16 lanes a row of up to 128 classes; few of more than 48 with an order take a wave each
//   sample_tile    a block a row, in registers; one wave up to 2048 classes, whose cuts cut_in_wave finds
//   split_*        a row's parts in blocks of their own: few long rows, rows beyond the registers
//   sample_rows    a block a row, read several times: the rest
//
// Measured: 1024 x 65536 float32 with a temperature: 135 us (2.0 TB/s), vector instructions (exponentials, the filters'
// comparisons, 64-bit sums) issued 62% of the time with one block a compute unit; 64 x 128011 bfloat16, mixed settings, in
// parts: 63 us, and 1 x 32003 float32 with top-k 50: 19 us, waves waiting about 60% of the time; 23265 x 590 bfloat16,
// mixed settings: 117 us, some 15 to 30 comparisons a value; 25600 x 20 float32, mixed settings: 14.3 us.
#include <cfloat>

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
    k = set.top_k ? set.top_k[r] : 0;
    if (k <= 0 || k > C) k = C;
    if (!(temperature > 0.0f)) k = 1;
    top_p = set.top_p ? set.top_p[r] : 1.0f;
    top_p = top_p > 0.0f ? fminf(top_p, 1.0f) : 0.0f;
    min_p = set.min_p ? set.min_p[r] : 0.0f;
    min_p = min_p > 0.0f ? fminf(min_p, 1.0f) : 0.0f;
  }
  // For a kernel whose waves have one row each.
  __device__ __forceinline__ RowSettings of_wave() const {
    RowSettings s = *this;
    s.u = same_in_wave(u);
    s.temperature = same_in_wave(temperature);
    s.top_p = same_in_wave(top_p);
    s.min_p = same_in_wave(min_p);
    s.k = same_in_wave(k);
    return s;
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
#pragma unroll 4
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
  sample_general<T, NT>(a, r, Row<T>(a.logits, r, a.ld, a.C), RowSettings(a.set, r, a.C).of_wave(), s);
}

// ------------------------------------------------------------------ rows in registers

constexpr int kBins = 1024;
constexpr float kBinsPer = (kBins - 1) / kFaintest;  // bins of equal width in t
__device__ __forceinline__ int bin_of(float t) { return min(kBins - 1, (int)(t * -kBinsPer)); }

// Lanes of each wave that the bound is taken from, at most: with n of 64 lanes -64 log(1 - n/64) of its values reach it.
template <int NT>
constexpr int kNthMost = NT == 256 ? 50 : 32;

template <int NT, int NV>
struct TileLds {
  static constexpr int kList = NT == kWave ? 1 : 1024;  // one wave finds the cut without a list
  static constexpr int kChunks = NV * NT / kWave;
  union {
    GeneralLds<NT> general;
    uint64_t mass[NT == kWave ? 1 : kBins];
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

// How the threads share the comparisons of n elements with one another: a thread takes every width-th element from
// its own on, and the others [from, to) to compare them with.
template <int NT>
struct Pairs {
  int width, from, to;
  __device__ __forceinline__ explicit Pairs(int n) {
    width = kWave;
    while (width < n && width < NT) width <<= 1;
    const int each = (n + NT / width - 1) / (NT / width);
    from = (int)threadIdx.x / width * each;
    to = min(n, from + each);
  }
};

// Beyond this many elements two sorts take less than all comparisons (1000 elements in 1024 threads: 50 us of comparisons).
constexpr int kSorted = 256;

// before[e] = sum of value(o) over o < e, for e < n.
template <int NT, class F>
__device__ __forceinline__ void block_before(int n, F value, uint64_t* before, uint64_t* red) {
  uint64_t base = 0;
  for (int e0 = 0; e0 < n; e0 += NT) {
    const int e = e0 + (int)threadIdx.x;
    const uint64_t w = e < n ? value(e) : 0;
    const uint64_t b = base + block_exclusive<NT>(w, red);
    if (e < n) before[e] = b;
    base += block_sum64<NT>(w, red);
  }
  __syncthreads();
}

// Weights of the n collected elements, and of each how many are ahead of it and what they weigh. Long lists are put in
// order.
template <int NT, class Lds>
__device__ __forceinline__ void order_list(const Weigh& weigh, int n, Lds& s) {
  const int tid = threadIdx.x;
  if (n > kSorted) block_sort<NT>(s.list, n);
  for (int e = tid; e < n; e += NT) {
    s.weight[e] = weigh(logit_of(s.list[e]));
    s.rank[e] = n > kSorted ? e : 0;
    s.before[e] = 0;
  }
  __syncthreads();
  if (n > kSorted) return block_before<NT>(n, [&](int e) { return (uint64_t)s.weight[e]; }, s.before, s.red);
  const Pairs<NT> by(n);
  for (int e = tid % by.width; e < n; e += by.width) {
    const uint64_t mine = s.list[e];
    uint64_t b = 0;
    uint32_t rank = 0;
#pragma unroll 4
    for (int o = by.from; o < by.to; ++o) {
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
}

// The cut of a row in one wave's registers: what is larger than `cut` is kept, and of what equals it the classes up to
// `last`. Top-k's is found by first_in_wave, top-p's in the same manner with the weights' sum beside the count.
template <class T, int NV>
__device__ __forceinline__ void cut_in_wave(const Tile<T, kWave, NV>& tile, const Row<T>& row, const RowSettings& set,
                                            const Weigh& weigh, int C, float& cut, int& last) {
  constexpr int kVec = Row<T>::kVec;
  struct Reach {
    int count;
    uint64_t mass;
  };
  uint32_t w[NV * kVec];
  if (set.top_p < 1.0f) {
#pragma unroll
    for (int i = 0; i < NV * kVec; ++i) w[i] = 0;
    tile.each_unrolled(row, [&](const float (&x)[kVec], int, int n) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) w[n * kVec + i] = (uint32_t)rintf(exp_down(weigh.plain_t(x[i])) * kUnit);
    });
  }
  // elements for which in(value, class), and their weight
  const auto reach_of = [&](auto in) {
    Reach v{0, 0};
    tile.each_unrolled(row, [&](const float (&x)[kVec], int q, int n) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const bool yes = in(x[i], row.first(q) + i);
        v.count += __popcll(__ballot(yes));
        v.mass += yes ? w[n * kVec + i] : 0;
      }
    });
    v.mass = wave_sum64(v.mass);
    return v;
  };
  // 24 temperatures below the largest no weight is left (and -inf has none)
  uint32_t lo = short_key<T>(fmaxf(weigh.max - 24.0f * set.temperature, -FLT_MAX));
  const uint32_t top = short_key<T>(weigh.max) + 1;
  lo = (uint32_t)same_in_wave((int)lo);
  cut = least_of<T>(lo);
  last = C;
  int n_lo = C;  // elements from lo on, of those below `top`; C for unknown
  if (set.k < C) {
    n_lo = count_in_wave(tile, row, [&](float x, int) { return x >= cut; });
    if (n_lo > set.k) first_in_wave(tile, row, C, set.k, lo, top, n_lo, cut, last);
  }
  if (set.top_p < 1.0f) {
    const uint64_t limit =
        set.limit(reach_of([&](float x, int j) { return (x > cut) | ((x == cut) & (j <= last)); }).mass);
    uint32_t hi = top;
    Reach above{0, 0};
    for (int step = 0; hi - lo > 1 && n_lo - above.count > 1; ++step) {
      const uint32_t mid = halfway<T>(lo, hi, step);
      const float least = least_of<T>(mid);
      const Reach v = reach_of([&](float x, int) { return x >= least; });
      if (v.mass >= limit) {
        lo = mid;
        n_lo = v.count;
      } else {
        hi = mid;
        above = v;
      }
    }
    if (n_lo - above.count == 1) {
      cut = least_of<T>(lo);
      last = C;
    } else {
      cut = value_of<T>(lo);
      last = first_class(C, [&](int c) {
        return above.mass + reach_of([&](float x, int j) { return (x == cut) & (j <= c); }).mass >= limit;
      });
    }
  }
}

// Draws from the n collected elements, which hold all that can be kept. sum: the weight that top-p is a part of; 0:
// that of the first k elements.
template <class T, int NT, int NV>
__device__ __forceinline__ void draw_from_list(const Sample& a, int64_t r, const Row<T>& row, const RowSettings& set,
                                               const Weigh& weigh, int n, uint64_t sum, TileLds<NT, NV>& s) {
  constexpr int kList = TileLds<NT, NV>::kList;
  const int tid = threadIdx.x;
  order_list<NT>(weigh, n, s);
  const Pairs<NT> by(n);
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
  // the same in the order of the classes, with the kept weights
  for (int e = tid; e < n; e += NT) {
    if (n > kSorted) s.list[e] = s.list[e] << 32 | s.weight[e];
    s.before[e] = 0;
  }
  __syncthreads();
  if (n > kSorted) {
    block_sort<NT>(s.list, n);
    block_before<NT>(n, [&](int e) { return (uint64_t)(uint32_t)s.list[e]; }, s.before, s.red);
  } else {
    for (int e = tid % by.width; e < n; e += by.width) {
      const uint32_t j = (uint32_t)s.list[e];
      uint64_t b = 0;
#pragma unroll 4
      for (int o = by.from; o < by.to; ++o) b += (uint32_t)s.list[o] < j ? s.weight[o] : 0;
      if (b) atomicAdd((unsigned long long*)&s.before[e], (unsigned long long)b);
    }
    __syncthreads();
  }
  for (int e = tid; e < n; e += NT) {
    const uint32_t w = n > kSorted ? (uint32_t)s.list[e] : s.weight[e];
    const int j = (int)(uint32_t)(n > kSorted ? s.list[e] >> 32 : s.list[e]);
    const uint64_t b = s.before[e];
    if (w && b <= point && point < b + w) a.answer(r, j, log_share(weigh, row.at(j), total), count);
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
  const int full = max(1, min(kWaves, row.Q / kWave));  // waves without idle lanes give the bound
  const bool few = set.k <= kNthMost<NT> * full;  // what top-k keeps can be collected
  const int nth = few ? (set.k + full - 1) / full : max(4, 16 / full);
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
  uint32_t bound = NT > kWave && wave < full ? wave_nth(own, nth) : UINT32_MAX;
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
  odd = same_in_wave(odd);
  const float m = same_in_wave(of_key(high));
  const Weigh weigh{m, 1.0f / set.temperature};
  if (odd || isinf(m) || (NT > kWave && !few && set.k < a.C) || (isinf(weigh.inv) && set.k != 1)) return false;
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
  const float least = same_in_wave(of_key(bound));
  int last = a.C;  // class of the last kept element at the cut
  // One loop over the row for all passes: the exponential's code is there once.
  //   kCollect  the elements that reach the bound (all that top-k keeps)
  //   kSum      the same, and the sum of all weights: perhaps the elements reach top-p of it
  //   kBin      else the weights by t
  //   kPart     and the elements of the part with the cut
  //   kShare    the kept weights of runs of 64 vectors, which follow one another in the order of the classes
  enum { kCollect, kSum, kBin, kPart, kShare };
  int mode = NT == kWave ? kShare : few ? kCollect : set.top_p < 1.0f ? kSum : kShare;
  uint64_t sum = 0, limit = 0, above = 0;
  uint32_t count = 0;
  float cut = -INFINITY;
  int part = 0, n = 0;
  if constexpr (NT == kWave) {
    if (set.k < a.C || set.top_p < 1.0f) cut_in_wave<T, NV>(tile, row, set, weigh, a.C, cut, last);
  }
  for (;;) {
    count = 0;
    uint64_t own_sum = 0;
    tile.each(row, [&](const float (&x)[kVec], int q, int) {
      // hidden from the compiler, which would make a loop of its own for every mode
      const int mode_here = NT == kWave ? kShare : __builtin_amdgcn_readfirstlane(mode + opaque_zero());
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
    if (NT == kWave || mode == kShare) break;
    __syncthreads();
    n = same_in_wave((int)s.n_list);
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
      draw_from_list<T, NT, NV>(a, r, row, set, weigh, n, sum, s);
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
      part = same_in_wave((int)s.part);
      above = s.above;
      mode = kPart;
    } else {
      order_list<NT>(weigh, n, s);
      for (int e = tid; e < n; e += NT) {
        const uint64_t mine = s.list[e], before = above + s.before[e];
        if (before < limit && before + s.weight[e] >= limit) {  // the last kept
          s.ured[0] = ~(uint32_t)(mine >> 32);  // (a key of 0's either sign stands for both)
          s.ired[0] = (int)(uint32_t)mine;
        }
      }
      __syncthreads();
      cut = same_in_wave(of_key(s.ured[0]));
      last = same_in_wave(s.ired[0]);
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
  const RowSettings set = RowSettings(a.set, r, a.C).of_wave();
  if (!sample_in_registers<T, NT, NV>(a, r, row, set, s)) sample_general<T, NT>(a, r, row, set, s.general);
}

// ------------------------------------------------------------------ few long rows, several blocks each

// A row of many vectors is shared among blocks of 256 threads, up to four vectors a thread:
//   split_max    every part's largest logit and the bound of its waves
//   split_sum    what top-k keeps, collected by the row's bound; else the weights by t for top-p
//   split_cut    (a block a row) the bin of the top-p cut
//   split_share  the kept weights of every part; the elements of that bin, collected
//   split_draw   (a block a row) the order of what was collected, the part of the point, the class
// The launches read the row again, from the caches. Each part has its own place for what it finds: atomics of blocks on
// several dies go to memory, one after another (64 rows of 128011 with top-k 50: 229 us with a common list, 37 so).
constexpr int kPartThreads = 256;
constexpr int kPartVectors = 4 * kPartThreads;
constexpr int kMostParts = 64;
constexpr int kRowList = 1024;
constexpr int kPartList = 256;
constexpr int kPool = 256;         // a row's largest of lanes, which its bound is one of

// The bin of the top-p cut, the weight above it and the limit.
struct CutBin {
  uint64_t above, limit;
  int bin;
};

struct Split {
  int parts;
  int each;          // vectors of a part
  float* max;        // [R][parts]
  int* arg;          // [R][parts] first class of it
  uint32_t* pool;    // [R][kPool], pool_used of them
  int of_wave;       // lanes' largest that a wave gives
  uint64_t* share;   // [R][parts] kept weights
  uint32_t* count;   // [R][parts] kept classes
  uint64_t* mass;    // [R][parts][kBins]
  uint64_t* list;    // [R][parts][kPartList]
  uint32_t* n_list;  // [R][parts], also what did not fit
  CutBin* cut;       // [R]

  __host__ __device__ int pooled() const { return parts * (kPartThreads / kWave) * of_wave; }
  static size_t carve(void* ws, int64_t R, int parts, Split* s) {
    Carve c(ws);
    Split t{};
    t.parts = parts;
    t.max = c.take<float>((size_t)R * parts);
    t.arg = c.take<int>((size_t)R * parts);
    t.pool = c.take<uint32_t>((size_t)R * kPool);
    t.of_wave = std::min(8, kPool / (parts * (kPartThreads / kWave)));
    t.share = c.take<uint64_t>((size_t)R * parts);
    t.count = c.take<uint32_t>((size_t)R * parts);
    t.mass = c.take<uint64_t>((size_t)R * parts * kBins);
    t.list = c.take<uint64_t>((size_t)R * parts * kPartList);
    t.n_list = c.take<uint32_t>((size_t)R * parts);
    t.cut = c.take<CutBin>((size_t)R);
    if (s) *s = t;
    return c.off;
  }
};

// Parts that a row is shared among: from the length on where several launches take less than one block, where the rows
// alone leave most compute units idle or do not fit a block's registers. In a block and in parts, kernels alone: by
// requests 64 x 40000 float32 54 and 43 us, 64 x 130000 bfloat16 133 and 61; with top-k 50 1 x 40000 float32 17 and 22,
// 1 x 130000 bfloat16 31 and 23. Beyond the registers, in passes and in parts: 64 x 131072 float32 with top-k 50 320 and
// 34, by requests, some with a top-k that is not collected, 345 and 383; 1000 x 131072 1390 and 286, 1314 and 688. A part
// has 10 KB of workspace: at most 320 MB.
inline int split_parts(int64_t R, int C, int dtype) {
  const int per = 16 / rows::type_size(dtype);
  const int Q = (C + 2 * per - 2) / per;  // as of a row that is not aligned
  const int parts = (Q + kPartVectors - 1) / kPartVectors;
  if (Q <= 8192 || parts > kMostParts) return 1;
  return R <= (Q <= 16 * 1024 ? cu_count() / 2 : (1 << 15) / parts) ? parts : 1;
}

// What the launches after the first know of a row.
struct SplitRow {
  float max;
  bool listed, cut;  // top-k is collected; a top-p cut is looked for
  bool general;      // neither: a longer top-k, or nothing but -inf
  __device__ __forceinline__ SplitRow(const Sample& a, const Split& s, int64_t r, const RowSettings& set) {
    const int l = threadIdx.x % kWave;
    const float m = l < s.parts ? s.max[r * s.parts + l] : -INFINITY;
    max = wave_reduce(m, Larger());
    listed = set.k <= s.pooled() - s.pooled() / 8;  // collected by the bound
    cut = set.k == a.C && set.top_p < 1.0f && !listed;
    general = max == -INFINITY || (!listed && set.k < a.C);
  }
};

template <class T>
__global__ __launch_bounds__(kPartThreads) void split_max(Sample a, Split s) {
  constexpr int kVec = Row<T>::kVec;
  constexpr int kWaves = kPartThreads / kWave;
  __shared__ float fred[kWaves];
  __shared__ int ired[kWaves];
  const int64_t r = blockIdx.x / s.parts;
  const int p = blockIdx.x % s.parts, tid = threadIdx.x;
  const Row<T> row(a.logits, r, a.ld, a.C);
  const RowSettings set = RowSettings(a.set, r, a.C).of_wave();
  const int q0 = p * s.each;
  uint4 u[4];
  load_vectors<T, kPartThreads>(row, u, q0, min(row.Q, q0 + s.each));
  if (tid == 0) s.n_list[r * s.parts + p] = 0;
  float m = -INFINITY;
  int at = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[kVec];
    unpack<T>(u[i], x);
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const bool up = x[k] > m;  // never for NaN
      m = up ? x[k] : m;
      at = up ? row.first(q0 + i * kPartThreads + tid) + k : at;
    }
  }
  uint32_t key = key_of(m);
  for (int k = 0; k < s.of_wave; ++k) {  // the wave's largest lanes, one after another
    const uint32_t v = wave_max_u32(key);
    if (lane_id() == (int)__builtin_ctzll(__ballot(key == v))) {
      key = 0;
      s.pool[r * kPool + (p * kWaves + tid / kWave) * s.of_wave + k] = v;
    }
  }
  const float most = wave_reduce(m, Larger());
  int first = m == most ? at : INT32_MAX;
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) first = min(first, __shfl_xor(first, off, kWave));
  if (tid % kWave == 0) {
    fred[tid / kWave] = most;
    ired[tid / kWave] = first;
  }
  __syncthreads();
  if (tid != 0) return;
  float all = fred[0];
  for (int k = 1; k < kWaves; ++k) all = fmaxf(all, fred[k]);
  first = INT32_MAX;
  for (int k = 0; k < kWaves; ++k) first = fred[k] == all ? min(first, ired[k]) : first;
  s.max[r * s.parts + p] = all;
  s.arg[r * s.parts + p] = first;
}

// A part's list, put together in LDS.
struct PartList {
  uint64_t entry_[kPartList];
  uint32_t n;
  __device__ __forceinline__ void add(float x, int j) {
    const uint32_t at = atomicAdd(&n, 1u);
    if (at < (uint32_t)kPartList) entry_[at] = entry(key_of(x), j);
  }
  __device__ __forceinline__ void put(const Split& s, int64_t part) const {  // after a barrier
    for (uint32_t e = threadIdx.x; e < min(n, (uint32_t)kPartList); e += kPartThreads)
      s.list[part * kPartList + e] = entry_[e];
    if (threadIdx.x == 0) s.n_list[part] = n;
  }
};

template <class T>
__global__ __launch_bounds__(kPartThreads) void split_sum(Sample a, Split s) {
  constexpr int kVec = Row<T>::kVec;
  __shared__ uint64_t mass[kBins];
  __shared__ PartList list;
  __shared__ uint32_t pool[kPool], bound;
  const int64_t r = blockIdx.x / s.parts;
  const int p = blockIdx.x % s.parts, tid = threadIdx.x;
  const RowSettings set = RowSettings(a.set, r, a.C).of_wave();
  const SplitRow known(a, s, r, set);
  if (set.k == 1 || known.general || !(known.listed || known.cut)) return;
  const Row<T> row(a.logits, r, a.ld, a.C);
  const int q0 = p * s.each;
  Tile<T, kPartThreads, 4> tile;
  tile.load(row, q0, min(row.Q, q0 + s.each));
  if (known.cut)
    for (int b = tid; b < kBins; b += kPartThreads) mass[b] = 0;
  if (tid == 0) list.n = 0;
  const int pooled = s.pooled();
  const uint32_t mine = tid < pooled ? s.pool[r * kPool + tid] : 0;
  pool[tid] = mine;
  __syncthreads();
  if (known.listed && tid < pooled) {  // the k-th largest of the pool
    int above = 0, equal = 0;
#pragma unroll 8
    for (int o = 0; o < pooled; ++o) {
      above += pool[o] > mine;
      equal += pool[o] == mine;
    }
    if (above < set.k && above + equal >= set.k) bound = mine;
  }
  __syncthreads();
  const float least = of_key(bound);
  const Weigh weigh{known.max, 1.0f / set.temperature};
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    float x[kVec];
    unpack<T>(tile.get(i), x);
    const int j = row.first(q0 + i * kPartThreads + tid);
    if (known.listed) {
#pragma unroll
      for (int k = 0; k < kVec; ++k)
        if (x[k] >= least && x[k] > -INFINITY) list.add(x[k], j + k);
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const float y = no_nan(x[k]);
        const uint32_t w = weigh(y);
        if (w) atomicAdd((unsigned long long*)&mass[bin_of(weigh.t(y))], (unsigned long long)w);
      }
    }
  }
  __syncthreads();
  const int64_t part = r * s.parts + p;
  if (known.listed) list.put(s, part);
  else
    for (int b = tid; b < kBins; b += kPartThreads) s.mass[part * kBins + b] = mass[b];
}

template <class T>
__global__ __launch_bounds__(kBins) void split_cut(Sample a, Split s) {
  __shared__ uint64_t red[kBins / kWave];
  const int64_t r = blockIdx.x;
  const RowSettings set = RowSettings(a.set, r, a.C).of_wave();
  const SplitRow known(a, s, r, set);
  if (set.k == 1 || known.general || !known.cut) return;
  uint64_t w = 0;
#pragma unroll 8
  for (int p = 0; p < s.parts; ++p) w += s.mass[(r * s.parts + p) * kBins + threadIdx.x];
  const uint64_t limit = set.limit(block_sum64<kBins>(w, red));
  const uint64_t b = block_exclusive<kBins>(w, red);
  if (b < limit && b + w >= limit) s.cut[r] = CutBin{b, limit, (int)threadIdx.x};
}

template <class T>
__global__ __launch_bounds__(kPartThreads) void split_share(Sample a, Split s) {
  constexpr int kVec = Row<T>::kVec;
  __shared__ uint64_t red[kPartThreads / kWave];
  __shared__ PartList list;
  const int64_t r = blockIdx.x / s.parts;
  const int p = blockIdx.x % s.parts, tid = threadIdx.x;
  const RowSettings set = RowSettings(a.set, r, a.C).of_wave();
  const SplitRow known(a, s, r, set);
  if (set.k == 1 || known.general || known.listed) return;
  const Row<T> row(a.logits, r, a.ld, a.C);
  const int q0 = p * s.each;
  Tile<T, kPartThreads, 4> tile;
  tile.load(row, q0, min(row.Q, q0 + s.each));
  const int bin = known.cut ? s.cut[r].bin : kBins;
  if (tid == 0) list.n = 0;
  __syncthreads();
  const Weigh weigh{known.max, 1.0f / set.temperature};
  uint64_t sum = 0, count = 0;
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    float x[kVec];
    unpack<T>(tile.get(i), x);
    const int j = row.first(q0 + i * kPartThreads + tid);
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const float y = no_nan(x[k]), t = weigh.t(y), e = exp_down(t);
      const uint32_t w = weigh.of(y, e);
      const int b = w ? bin_of(t) : kBins + 1;
      if (b == bin) list.add(y, j + k);
      const bool in = (b < bin) & (e >= set.min_p);
      sum += in ? w : 0;
      count += in;
    }
  }
  sum = block_sum64<kPartThreads>(sum, red);
  count = block_sum64<kPartThreads>(count, red);
  if (tid == 0) {
    s.share[r * s.parts + p] = sum;
    s.count[r * s.parts + p] = (uint32_t)count;
  }
  list.put(s, r * s.parts + p);
}

constexpr int kDrawThreads = 1024;

template <class T>
__global__ __launch_bounds__(kDrawThreads) void split_draw(Sample a, Split s) {
  using Lds = TileLds<kDrawThreads, 4>;
  __shared__ Lds lds;
  __shared__ uint64_t share[kMostParts], last_kept;
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid % kWave;
  const Row<T> row(a.logits, r, a.ld, a.C);
  const RowSettings set = RowSettings(a.set, r, a.C).of_wave();
  const SplitRow known(a, s, r, set);
  // where each part's collected elements go in the row's list
  const uint32_t own = lane < s.parts ? s.n_list[r * s.parts + lane] : 0;
  const uint32_t upto_own = (uint32_t)wave_upto64(own);
  const uint32_t n = (uint32_t)__builtin_amdgcn_readlane((int)upto_own, kWave - 1);
  if (known.general || n > (uint32_t)kRowList || __ballot(own > (uint32_t)kPartList)) return sample_general<T, kDrawThreads>(a, r, row, set, lds.general);
  if (set.k == 1) {
    int at = lane < s.parts && s.max[r * s.parts + lane] == known.max ? s.arg[r * s.parts + lane] : INT32_MAX;
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) at = min(at, __shfl_xor(at, off, kWave));
    if (tid == 0) a.answer(r, at, 0.0f, 1);
    return;
  }
  const Weigh weigh{known.max, 1.0f / set.temperature};
  for (int p = tid / kWave; p < s.parts; p += kDrawThreads / kWave) {
    const uint32_t to = (uint32_t)__builtin_amdgcn_readlane((int)upto_own, p);
    const uint32_t m = (uint32_t)__builtin_amdgcn_readlane((int)own, p);
    for (uint32_t e = lane; e < m; e += kWave) lds.list[to - m + e] = s.list[(r * s.parts + p) * kPartList + e];
  }
  __syncthreads();
  if (known.listed) {
    return draw_from_list<T, kDrawThreads, 4>(a, r, row, set, weigh, (int)n, 0, lds);
  }
  // the parts' kept weights, with those of the cut's bin that are kept
  uint64_t counted = 0;
  if (tid < kMostParts) share[tid] = tid < s.parts ? s.share[r * s.parts + tid] : 0;
  if (tid < s.parts) counted = s.count[r * s.parts + tid];
  float cut = -INFINITY;
  int last = a.C;
  if (known.cut) {
    const CutBin at = s.cut[r];
    order_list<kDrawThreads>(weigh, (int)n, lds);
    if (tid < (int)n) {  // n <= kRowList = kDrawThreads
      const uint64_t mine = lds.list[tid], before = at.above + lds.before[tid];
      const uint32_t w = lds.weight[tid];
      if (before < at.limit) {
        if (before + w >= at.limit) last_kept = mine;
        if (weigh.e(logit_of(mine)) >= set.min_p) {
          atomicAdd((unsigned long long*)&share[((int)(uint32_t)mine + row.lead) / Row<T>::kVec / s.each],
                    (unsigned long long)w);
          ++counted;
        }
      }
    }
    __syncthreads();
    cut = logit_of(last_kept);
    last = (int)(uint32_t)last_kept;
  }
  counted = block_sum64<kDrawThreads>(counted, lds.red);
  __syncthreads();
  const uint64_t mine = share[lane], upto = wave_upto64(mine), total = lane_of64(upto, kWave - 1);
  const uint64_t point = set.point(total);
  const int p = (int)__builtin_ctzll(__ballot(upto > point));
  const auto kept = [&](float x, int j) -> uint64_t {
    const float e = weigh.e(x);
    return ((x > cut) | ((x == cut) & (j <= last))) & (e >= set.min_p) ? weigh.of(x, e) : 0;
  };
  const int j = find_in_order<T, kDrawThreads>(row, kept, point - lane_of64(upto - mine, p), lds.red, p * s.each,
                                               min(row.Q, (p + 1) * s.each));
  if (tid == 0) a.answer(r, j, log_share(weigh, no_nan(row.at(j)), total), (int)counted);
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" size_t snn_readout_sample_workspace(int64_t R, int C, int dtype) {
  if (R <= 0 || R > INT32_MAX || bad_dim(C) || C > rows::kMaxClasses || rows::type_size(dtype) == 0) return 0;
  const int parts = split_parts(R, C, dtype);
  return parts > 1 ? Split::carve(nullptr, R, parts, nullptr) : 0;
}

extern "C" snn_status snn_readout_sample(const void* logits, int dtype, int64_t R, int C, int64_t ld, const float* u,
                                         const float* temperature, const int32_t* top_k, const float* top_p,
                                         const float* min_p, int32_t* cls, float* logp, int32_t* kept, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  const snn_status ok = rows::check_rows(logits, dtype, R, C, ld);
  if (ok != SNN_OK) return ok;
  if (!u || !cls) return SNN_ERR_INVALID_ARG;
  const size_t need = snn_readout_sample_workspace(R, C, dtype);
  if (need && (!workspace || workspace_bytes < need)) return SNN_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return rows::for_type(dtype, [&](auto type) {
    using T = decltype(type);
    const int Q = rows::most_vectors<T>(logits, C, ld);
    return rows::in_launches(R, [&](int64_t first, int64_t n) {
      using rows::or_null;
      const Sample a{static_cast<const T*>(logits) + first * ld, n, C, ld,
                     Settings{u + first, or_null(temperature, first), or_null(top_k, first), or_null(top_p, first),
                              or_null(min_p, first)},
                     cls + first, or_null(logp, first), or_null(kept, first)};
      const dim3 grid((unsigned)n);
      // 16 lanes a row compare each value with all others where an order is asked for: few rows of many classes go a wave
      // each. By requests, float32, a wave each and so, kernels alone: 16 x 20 8 and 6 us, 2048 x 48 13 and 11, 2048 x 100 13
      // and 26, 20000 x 100 47 and 40, 20000 x 128 49 and 55 (bfloat16 with top-k 50 77 and 55); without an order 256 x 128
      // bfloat16 6 and 5, 20000 x 128 36 and 9.
      const bool ordered = top_k || top_p;
      if (C <= rows::kShortRow && (C <= 48 || !ordered || R >= 100 * (C - 32)))
        hipLaunchKernelGGL((sample_short<T>), dim3((unsigned)((n + rows::kShortRows - 1) / rows::kShortRows)), dim3(256),
                           0, s, a);
      // up to 32 values a lane: one wave, without barriers (in a block of 256 that lists and orders what is kept 23265 rows
      // of 590 bfloat16 with top-k 50 took 492 us, 110 so; one row of 1000 float32 14 and 10)
      else if (Q <= rows::kWaveVectors<T> * kWave)
        hipLaunchKernelGGL((sample_tile<T, kWave, rows::kWaveVectors<T>>), grid, dim3(kWave), 0, s, a);
      else if (Q <= 4 * 256)
        hipLaunchKernelGGL((sample_tile<T, 256, 4>), grid, dim3(256), 0, s, a);
      else if (Q <= 4 * 1024)
        hipLaunchKernelGGL((sample_tile<T, 1024, 4>), grid, dim3(1024), 0, s, a);
      // (the workspace's size is that of rows that are not aligned, which may be a vector longer)
      else if (const int parts = split_parts(R, C, dtype); parts > 1 && (Q > 16 * 1024 || R <= cu_count() / 2)) {
        Split split;
        Split::carve(workspace, R, parts, &split);
        split.each = (Q + parts - 1) / parts;
        const dim3 all((unsigned)(R * parts)), threads(kPartThreads);
        hipLaunchKernelGGL((split_max<T>), all, threads, 0, s, a, split);
        if (top_k || top_p) hipLaunchKernelGGL((split_sum<T>), all, threads, 0, s, a, split);
        if (top_p) hipLaunchKernelGGL((split_cut<T>), grid, dim3(kBins), 0, s, a, split);
        hipLaunchKernelGGL((split_share<T>), all, threads, 0, s, a, split);
        hipLaunchKernelGGL((split_draw<T>), grid, dim3(kDrawThreads), 0, s, a, split);
      } else if (Q <= 16 * 1024)
        hipLaunchKernelGGL((sample_tile<T, 1024, 16>), grid, dim3(1024), 0, s, a);
      else
        hipLaunchKernelGGL((sample_rows<T, 1024>), grid, dim3(1024), 0, s, a);
      return launch_status();
    });
  });
}
