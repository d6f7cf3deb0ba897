// A teacher's record of its answers: the K largest logits of every row with their classes, largest first and equal
// ones by class, and the row's log-sum-exp at a temperature, which gives the listed classes' probabilities and what
// is left for the others.
//
// A row is read once into registers (up to 64 float32 or 128 16-bit values a thread). What is listed is found by a
// bound from below that costs no pass: with each lane's largest value at hand, the ceil(K/waves)-th largest of every
// wave's lanes, and the smallest of those over the waves. At least K values reach it, and hardly more do when values
// lie in no particular order along the row (a thread's vectors are a block's width apart, so that a run of likely
// classes is spread over all waves). One comparison a value collects them in LDS, where each counts those before it.
// Rows of up to 128 classes go 16 lanes each (top_short), of up to 2048 a wave each, which finds the cut by halving a
// range of values and lists just the K before it (top_wave). Where too many reach the bound (long runs of equal values),
// where K needs more than kNthMost of a wave, and for rows beyond the registers, the cut is found by histograms of the
// row as it lies in memory (top_general).
//
// Measured: 128000 x 100 float32, K 8: 20.5 us (2.9 TB/s), bound by vector instructions (issued 78% of the time, 409 a wave
// of four rows); 2048 x 32003 bfloat16, K 64: 48.7 us (2.7 TB/s), vector instructions 58% of the time, waves waiting 48% of
// theirs; 24 x 131072 float16, K 50, in parts: 22.6 us, two launches that wait 58 and 78% of the time.
#include "rows.h"

namespace snn {
namespace {

using namespace rows;

// Lanes of each wave that the bound is taken from, at most: with n of 64 lanes -64 log(1 - n/64) of its values reach it,
// somewhat more where the smallest of several waves counts.
constexpr int kNthMost = 32;
// Waves of a block whose lanes all hold a vector of a row with at least Q of them.
template <int NT>
__host__ __device__ constexpr int full_waves(int Q) {
  return Q / kWave < 1 ? 1 : Q / kWave < NT / kWave ? Q / kWave : NT / kWave;
}
template <int NT>
__host__ __device__ constexpr int nth_of(int K, int Q) {
  return (K + full_waves<NT>(Q) - 1) / full_waves<NT>(Q);
}
constexpr float kLog2e = 1.44269504088896340736f;

template <int NT>
struct TopLds {
  static constexpr int kList = 1024;
  union {
    SelectLds<NT> select;
    uint64_t list[kList];
  };
  uint64_t taken[kMaxListed];
  float fred[NT / kWave];
  uint32_t ured[NT / kWave];
  uint32_t n_taken;
};

struct Top {
  const void* logits;
  int64_t R;
  int C;
  int64_t ld;
  int K;
  float inv;
  int32_t* ids;
  float* vals;
  float* lse;
  int parts;   // of a row, each with a record of its own
  int part_C;  // classes of a part
};

__device__ __forceinline__ uint64_t entry(uint32_t key, int j) { return (uint64_t)~key << 32 | (uint32_t)j; }

// Beyond this many entries a sort takes less than comparing each with all others.
template <int NT>
constexpr int kSorted = NT == kWave ? 64 : 256;

// Classes and logits of the n collected entries by their place among them; the record's end where there are fewer.
template <class T, int NT>
__device__ __forceinline__ void write_record(const Row<T>& row, const Top& a, int64_t r, uint64_t* list, int n) {
  const bool sorted = n > kSorted<NT>;
  if (sorted) block_sort<NT>(list, n);
  for (int e = threadIdx.x; e < (sorted ? a.K : max(n, a.K)); e += NT) {
    int place = e, id = -1;
    float v = -INFINITY;
    if (e < n) {
      const uint64_t mine = list[e];
      place = sorted ? e : 0;
#pragma unroll 4
      for (int o = 0; o < (sorted ? 0 : n); ++o) place += list[o] < mine;
      id = (int)(uint32_t)mine;
      if (place < a.K) v = row.at(id);
    }
    if (place < a.K) {
      a.ids[r * a.K + place] = id;
      a.vals[r * a.K + place] = v;
    }
  }
}

// Rows of at most kShortRow classes. A lane's largest value has so many lanes' above it; the smallest of those with
// fewer than K above bounds the K-th value from below (with K > 16 every value is collected).
template <class T>
__global__ __launch_bounds__(256) void top_short(Top a) {
  __shared__ uint64_t list[kShortRows][kShortRow];
  const int slot = threadIdx.x / 16, l = threadIdx.x % 16;
  const int64_t r = (int64_t)blockIdx.x * kShortRows + slot;
  const bool live = r < a.R;
  const Row<T> row(a.logits, min(r, a.R - 1), a.ld, a.C);
  float x[kShortEach];
  load_short(row, x);
  float most = -INFINITY;
  uint32_t key[kShortEach], own = 0;
#pragma unroll
  for (int i = 0; i < kShortEach; ++i) {
    x[i] = no_nan(x[i]);
    most = fmaxf(most, x[i]);
    key[i] = key_of(x[i]);
    own = max(own, key[i]);
  }
  uint32_t bound = 0;
  if (a.K <= 16) {
    int above = 0;
#define SNN_STEP(n) above += (uint32_t)__builtin_amdgcn_mov_dpp((int)own, 0x120 + n, 0xf, 0xf, true) > own
    SNN_STEP(1); SNN_STEP(2); SNN_STEP(3); SNN_STEP(4); SNN_STEP(5); SNN_STEP(6); SNN_STEP(7); SNN_STEP(8);
    SNN_STEP(9); SNN_STEP(10); SNN_STEP(11); SNN_STEP(12); SNN_STEP(13); SNN_STEP(14); SNN_STEP(15);
#undef SNN_STEP
    bound = above < a.K ? own : UINT32_MAX;
#define SNN_STEP(ctrl) bound = min(bound, (uint32_t)__builtin_amdgcn_mov_dpp((int)bound, ctrl, 0xf, 0xf, true))
    SNN_STEP(0xb1); SNN_STEP(0x4e); SNN_STEP(0x141); SNN_STEP(0x140);
#undef SNN_STEP
  }
  int n = 0;
#pragma unroll
  for (int i = 0; i < kShortEach; ++i) {
    if (16 * i >= a.C) break;
    const bool on = key[i] >= bound && x[i] > -INFINITY;
    int count;
    const int at = n + row16_place(on, count);
    if (on) list[slot][at] = entry(key[i], 16 * i + l);
    n += count;
  }
  if (a.lse) {
    most = row16_reduce(most, Larger());
    const Exponent ex = exponent_of(most, a.inv * kLog2e);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kShortEach; ++i) {
      if (16 * i >= a.C) break;
      sum += exp2_fast(fmaf(x[i], ex.c, -ex.mc));
    }
    sum = row16_reduce(sum, Plus());
    if (live && l == 0) a.lse[r] = isinf(most) ? most : most * a.inv + logf(sum);
  }
  __syncthreads();
  if (!live) return;
  for (int e = l; e < max(n, a.K); e += 16) {
    int place = e, id = -1;
    float v = -INFINITY;
    if (e < n) {
      const uint64_t mine = list[slot][e];
      place = 0;
#pragma unroll 4
      for (int o = 0; o < n; ++o) place += list[slot][o] < mine;
      id = (int)(uint32_t)mine;
      if (place < a.K) v = row.at(id);
    }
    if (place < a.K) {
      a.ids[r * a.K + place] = id;
      a.vals[r * a.K + place] = v;
    }
  }
}

template <class T, int NT>
__device__ __forceinline__ void top_general(const Row<T>& row, const Top& a, int64_t r, TopLds<NT>& s) {
  constexpr int kVec = Row<T>::kVec;
  const int tid = threadIdx.x;
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
  const auto larger = [](float x, float y) { return fmaxf(x, y); };
  const auto smaller = [](float x, float y) { return fminf(x, y); };
  const auto add = [](auto x, auto y) { return x + y; };
  m = block_reduce<NT>(m, larger, s.fred);
  least = block_reduce<NT>(least, smaller, s.fred);
  count = block_sum64<NT>(count, s.select.red);
  if (a.lse) {
    float sum = 0.0f;
    const float safe = isinf(m) ? 0.0f : m;
    for (int q = tid; q < row.Q; q += NT) {
      float x[kVec];
      row.load(q, x);
#pragma unroll
      for (int i = 0; i < kVec; ++i) sum += expf((no_nan(x[i]) - safe) * a.inv);
    }
    sum = block_reduce<NT>(sum, add, s.fred);
    if (tid == 0) a.lse[r] = isinf(m) ? m : m * a.inv + logf(sum);
  }
  uint32_t cut_key = 0;
  int last = a.C;  // class of the last listed element at the cut
  if (count > (uint64_t)a.K) {
    const auto one = [](float x) { return (uint32_t)(x > -INFINITY); };
    const Cut c = find_cut<T, NT, false>(row, one, key_of(least), key_of(m), (uint64_t)a.K, false, s.select);
    cut_key = c.key;
    const uint32_t ties = a.K - c.above_count;
    if (ties < c.equal)
      last = find_in_order<T, NT>(row, [&](float x, int) { return (uint64_t)(key_of(x) == cut_key); }, ties - 1,
                                  s.select.red, 0, row.Q);
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
        s.taken[atomicAdd(&s.n_taken, 1u)] = entry(k, j);
    }
  }
  __syncthreads();
  write_record<T, NT>(row, a, r, s.taken, (int)s.n_taken);
}

template <class T, int NT>
__global__ __launch_bounds__(NT) void top_rows(Top a) {
  __shared__ TopLds<NT> s;
  const int64_t r = blockIdx.x;
  top_general<T, NT>(Row<T>(a.logits, r, a.ld, a.C), a, r, s);
}

// False where the row takes the general way.
template <class T, int NT, int NV>
__device__ __forceinline__ bool top_in_registers(const Row<T>& row, const Top& a, int64_t r, TopLds<NT>& s) {
  constexpr int kVec = Row<T>::kVec;
  constexpr int kWaves = NT / kWave;
  const int tid = threadIdx.x;
  Tile<T, NT, NV> tile;
  tile.load(row);
  float most = -INFINITY;
  bool nan = false;
  tile.each_unrolled(row, [&](const float (&x)[kVec], int, int) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      most = fmaxf(most, x[i]);
      nan |= x[i] != x[i];
    }
  });
  const uint32_t key = nan ? 0u : key_of(most);  // 0 is no value's key
  uint32_t high = wave_max_u32(key);
  uint32_t bound = UINT32_MAX;  // a wave with idle lanes has no part in it
  const bool all = nth_of<NT>(a.K, row.Q) > kNthMost;  // every value is collected (of a short last part)
  if (tid / kWave < full_waves<NT>(row.Q)) bound = wave_nth(key, all ? 1 : nth_of<NT>(a.K, row.Q));
  bool odd = __ballot(nan) != 0;
  if (tid == 0) s.n_taken = 0;
  if (NT > kWave) {
    if (tid % kWave == 0) {
      s.ured[tid / kWave] = odd ? 0u : bound;
      s.fred[tid / kWave] = of_key(high);
    }
    __syncthreads();
    uint32_t b = s.ured[0];
    float m = s.fred[0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) {
      b = min(b, s.ured[k]);
      m = fmaxf(m, s.fred[k]);
    }
    bound = b;
    odd = b == 0;
    high = key_of(m);
  } else {
    __syncthreads();
  }
  const float m = of_key(high);
  if (odd || isinf(m)) return false;
  const float least = all ? -INFINITY : of_key(bound);
  const Exponent ex = exponent_of(m, a.inv * kLog2e);
  float sum = 0.0f;
  uint32_t some = 0;  // the vectors with a value that reaches the bound
  tile.each_unrolled(row, [&](const float (&x)[kVec], int, int n) {
    float part = 0.0f;
    bool any = false;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      part += exp2_fast(fmaf(x[i], ex.c, -ex.mc));
      any |= x[i] >= least;
    }
    sum += part;
    some |= any ? 1u << n : 0u;
  });
#pragma unroll 1
  for (int n = 0; n < NV; ++n) {
    if (__ballot(some >> n & 1) == 0) continue;
    if (some >> n & 1) {
      float x[kVec];
      unpack<T>(tile.get(n), x);
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (x[i] >= least && x[i] > -INFINITY) {
          const uint32_t at = atomicAdd(&s.n_taken, 1u);
          if (at < (uint32_t)TopLds<NT>::kList) s.list[at] = entry(key_of(x[i]), row.first(n * NT + tid) + i);
        }
    }
  }
  if (a.lse) {
    sum = block_reduce<NT>(sum, [](float x, float y) { return x + y; }, s.fred);
    if (tid == 0) a.lse[r] = m * a.inv + logf(sum);
  }
  __syncthreads();
  const int n = (int)s.n_taken;
  if (n > TopLds<NT>::kList) return false;
  write_record<T, NT>(row, a, r, s.list, n);
  return true;
}

template <class T, int NT, int NV>
__global__ __launch_bounds__(NT) void top_tile(Top a) {
  __shared__ TopLds<NT> s;
  const int64_t r = blockIdx.x;
  const int from = (int)(r % a.parts) * a.part_C;
  const Row<T> row(static_cast<const T*>(a.logits) + r / a.parts * a.ld + from, min(a.part_C, a.C - from));
  if (!top_in_registers<T, NT, NV>(row, a, r, s)) {
    __syncthreads();
    top_general<T, NT>(row, a, r, s);
  }
}

// ------------------------------------------------------------------ rows that one wave holds

// The K first are known by the cut, collected in a list of just their number and ordered there.
template <class T>
__global__ __launch_bounds__(kWave) void top_wave(Top a) {
  extern __shared__ uint64_t list[];  // K, up to the next power of two
  constexpr int kVec = Row<T>::kVec;
  const int64_t r = blockIdx.x;
  const Row<T> row(a.logits, r, a.ld, a.C);
  Tile<T, kWave, kWaveVectors<T>> tile;
  tile.load(row);
  float most = -INFINITY, least = INFINITY;
  tile.each_unrolled(row, [&](const float (&x)[kVec], int, int) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      most = fmaxf(most, x[i]);
      least = x[i] > -INFINITY ? fminf(least, x[i]) : least;
    }
  });
  const float m = of_key(wave_max_u32(key_of(most)));
  if (a.lse) {
    const Exponent ex = exponent_of(m, a.inv * kLog2e);
    float sum = 0.0f;
    tile.each_unrolled(row, [&](const float (&x)[kVec], int, int) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) sum += exp2_fast(fmaf(no_nan(x[i]), ex.c, -ex.mc));
    });
    sum = wave_reduce(sum, Plus());
    if (threadIdx.x == 0) a.lse[r] = isinf(m) ? m : m * a.inv + logf(sum);
  }
  float cut = -INFINITY;
  int last = INT32_MIN;  // none of -inf, which also stands around the row
  int n = count_in_wave(tile, row, [&](float x, int) { return x > -INFINITY; });
  if (n > a.K) {
    uint32_t lo = short_key<T>(of_key(~wave_max_u32(~key_of(least))));
    first_in_wave(tile, row, a.C, a.K, lo, short_key<T>(m) + 1, n, cut, last);
  }
  n = 0;
  tile.each_unrolled(row, [&](const float (&x)[kVec], int q, int) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int j = row.first(q) + i;
      const bool in = (x[i] > cut) | ((x[i] == cut) & (j <= last));
      const uint64_t all = __ballot(in);
      if (in) list[n + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0))] =
          entry(key_of(x[i]), j);
      n += __popcll(all);
    }
  });
  __syncthreads();
  write_record<T, kWave>(row, a, r, list, n);
}

// ------------------------------------------------------------------ few long rows, several blocks each

constexpr int kPartThreads = 512;
constexpr int kPartVectors = 4 * kPartThreads;
constexpr int kMerged = 1024;  // listed classes of a row's parts

// Rows of at least so many classes are shared among blocks though one block could hold them, where they leave most
// compute units idle. In a block each and so, K 50, kernels alone: 24 x 130000 float16 31 and 23 us, bfloat16 26 and 22;
// 128 x 130000 bfloat16 32 and 29; but 64 x 80000 bfloat16 21 and 22, 24 x 60000 float32 18 and 21, 24 x 20000 14 and 18.
constexpr int kSharedRow = 98304;
// Parts that a row is shared among: 1, or beyond a block's registers as many as hold it (8192 x 131072 float32, K 50: 2.9 ms
// in passes by a block each, 1.4 ms so). The parts' records take up to 8 KB a row: of at most 2^14 rows.
inline int top_parts(int64_t R, int C, int dtype, int K) {
  const int per = 16 / rows::type_size(dtype);
  const int Q = (C + 2 * per - 2) / per;  // as of a row that is not aligned
  if (Q <= 16 * 1024 ? C < kSharedRow || R > cu_count() / 2 : R > (1 << 14)) return 1;
  if (K > kPartThreads / kWave * 16) return 1;
  const int parts = (Q + kPartVectors - 2) / (kPartVectors - 1);  // the cuts may add a vector to each
  return parts * K <= kMerged && parts <= kWave ? parts : 1;
}
inline size_t top_carve(void* ws, int64_t R, int parts, int K, Top* a) {
  Carve c(ws);
  int32_t* ids = c.take<int32_t>((size_t)R * parts * K);
  float* vals = c.take<float>((size_t)R * parts * K);
  float* lse = c.take<float>((size_t)R * parts);
  if (a) {
    a->ids = ids;
    a->vals = vals;
    a->lse = lse;
  }
  return c.off;
}

// A row's record from its parts': `part` is the launch that wrote those, `a` the call's own.
__global__ __launch_bounds__(kMerged) void top_merge(Top part, Top a) {
  __shared__ uint64_t list[kMerged];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, n = part.parts * a.K;
  if (tid < n) {
    const int64_t e = r * n + tid;
    const int id = part.ids[e];
    list[tid] = id < 0 ? UINT64_MAX : entry(key_of(part.vals[e]), id + tid / a.K * part.part_C);
  }
  if (a.lse && tid < kWave) {
    const float x = tid < part.parts ? part.lse[r * part.parts + tid] : -INFINITY;
    const float m = wave_reduce(x, Larger()), safe = isinf(m) ? 0.0f : m;
    const float sum = wave_reduce(expf(x - safe), Plus());
    if (tid == 0) a.lse[r] = isinf(m) ? m : m + logf(sum);
  }
  __syncthreads();
  block_sort<kMerged>(list, n);
  if (tid < a.K) {
    const uint64_t e = list[tid];
    a.ids[r * a.K + tid] = e == UINT64_MAX ? -1 : (int)(uint32_t)e;
    a.vals[r * a.K + tid] = e == UINT64_MAX ? -INFINITY : of_key(~(uint32_t)(e >> 32));
  }
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" size_t snn_readout_top_workspace(int64_t R, int C, int dtype, int K) {
  if (R <= 0 || R > INT32_MAX || bad_dim(C) || C > rows::kMaxClasses || rows::type_size(dtype) == 0 || K <= 0 || K > C)
    return 0;
  const int parts = top_parts(R, C, dtype, K);
  return parts > 1 ? top_carve(nullptr, R, parts, K, nullptr) : 0;
}

extern "C" snn_status snn_readout_top(const void* logits, int dtype, int64_t R, int C, int64_t ld, int K, float tau,
                                      int32_t* ids, float* vals, float* lse, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  const snn_status ok = rows::check_rows(logits, dtype, R, C, ld);
  if (ok != SNN_OK) return ok;
  if (!ids || !vals || K <= 0 || K > C || !(tau > 0.0f) || isinf(tau)) return SNN_ERR_INVALID_ARG;
  if (K > rows::kMaxListed) return SNN_ERR_UNSUPPORTED;
  const size_t need = snn_readout_top_workspace(R, C, dtype, K);
  if (need && (!workspace || workspace_bytes < need)) return SNN_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return rows::for_type(dtype, [&](auto type) {
    using T = decltype(type);
    const int Q = rows::most_vectors<T>(logits, C, ld), least = C / rows::Row<T>::kVec;
    return rows::in_launches(R, [&](int64_t first, int64_t n) {
      const Top a{static_cast<const T*>(logits) + first * ld, n, C, ld, K, 1.0f / tau, ids + first * K, vals + first * K,
                  rows::or_null(lse, first), 1, C};
      const dim3 grid((unsigned)n);
      if (C <= rows::kShortRow)
        hipLaunchKernelGGL((top_short<T>), dim3((unsigned)((n + rows::kShortRows - 1) / rows::kShortRows)), dim3(256), 0,
                           s, a);
      // one wave (20000 rows of 700 float32, K 8, 40, 100: 38, 84, 338 us in blocks with the bound; 33, 39, 61 so)
      else if (Q <= rows::kWaveVectors<T> * kWave) {
        int size = 2;
        while (size < K) size <<= 1;
        hipLaunchKernelGGL((top_wave<T>), grid, dim3(kWave), size * sizeof(uint64_t), s, a);
      }
      // (the workspace's size is that of rows that are not aligned, which may be a vector longer)
      else if (const int parts = top_parts(R, C, dtype, K); parts > 1 && (Q > 16 * 1024 || (C >= kSharedRow && R <= cu_count() / 2))) {
        constexpr int kVec = rows::Row<T>::kVec;
        Top part = a;
        part.parts = parts;
        part.part_C = ((C + parts - 1) / parts + kVec - 1) / kVec * kVec;
        top_carve(workspace, R, parts, K, &part);
        hipLaunchKernelGGL((top_tile<T, kPartThreads, 4>), dim3((unsigned)(R * parts)), dim3(kPartThreads), 0, s, part);
        hipLaunchKernelGGL(top_merge, grid, dim3(kMerged), 0, s, part, a);
      } else if (Q <= 4 * 256 && nth_of<256>(K, least) <= kNthMost)
        hipLaunchKernelGGL((top_tile<T, 256, 4>), grid, dim3(256), 0, s, a);
      // (in 1024 threads and in 512, K 50, kernels alone: 64 x 9000 float32 15 and 10 us; bfloat16 256 x 32003 18 and 15,
      // 64 x 16000 16 and 11, but 16 x 32003 13 and 14)
      else if (Q <= 8 * 512 && nth_of<512>(K, least) <= kNthMost && (sizeof(T) == 4 || R >= cu_count() / 4))
        hipLaunchKernelGGL((top_tile<T, 512, 8>), grid, dim3(512), 0, s, a);
      else if (Q <= 4 * 1024 && nth_of<1024>(K, least) <= kNthMost)
        hipLaunchKernelGGL((top_tile<T, 1024, 4>), grid, dim3(1024), 0, s, a);
      else if (Q <= 16 * 1024 && nth_of<1024>(K, least) <= kNthMost)
        hipLaunchKernelGGL((top_tile<T, 1024, 16>), grid, dim3(1024), 0, s, a);
      else if (Q <= 4096)
        hipLaunchKernelGGL((top_rows<T, 256>), grid, dim3(256), 0, s, a);
      else
        hipLaunchKernelGGL((top_rows<T, 1024>), grid, dim3(1024), 0, s, a);
      return launch_status();
    });
  });
}
