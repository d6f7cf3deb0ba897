// Rows of an embedding picked by token, times a scale, and the embedding's gradient.
//
//   out[r] = scale E[id_r],   dE[v] = scale sum over the rows r with id_r = v of dout[r]
//
// Both are streams: the lookup reads and writes R rows of N, the gradient reads R rows and writes V. A token's rows are
// summed in their order, so the rows are first sorted by token (stable):
//   up to 16384 rows: every row counts the rows that come before it (embed_rank, one launch, R^2 comparisons)
//   more: by digits of 9 bits from the lowest on, a pass of counts, their prefix and places each
// and the sorted rows are cut into chunks of `per` rows: embed_sum sums the runs of a token inside a chunk and writes the
// gradient of tokens that lie wholly in one; what reaches over a chunk's end is kept as partial sums, which embed_rest
// adds up in a fixed order while it clears the rows of tokens that did not occur. Frequent tokens (a tenth of a text is one
// token) so are the work of many blocks, and the result does not depend on which of them ends first. Sums are float32
// over at most 128 rows, float64 over the chunks; a result is rounded once. 128000 rows of 131072 x 1024 float32: the lookup 139
// us, the gradient 280, of which the sort 47; 8192 of 32003 x 1024 bfloat16: 6 and 31, the sort 10.
#include <algorithm>

#include "vectors.h"

namespace snn {
namespace {

using namespace vectors;

constexpr int kThreads = 256;
// Rows sorted by counting (64 KB of keys in LDS); us of lookup and gradient of rows x 256 float32 so and by digits: 8192
// rows of 32003 tokens 29, 53; 16384 45, 57, of 500 tokens (one digit less) 43, 39.
constexpr int kRankRows = 16384;
constexpr int kRankThreads = 1024;
constexpr int kRankShare = 32;     // threads that share a row's comparisons
constexpr int kDigit = 9;          // bits of a digit
constexpr int kBins = 1 << kDigit;
constexpr int kSortThreads = 256;
// Steps of 64 rows of a wavefront: few where that is needed to fill the card (128000 rows, two passes: counts and places
// 11 us a pass with 4, 23 with 16), more for the longest lists, whose counts (a block's 512 each) would grow too large.
constexpr int kFewSteps = 4, kManySteps = 16;
constexpr int64_t kFewStepsRows = (int64_t)1 << 20;
int sort_rows(int64_t R) { return kSortThreads * (R <= kFewStepsRows ? kFewSteps : kManySteps); }
constexpr int kMaxPer = 128;
constexpr int kMaxWidth = 1 << 20;

// Lanes that share a row of N: a power of two, at most a wavefront.
int lanes_log2(int N, int E) {
  const int q = (N + E - 1) / E;
  int s = 2;
  while (s < 6 && (1 << s) < q) ++s;
  return s;
}

template <class T>
constexpr int kE = 16 / (int)sizeof(T);

// x * scale as a float32: the compiler would form a float16 product and its rounding in one instruction, whose results differ
// from the other types' way (product in float32, then rounded) by the second rounding.
__device__ __forceinline__ float scaled(float x, float scale) {
  float p = x * scale;
  asm("" : "+v"(p));
  return p;
}

template <class T>
__global__ __launch_bounds__(kThreads) void embed_lookup(const T* __restrict__ E, int64_t V, int N, int64_t ld_e,
                                                         const int32_t* __restrict__ ids, int64_t R, float scale,
                                                         T* __restrict__ out, int64_t ld_out, int sh) {
  const int64_t r = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> sh;
  if (r >= R) return;
  const int lanes = 1 << sh;
  const int l = threadIdx.x & (lanes - 1);
  const int64_t id = ids[r];
  const bool ok = id >= 0 && id < V;
  const T* e = E + (ok ? id : 0) * ld_e;
  T* o = out + r * ld_out;
  constexpr int kAhead = 4;  // vectors under way
  for (int i = l * kE<T>; i < N; i += kAhead * lanes * kE<T>) {
    Raw<T, kE<T>> raw[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) raw[q] = span_load<T, kE<T>>(e, i + q * lanes * kE<T>, N);
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      float x[kE<T>];
      raw[q].to(x);
#pragma unroll
      for (int u = 0; u < kE<T>; ++u) x[u] = ok ? scaled(x[u], scale) : 0.0f;
      span_store<T, kE<T>, true>(o, i + q * lanes * kE<T>, N, x);
    }
  }
}

// ------------------------------------------------------------------ rows sorted by token

// A row's key: its token, or V for a row without one (these come last and are left out).
__device__ __forceinline__ uint32_t key_of(int32_t id, int64_t V) {
  return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V;
}

__global__ void embed_clear_ends(int32_t* __restrict__ first, int64_t V) {
  for (int64_t v = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; v < V; v += (int64_t)gridDim.x * blockDim.x)
    first[v] = -1;
}

// The place of each row among all R <= kRankRows: how many rows have a smaller key, or the same and come before it. A block
// ranks 32 rows, 32 threads share a row, four keys a read. first[v] = -1 for every token on the way. 8192 rows: 10 us
// (56 with 8 threads a row, 256 a block and a key a read).
__global__ __launch_bounds__(kRankThreads) void embed_rank(const int32_t* __restrict__ ids, int R, int64_t V,
                                                           uint32_t* __restrict__ keys, int32_t* __restrict__ order,
                                                           int32_t* __restrict__ first) {
  extern __shared__ __attribute__((aligned(16))) uint32_t k[];  // R keys, up to a multiple of 4 of the largest value
  const int Q = (R + 3) / 4;
  for (int64_t v = (int64_t)blockIdx.x * kRankThreads + threadIdx.x; v < V; v += (int64_t)gridDim.x * kRankThreads) first[v] = -1;
  if (blockIdx.x * (kRankThreads / kRankShare) >= (unsigned)R) return;
  for (int i = threadIdx.x; i < 4 * Q; i += kRankThreads) k[i] = i < R ? key_of(ids[i], V) : 0xffffffffu;
  __syncthreads();
  const int r = min(blockIdx.x * (kRankThreads / kRankShare) + threadIdx.x / kRankShare, (unsigned)R - 1);
  const int part = threadIdx.x % kRankShare;
  const uint32_t mine = k[r];  // at most 2^31 - 1
  const int own = r / 4;
  const uint4* k4 = reinterpret_cast<const uint4*>(k);
  int before = 0;
  const auto count = [&](int q, uint32_t than) {
    const uint4 x = k4[q];
    before += (x.x < than) + (x.y < than) + (x.z < than) + (x.w < than);
  };
#pragma unroll 4
  for (int q = part; q < own; q += kRankShare) count(q, mine + 1);
#pragma unroll 4
  for (int q = own + 1 + part; q < Q; q += kRankShare) count(q, mine);
  if (part < 4) {
    const int j = 4 * own + part;
    before += k[j] < mine + (j < r ? 1 : 0);
  }
#pragma unroll
  for (int off = kRankShare / 2; off > 0; off >>= 1) before += __shfl_xor(before, off, kWave);
  if (part == 0 && blockIdx.x * (kRankThreads / kRankShare) + threadIdx.x / kRankShare < (unsigned)R) {
    keys[before] = mine;
    order[before] = r;
  }
}

__device__ __forceinline__ int digit_of(uint32_t k, int shift) { return (int)(k >> shift) & (kBins - 1); }

// counts[d * blocks + block]: the block's rows with digit d. keys NULL: the rows' own (the first pass).
template <int kSortSteps>
__global__ __launch_bounds__(kSortThreads) void embed_count(const uint32_t* __restrict__ keys,
                                                            const int32_t* __restrict__ ids, int R, int64_t V, int shift,
                                                            int32_t* __restrict__ counts) {
  __shared__ int n[kBins];
  for (int d = threadIdx.x; d < kBins; d += kSortThreads) n[d] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * (kSortThreads * kSortSteps);
  for (int s = 0; s < kSortSteps; ++s) {
    const int64_t i = base + s * kSortThreads + threadIdx.x;
    if (i < R) atomicAdd(&n[digit_of(keys ? keys[i] : key_of(ids[i], V), shift)], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < kBins; d += kSortThreads) counts[(size_t)d * gridDim.x + blockIdx.x] = n[d];
}

// Each row to its place: after the rows of smaller digits, of the same digit in earlier blocks (offs, the prefix of
// counts), in earlier wavefronts of the block and in earlier lanes. A wavefront owns kSortSteps * 64 rows in a row.
template <int kSortSteps>
__global__ __launch_bounds__(kSortThreads) void embed_place(const uint32_t* __restrict__ keys,
                                                            const int32_t* __restrict__ order,
                                                            const int32_t* __restrict__ ids, int R, int64_t V, int shift,
                                                            const int32_t* __restrict__ offs,
                                                            uint32_t* __restrict__ keys_out,
                                                            int32_t* __restrict__ order_out) {
  constexpr int W = kSortThreads / kWave;
  __shared__ int at[W][kBins];
  const int w = threadIdx.x / kWave, l = lane_id();
  for (int d = threadIdx.x; d < W * kBins; d += kSortThreads) (&at[0][0])[d] = 0;
  __syncthreads();
  const int64_t base = ((int64_t)blockIdx.x * (kSortThreads / kWave) + w) * (kSortSteps * kWave);
  uint32_t k[kSortSteps];
#pragma unroll
  for (int s = 0; s < kSortSteps; ++s) {
    const int64_t i = base + s * kWave + l;
    k[s] = i < R ? (keys ? keys[i] : key_of(ids[i], V)) : 0u;
    if (i < R) atomicAdd(&at[w][digit_of(k[s], shift)], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < kBins; d += kSortThreads) {
    int o = offs[(size_t)d * gridDim.x + blockIdx.x];
#pragma unroll
    for (int q = 0; q < W; ++q) {
      const int n = at[q][d];
      at[q][d] = o;
      o += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < kSortSteps; ++s) {
    const int64_t i = base + s * kWave + l;
    const bool in = i < R;
    const int d = digit_of(k[s], shift);
    uint64_t same = __ballot(in);
#pragma unroll
    for (int b = 0; b < kDigit; ++b) {
      const bool bit = (d >> b) & 1;
      const uint64_t m = __ballot(in && bit);
      same &= bit ? m : ~m;
    }
    const int p = in ? at[w][d] : 0;
    __builtin_amdgcn_wave_barrier();  // every lane has read its place before one moves it on
    const int before = mask_prefix(same);
    if (in && before == 0) at[w][d] = p + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (in) {
      keys_out[p + before] = k[s];
      order_out[p + before] = order ? order[i] : (int32_t)i;
    }
  }
}

// ------------------------------------------------------------------ sums

// Chunk c of `per` sorted rows: lanes 1 << sh a chunk and slab of columns. first[v], last[v]: the sorted rows of token v.
// head[c], tail[c]: partial sums of the run that began before the chunk and of the one that goes on after it (a run
// that does both is a head).
template <class T>
__global__ __launch_bounds__(kThreads) void embed_sum(const uint32_t* __restrict__ keys, const int32_t* __restrict__ order,
                                                      int R, int64_t V, int N, const T* __restrict__ dout, int64_t ld,
                                                      float scale, int per, int chunks, int slabs, int sh,
                                                      T* __restrict__ dE, int64_t ld_e, int accumulate,
                                                      int32_t* __restrict__ first, int32_t* __restrict__ last,
                                                      float* __restrict__ head, float* __restrict__ tail) {
  const int64_t job = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> sh;
  const int c = (int)(job / slabs), slab = (int)(job % slabs);
  if (c >= chunks) return;
  const int l = threadIdx.x & ((1 << sh) - 1);
  const int i = (slab * (1 << sh) + l) * kE<T>;  // this lane's columns
  const int lo = c * per, hi = min(R, lo + per);
  constexpr int kAhead = 8;  // rows under way
  float acc[kE<T>];
#pragma unroll
  for (int u = 0; u < kE<T>; ++u) acc[u] = 0.0f;
  uint32_t prev = lo > 0 ? keys[lo - 1] : 0xffffffffu;  // no key: V <= 2^31 - 1
  const uint32_t after = hi < R ? keys[hi] : 0xffffffffu;
  bool began = keys[lo] != prev;                        // the present run began in this chunk
  struct Batch {
    Raw<T, kE<T>> raw[kAhead];
    uint32_t k[kAhead + 1];
  };
  const auto fetch = [&](Batch& f, int p) {
    int32_t r[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      f.k[u] = p + u < hi ? keys[p + u] : after;
      r[u] = order[min(p + u, hi - 1)];
    }
    f.k[kAhead] = p + kAhead < hi ? keys[p + kAhead] : after;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) f.raw[u] = span_load<T, kE<T>>(dout + r[u] * ld, i, N);
  };
  const auto add = [&](const Batch& f, int p) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const uint32_t k = f.k[u];
      if (p + u < hi && k < (uint32_t)V) {
        float x[kE<T>];
        f.raw[u].to(x);
#pragma unroll
        for (int q = 0; q < kE<T>; ++q) acc[q] += x[q];
        const bool begins = k != prev, ends = f.k[u + 1] != k || p + u + 1 == R;
        if (begins && slab == 0 && l == 0) first[k] = p + u;
        if (ends && slab == 0 && l == 0) last[k] = p + u + 1;
        if (begins) began = true;
        if (ends || p + u + 1 == hi) {
          if (began && ends) {
            T* row = dE + (int64_t)k * ld_e;
            if (i < N) {
              float y[kE<T>], old[kE<T>];
              if (accumulate) span_load<T, kE<T>>(row, i, N).to(old);
#pragma unroll
              for (int q = 0; q < kE<T>; ++q) y[q] = accumulate ? fmaf(acc[q], scale, old[q]) : acc[q] * scale;
              span_store<T, kE<T>, true>(row, i, N, y);
            }
          } else {
            float* part = (began ? tail : head) + (size_t)c * N;
            if (i < N) span_store<float, kE<T>, false>(part, i, N, acc);
          }
#pragma unroll
          for (int q = 0; q < kE<T>; ++q) acc[q] = 0.0f;
        }
      }
      prev = k;
    }
  };
  // the next batch's rows are requested before the present one's sums are stored: loads and stores retire in order
  Batch f0, f1;
  fetch(f0, lo);
  for (int p = lo; p < hi; p += 2 * kAhead) {
    if (p + kAhead < hi) fetch(f1, p + kAhead);
    add(f0, p);
    if (p + kAhead < hi) {
      if (p + 2 * kAhead < hi) fetch(f0, p + 2 * kAhead);
      add(f1, p + kAhead);
    }
  }
}

// Blocks [0, jobs): a chunk and slab each, the token whose rows begin in the chunk and go on behind it, if there is one: its
// partial sums in float64 (a chunk has at most 128 rows, so their number grows with the token's), the wavefronts a quarter
// of them each. The others: rows of zeros for the tokens that did not occur
// (first[v] < 0), a wavefront kZeros tokens.
constexpr int kZeros = 4;
template <class T>
__global__ __launch_bounds__(kThreads) void embed_rest(const uint32_t* __restrict__ keys, int R, int64_t V, int N,
                                                       const int32_t* __restrict__ first,
                                                       const int32_t* __restrict__ last, const float* __restrict__ head,
                                                       const float* __restrict__ tail, float scale, int per, int slabs,
                                                       int jobs, T* __restrict__ dE, int64_t ld_e, int accumulate) {
  constexpr int W = kThreads / kWave;
  const int w = threadIdx.x / kWave, l = lane_id();
  if ((int)blockIdx.x >= jobs) {
    float zero[kE<T>];
#pragma unroll
    for (int u = 0; u < kE<T>; ++u) zero[u] = 0.0f;
    for (int64_t v0 = ((int64_t)(blockIdx.x - jobs) * W + w) * kZeros; v0 < V;
         v0 += (int64_t)(gridDim.x - jobs) * W * kZeros) {
      uint64_t absent = __ballot(l < kZeros && v0 + l < V && first[min(v0 + l, V - 1)] < 0);
      while (absent) {
        const int64_t v = v0 + __builtin_ctzll(absent);
        absent &= absent - 1;
        for (int i = l * kE<T>; i < N; i += kWave * kE<T>) store_past_in<T, kE<T>>(dE + v * ld_e, i, N, zero);
      }
    }
    return;
  }
  const int c0 = blockIdx.x / slabs, slab = blockIdx.x % slabs;
  const int64_t hi = (int64_t)(c0 + 1) * per;
  if (hi >= R) return;
  const uint32_t k = keys[hi - 1];
  if (k >= (uint32_t)V || keys[hi] != k || first[k] / per != c0) return;
  const int n = (last[k] - 1) / per - c0;  // chunks behind c0
  const int share = (n + W - 1) / W;
  const int i = (slab * kWave + l) * kE<T>;
  double y[kE<T>];
#pragma unroll
  for (int u = 0; u < kE<T>; ++u) y[u] = 0.0;
  if (w == 0) {
    float x[kE<T>];
    span_load<float, kE<T>>(tail + (size_t)c0 * N, i, N).to(x);
#pragma unroll
    for (int u = 0; u < kE<T>; ++u) y[u] = (double)x[u];
  }
#pragma unroll 8
  for (int c = c0 + 1 + w * share; c <= c0 + min(n, (w + 1) * share); ++c) {
    float x[kE<T>];
    span_load<float, kE<T>>(head + (size_t)c * N, i, N).to(x);
#pragma unroll
    for (int u = 0; u < kE<T>; ++u) y[u] += (double)x[u];
  }
  __shared__ double all[W][kWave][kE<T> + 1];
#pragma unroll
  for (int u = 0; u < kE<T>; ++u) all[w][l][u] = y[u];
  __syncthreads();
  if (w > 0 || i >= N) return;
  T* row = dE + (int64_t)k * ld_e;
  float old[kE<T>], out[kE<T>];
  if (accumulate) span_load<T, kE<T>>(row, i, N).to(old);
#pragma unroll
  for (int u = 0; u < kE<T>; ++u) {
#pragma unroll
    for (int o = 1; o < W; ++o) y[u] += all[o][l][u];
    out[u] = (float)(accumulate ? fma(y[u], (double)scale, (double)old[u]) : y[u] * (double)scale);
  }
  span_store<T, kE<T>, true>(row, i, N, out);
}

struct GradPlan {
  int per, chunks;
  int sort_blocks, passes;
};

GradPlan plan_grad(int64_t R, int64_t V) {
  GradPlan p;
  p.per = 8;
  while (p.per < kMaxPer && (R + p.per - 1) / p.per > 2048) p.per *= 2;
  p.chunks = (int)((R + p.per - 1) / p.per);
  p.sort_blocks = (int)((R + sort_rows(R) - 1) / sort_rows(R));
  p.passes = 0;
  for (int64_t top = V; top > 0; top >>= kDigit) ++p.passes;  // the largest key is V
  return p;
}

struct GradWorkspace {
  uint32_t* keys[2];
  int32_t* order[2];
  int32_t *counts, *offs, *temp, *first, *last;
  int64_t* total;
  float *head, *tail;
  size_t bytes;
};

GradWorkspace carve_grad(void* ws, int64_t R, int64_t V, int N, const GradPlan& p) {
  Carve c(ws);
  GradWorkspace g;
  const bool rank = R <= kRankRows;
  for (int k = 0; k < 2; ++k) {
    const size_t n = rank && k == 1 ? 0 : (size_t)R;
    g.keys[k] = c.take<uint32_t>(n);
    g.order[k] = c.take<int32_t>(n);
  }
  const size_t counts = rank ? 0 : (size_t)kBins * p.sort_blocks;
  g.counts = c.take<int32_t>(counts);
  g.offs = c.take<int32_t>(counts + 1);
  g.temp = c.take<int32_t>(rank ? 0 : scan_temp_elems((int)counts));
  g.total = c.take<int64_t>(1);
  g.first = c.take<int32_t>((size_t)V);
  g.last = c.take<int32_t>((size_t)V);
  g.head = c.take<float>((size_t)p.chunks * N);
  g.tail = c.take<float>((size_t)p.chunks * N);
  g.bytes = c.off;
  return g;
}

template <class T>
void launch_lookup(const void* E, int64_t V, int N, int64_t ld_e, const int32_t* ids, int64_t R, float scale, void* out,
                   int64_t ld_out, hipStream_t s) {
  const int sh = lanes_log2(N, kE<T>);
  const int64_t step = (int64_t)1 << 22;  // rows of a launch: a dispatch counts threads in 32 bits
  for (int64_t r = 0; r < R; r += step) {
    const int64_t n = std::min(step, R - r);
    hipLaunchKernelGGL(embed_lookup<T>, dim3((unsigned)(((n << sh) + kThreads - 1) / kThreads)), dim3(kThreads), 0, s,
                       static_cast<const T*>(E), V, N, ld_e, ids + r, n, scale, static_cast<T*>(out) + r * ld_out, ld_out,
                       sh);
  }
}

template <class T>
void launch_sums(int R, int64_t V, int N, const void* dout, int64_t ld, float scale, void* dE, int64_t ld_e,
                 int accumulate, const GradPlan& p, const GradWorkspace& g, const uint32_t* keys, const int32_t* order,
                 hipStream_t s) {
  const int sh = lanes_log2(N, kE<T>);
  const int slabs = (N + (kE<T> << sh) - 1) / (kE<T> << sh);
  const int64_t threads = ((int64_t)p.chunks * slabs) << sh;
  hipLaunchKernelGGL(embed_sum<T>, dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, keys,
                     order, R, V, N, static_cast<const T*>(dout), ld, scale, p.per, p.chunks, slabs, sh,
                     static_cast<T*>(dE), ld_e, accumulate, g.first, g.last, g.head, g.tail);
  const int wide = (N + kE<T> * kWave - 1) / (kE<T> * kWave);
  const int jobs = p.chunks * wide;
  const int64_t zeros = accumulate ? 0 : std::min<int64_t>((V + kZeros * kThreads / kWave - 1) / (kZeros * kThreads / kWave), 1 << 20);
  hipLaunchKernelGGL(embed_rest<T>, dim3((unsigned)(jobs + zeros)), dim3(kThreads), 0, s, keys, R, V, N, g.first, g.last,
                     g.head, g.tail, scale, p.per, wide, jobs, static_cast<T*>(dE), ld_e, accumulate);
}

// The sizes that both calls refuse.
snn_status check_sizes(int dtype, int64_t V, int N, int64_t R) {
  if (!dtype_size(dtype) || V <= 0 || N <= 0 || R <= 0) return SNN_ERR_INVALID_ARG;
  if (V > INT32_MAX || R > INT32_MAX || N > kMaxWidth) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

// Whether the grids of embed_sum and embed_rest can be launched.
bool sums_fit(int64_t R, int64_t V, int N) {
  const GradPlan p = plan_grad(R, V);
  // a dispatch counts threads in 32 bits
  return R < ((int64_t)1 << 30) && (int64_t)p.chunks * ((N + 255) / 256) * kThreads < ((int64_t)1 << 31);
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" snn_status snn_embed(const void* E, int dtype, int64_t V, int N, int64_t ld_e, const int32_t* ids, int64_t R,
                                float scale, void* out, int64_t ld_out, void* stream) {
  if (!E || !ids || !out) return SNN_ERR_INVALID_ARG;
  if (const snn_status st = check_sizes(dtype, V, N, R)) return st;
  if (ld_e < N || ld_out < N || isnan(scale)) return SNN_ERR_INVALID_ARG;
  if (misaligned(E, dtype) || misaligned(out, dtype)) return SNN_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == SNN_F32) launch_lookup<float>(E, V, N, ld_e, ids, R, scale, out, ld_out, s);
  else if (dtype == SNN_BF16) launch_lookup<Bf16>(E, V, N, ld_e, ids, R, scale, out, ld_out, s);
  else launch_lookup<F16>(E, V, N, ld_e, ids, R, scale, out, ld_out, s);
  return launch_status();
}

extern "C" size_t snn_embed_grad_workspace(int dtype, int64_t V, int N, int64_t R) {
  if (check_sizes(dtype, V, N, R) != SNN_OK || !sums_fit(R, V, N)) return 0;
  return carve_grad(nullptr, R, V, N, plan_grad(R, V)).bytes;
}

extern "C" snn_status snn_embed_grad(const int32_t* ids, int64_t R, const void* dout, int dtype, int64_t ld_out, int64_t V,
                                     int N, float scale, void* dE, int64_t ld_e, int accumulate, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  if (!ids || !dout || !dE || !workspace) return SNN_ERR_INVALID_ARG;
  if (const snn_status st = check_sizes(dtype, V, N, R)) return st;
  if (ld_e < N || ld_out < N || isnan(scale)) return SNN_ERR_INVALID_ARG;
  if (misaligned(dout, dtype) || misaligned(dE, dtype)) return SNN_ERR_INVALID_ARG;
  if (!sums_fit(R, V, N)) return SNN_ERR_UNSUPPORTED;
  const GradPlan p = plan_grad(R, V);
  const GradWorkspace g = carve_grad(workspace, R, V, N, p);
  if (workspace_bytes < g.bytes) return SNN_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  int at = 0;
  if (R <= kRankRows) {
    const int64_t clear = std::min<int64_t>((V + 4095) / 4096, 256);  // blocks past the rows clear first[] alone
    const int rows = kRankThreads / kRankShare;
    hipLaunchKernelGGL(embed_rank, dim3((unsigned)std::max((R + rows - 1) / rows, clear)), dim3(kRankThreads),
                       (size_t)(R + 3) / 4 * 16, s, ids, (int)R, V, g.keys[0], g.order[0], g.first);
  } else {
    hipLaunchKernelGGL(embed_clear_ends, dim3((unsigned)std::min<int64_t>((V + 255) / 256, 4096)), dim3(256), 0, s, g.first,
                       V);
    for (int pass = 0; pass < p.passes; ++pass) {
      const uint32_t* from = pass ? g.keys[at] : nullptr;
      const int32_t* rows = pass ? g.order[at] : nullptr;
      const int to = pass ? at ^ 1 : 0;
      const dim3 grid((unsigned)p.sort_blocks);
      const bool few = R <= kFewStepsRows;
      hipLaunchKernelGGL((few ? embed_count<kFewSteps> : embed_count<kManySteps>), grid, dim3(kSortThreads), 0, s, from, ids,
                         (int)R, V, pass * kDigit, g.counts);
      launch_exclusive_scan(g.counts, kBins * p.sort_blocks, g.offs, g.total, g.temp, s);
      hipLaunchKernelGGL((few ? embed_place<kFewSteps> : embed_place<kManySteps>), grid, dim3(kSortThreads), 0, s, from, rows,
                         ids, (int)R, V, pass * kDigit, g.offs, g.keys[to], g.order[to]);
      at = to;
    }
  }
  if (dtype == SNN_F32)
    launch_sums<float>((int)R, V, N, dout, ld_out, scale, dE, ld_e, accumulate, p, g, g.keys[at], g.order[at], s);
  else if (dtype == SNN_BF16)
    launch_sums<Bf16>((int)R, V, N, dout, ld_out, scale, dE, ld_e, accumulate, p, g, g.keys[at], g.order[at], s);
  else
    launch_sums<F16>((int)R, V, N, dout, ld_out, scale, dE, ld_e, accumulate, p, g, g.keys[at], g.order[at], s);
  return launch_status();
}
