// Rows of an embedding picked by token, times a scale, and the embedding's gradient.
//
//   out[r] = scale E[id_r],   dE[v] = scale sum over the rows r with id_r = v of dout[r]
//
// Both are streams: the lookup reads and writes R rows of N, the gradient reads R rows and writes V. A token's rows are
// summed in their order, so the rows are first sorted by token (stable):
//   up to kRankRows rows: every row counts the rows that come before it (embed_rank, one launch, R^2 comparisons)
//   more: by digits of 9 bits from the lowest on, a pass of counts, their prefix and places each
// and the sorted rows are cut into chunks of `per` rows: embed_sum sums the runs of a token inside a chunk and writes the
// gradient of tokens that lie wholly in one; what reaches over a chunk's end is kept as a partial sum, which embed_rest
// adds up in order while it clears the rows of tokens that did not occur. Frequent tokens (a tenth of a text is one
// token) so are the work of many blocks, and the result does not depend on which of them ends first. Sums are float32
// over at most 128 rows, then over the chunks; a result is rounded once.
#include <algorithm>

#include "vectors.h"

namespace snn {
namespace {

using namespace vectors;

constexpr int kThreads = 256;
constexpr int kRankRows = 8192;    // rows sorted by counting
constexpr int kDigit = 9;          // bits of a digit
constexpr int kBins = 1 << kDigit;
constexpr int kSortThreads = 256;
constexpr int kSortSteps = 16;     // steps of 64 rows of a wavefront
constexpr int kSortRows = kSortThreads * kSortSteps;
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
  for (int i = l * kE<T>; i < N; i += lanes * kE<T>) {
    float x[kE<T>];
    load_in<T, kE<T>>(e, i, N, x);
#pragma unroll
    for (int u = 0; u < kE<T>; ++u) x[u] = ok ? x[u] * scale : 0.0f;
    store_in<T, kE<T>>(o, i, N, x);
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

// The place of each row among all R <= kRankRows. A block ranks 32 rows, 8 threads a row share the comparisons.
// first[v] = -1 for every token on the way.
__global__ __launch_bounds__(kThreads) void embed_rank(const int32_t* __restrict__ ids, int R, int64_t V,
                                                       uint32_t* __restrict__ keys, int32_t* __restrict__ order,
                                                       int32_t* __restrict__ first) {
  __shared__ uint32_t k[kRankRows];
  for (int i = threadIdx.x; i < R; i += kThreads) k[i] = key_of(ids[i], V);
  for (int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x; v < V; v += (int64_t)gridDim.x * kThreads) first[v] = -1;
  __syncthreads();
  const int r = blockIdx.x * 32 + threadIdx.x / 8;
  const int part = threadIdx.x % 8;
  if (r >= R) return;
  const uint32_t mine = k[r];
  int before = 0;
  for (int j = part; j < r; j += 8) before += k[j] <= mine;
  for (int j = r + 1 + part; j < R; j += 8) before += k[j] < mine;
#pragma unroll
  for (int off = 4; off > 0; off >>= 1) before += __shfl_xor(before, off, kWave);
  if (part == 0) {
    keys[before] = mine;
    order[before] = r;
  }
}

__device__ __forceinline__ int digit_of(uint32_t k, int shift) { return (int)(k >> shift) & (kBins - 1); }

// counts[d * blocks + block]: the block's rows with digit d. keys NULL: the rows' own (the first pass).
__global__ __launch_bounds__(kSortThreads) void embed_count(const uint32_t* __restrict__ keys,
                                                            const int32_t* __restrict__ ids, int R, int64_t V, int shift,
                                                            int32_t* __restrict__ counts) {
  __shared__ int n[kBins];
  for (int d = threadIdx.x; d < kBins; d += kSortThreads) n[d] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortRows;
  for (int s = 0; s < kSortSteps; ++s) {
    const int64_t i = base + s * kSortThreads + threadIdx.x;
    if (i < R) atomicAdd(&n[digit_of(keys ? keys[i] : key_of(ids[i], V), shift)], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < kBins; d += kSortThreads) counts[(size_t)d * gridDim.x + blockIdx.x] = n[d];
}

// Each row to its place: after the rows of smaller digits, of the same digit in earlier blocks (offs, the prefix of
// counts), in earlier wavefronts of the block and in earlier lanes. A wavefront owns kSortSteps * 64 rows in a row.
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
  const int64_t base = (int64_t)blockIdx.x * kSortRows + w * kSortSteps * kWave;
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
  constexpr int kAhead = 8;
  float acc[kE<T>];
#pragma unroll
  for (int u = 0; u < kE<T>; ++u) acc[u] = 0.0f;
  uint32_t prev = lo > 0 ? keys[lo - 1] : 0xffffffffu;  // no key: V <= 2^31 - 1
  const uint32_t after = hi < R ? keys[hi] : 0xffffffffu;
  bool began = keys[lo] != prev;                        // the present run began in this chunk
  for (int p = lo; p < hi; p += kAhead) {
    float x[kAhead][kE<T>];
    uint32_t k[kAhead + 1];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) k[u] = p + u < hi ? keys[p + u] : after;
    k[kAhead] = p + kAhead < hi ? keys[p + kAhead] : after;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t r = order[min(p + u, hi - 1)];
      load_in<T, kE<T>>(dout + r * ld, min(i, N), N, x[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (p + u < hi && k[u] < (uint32_t)V) {
#pragma unroll
        for (int q = 0; q < kE<T>; ++q) acc[q] += x[u][q];
        const bool begins = k[u] != prev, ends = k[u + 1] != k[u] || p + u + 1 == R;
        if (begins && slab == 0 && l == 0) first[k[u]] = p + u;
        if (ends && slab == 0 && l == 0) last[k[u]] = p + u + 1;
        if (begins) began = true;
        if (ends || p + u + 1 == hi) {
          if (began && ends) {
            T* row = dE + (int64_t)k[u] * ld_e;
            if (i < N) {
              float y[kE<T>], old[kE<T>];
              if (accumulate) load_in<T, kE<T>>(row, i, N, old);
#pragma unroll
              for (int q = 0; q < kE<T>; ++q) y[q] = accumulate ? fmaf(acc[q], scale, old[q]) : acc[q] * scale;
              store_in<T, kE<T>>(row, i, N, y);
            }
          } else {
            float* part = (began ? tail : head) + (size_t)c * N;
            if (i < N) store_in<float, kE<T>>(part, i, N, acc);
          }
#pragma unroll
          for (int q = 0; q < kE<T>; ++q) acc[q] = 0.0f;
        }
      }
      prev = k[u];
    }
  }
}

// Tokens that reach over several chunks, and (without accumulate) rows of zeros for those that did not occur.
template <class T>
__global__ __launch_bounds__(kThreads) void embed_rest(int64_t V, int N, const int32_t* __restrict__ first,
                                                       const int32_t* __restrict__ last, const float* __restrict__ head,
                                                       const float* __restrict__ tail, float scale, int per, int sh,
                                                       T* __restrict__ dE, int64_t ld_e, int accumulate) {
  const int lanes = 1 << sh;
  const int l = threadIdx.x & (lanes - 1);
  for (int64_t v = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> sh; v < V; v += ((int64_t)gridDim.x * kThreads) >> sh) {
    const int f = first[v];
    int c0 = 0, c1 = -1;
    if (f >= 0) {
      c0 = f / per;
      c1 = (last[v] - 1) / per;
      if (c0 == c1) continue;
    } else if (accumulate) {
      continue;
    }
    T* row = dE + v * ld_e;
    for (int i = l * kE<T>; i < N; i += lanes * kE<T>) {
      float y[kE<T>];
#pragma unroll
      for (int u = 0; u < kE<T>; ++u) y[u] = 0.0f;
      if (f >= 0) {
        load_in<float, kE<T>>(tail + (size_t)c0 * N, i, N, y);
#pragma unroll 4
        for (int c = c0 + 1; c <= c1; ++c) {
          float x[kE<T>];
          load_in<float, kE<T>>(head + (size_t)c * N, i, N, x);
#pragma unroll
          for (int u = 0; u < kE<T>; ++u) y[u] += x[u];
        }
        float old[kE<T>];
        if (accumulate) load_in<T, kE<T>>(row, i, N, old);
#pragma unroll
        for (int u = 0; u < kE<T>; ++u) y[u] = accumulate ? fmaf(y[u], scale, old[u]) : y[u] * scale;
      }
      store_in<T, kE<T>>(row, i, N, y);
    }
  }
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
  p.sort_blocks = (int)((R + kSortRows - 1) / kSortRows);
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
  const int64_t rest = std::min<int64_t>(((V << sh) + kThreads - 1) / kThreads, (int64_t)1 << 20);
  hipLaunchKernelGGL(embed_rest<T>, dim3((unsigned)rest), dim3(kThreads), 0, s, V, N, g.first, g.last, g.head, g.tail,
                     scale, p.per, sh, static_cast<T*>(dE), ld_e, accumulate);
}

// The sizes that both calls refuse.
snn_status check_sizes(int dtype, int64_t V, int N, int64_t R) {
  if (!dtype_size(dtype) || V <= 0 || N <= 0 || R <= 0) return SNN_ERR_INVALID_ARG;
  if (V > INT32_MAX || R > INT32_MAX || N > kMaxWidth) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

// embed_sum's grid and partial sums: chunks of at least kMaxPer rows where R is large.
bool sums_fit(int64_t R, int64_t V, int N) {
  const GradPlan p = plan_grad(R, V);
  return (int64_t)p.chunks * ((N + 255) / 256) * kWave < ((int64_t)1 << 32) && R < ((int64_t)1 << 30);
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
    const int64_t clear = std::min<int64_t>((V + 1023) / 1024, 256);  // blocks past the rows clear first[] alone
    hipLaunchKernelGGL(embed_rank, dim3((unsigned)std::max((R + 31) / 32, clear)), dim3(kThreads), 0, s, ids, (int)R, V, g.keys[0],
                       g.order[0], g.first);
  } else {
    hipLaunchKernelGGL(embed_clear_ends, dim3((unsigned)std::min<int64_t>((V + 255) / 256, 4096)), dim3(256), 0, s, g.first,
                       V);
    for (int pass = 0; pass < p.passes; ++pass) {
      const uint32_t* from = pass ? g.keys[at] : nullptr;
      const int32_t* rows = pass ? g.order[at] : nullptr;
      const int to = pass ? at ^ 1 : 0;
      const dim3 grid((unsigned)p.sort_blocks);
      hipLaunchKernelGGL(embed_count, grid, dim3(kSortThreads), 0, s, from, ids, (int)R, V, pass * kDigit, g.counts);
      launch_exclusive_scan(g.counts, kBins * p.sort_blocks, g.offs, g.total, g.temp, s);
      hipLaunchKernelGGL(embed_place, grid, dim3(kSortThreads), 0, s, from, rows, ids, (int)R, V, pass * kDigit, g.offs,
                         g.keys[to], g.order[to]);
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
