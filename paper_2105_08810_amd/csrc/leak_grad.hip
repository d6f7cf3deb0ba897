// The adjoint of a leaky integration over time, the recurrence of Proposition 1 by itself:
//
//   y[T-1] = 0,   y[t] = alpha y[t+1] + x[t+1]      for every (sample, column)
//
// If u[t+1] = alpha u[t] + i[t] and x is a loss's gradient by u, y is its gradient by i: from a layer's gated spike
// gradients (entries of its active set) to the gradient of its input currents, and from the gradient of a readout's input
// trace to that of the spikes (wanted at the entries of the layer below). Each side is a dense [T,B,N] tensor or the
// entries of a CSR over the rows (t, b).
//
// Bound: memory, each dense side once. A block owns one sample's 256 columns, a thread a column, and walks time downwards
// in tiles of 32 steps: a dense x is loaded a tile ahead into registers, entries are spread into an LDS tile [step][column]
// (8 threads a row); y goes to memory, or to the same LDS tile, from which the rows' entries are picked.
#include "common.h"

namespace snn {
namespace {

constexpr int kCols = 256;
constexpr int kSteps = 32;
constexpr int kRowLanes = kCols / kSteps;  // threads that share a row's entries

struct Entries {
  const int32_t* row_ptr;
  const int32_t* col;
  const float* g;  // factor of each entry, or NULL
  int64_t cap;
};

constexpr int kEntries = 4;  // of a thread under way

__device__ __forceinline__ int64_t clamped(int32_t e, int64_t cap) { return e < 0 ? 0 : (e > cap ? cap : e); }

template <bool IN, bool OUT>
__global__ __launch_bounds__(kCols) void leak_walk(int T, int B, int N, int slabs, float alpha,
                                                   const float* __restrict__ x, Entries in, float* __restrict__ y,
                                                   Entries out) {
  __shared__ float tile[IN || OUT ? kSteps : 1][kCols];
  const int b = blockIdx.x / slabs;
  const int c0 = (int)(blockIdx.x % slabs) * kCols;
  const int c = threadIdx.x;
  const bool valid = c0 + c < N;
  const size_t step = (size_t)B * N;
  const size_t k = (size_t)b * N + (valid ? c0 + c : c0);
  const int row = threadIdx.x / kRowLanes, lane = threadIdx.x % kRowLanes;
  // step u of tile t1: x[t1 - u] enters y[t1 - u - 1], for t1 - u >= 1
  const auto load = [&](float (&v)[kSteps], int t1) {
#pragma unroll
    for (int u = 0; u < kSteps; ++u) v[u] = x[(size_t)max(t1 - u, 0) * step + k];
  };
  float v[kSteps];
  if (!IN && T > 1) load(v, T - 1);
  // y[T-1] = 0
  if (OUT) {
    const int64_t r = (int64_t)(T - 1) * B + b;
    const int64_t e1 = clamped(out.row_ptr[r + 1], out.cap);
    for (int64_t e = clamped(out.row_ptr[r], out.cap) + c; e < e1; e += kCols)
      if ((unsigned)(out.col[e] - c0) < (unsigned)kCols) y[e] = 0.0f;
  } else if (valid) {
    y[(size_t)(T - 1) * step + k] = 0.0f;
  }
  float d = 0.0f;
  for (int t1 = T - 1; t1 > 0; t1 -= kSteps) {
    if (IN) {
#pragma unroll
      for (int u = 0; u < kSteps; ++u) tile[u][c] = 0.0f;
      __syncthreads();
      if (t1 - row >= 1) {
        const int64_t r = (int64_t)(t1 - row) * B + b;
        const int64_t e1 = clamped(in.row_ptr[r + 1], in.cap);
        for (int64_t e = clamped(in.row_ptr[r], in.cap) + lane; e < e1; e += kEntries * kRowLanes) {
          int j[kEntries];
          float xe[kEntries], ge[kEntries];
#pragma unroll
          for (int q = 0; q < kEntries; ++q) {
            const int64_t at = min(e + q * kRowLanes, e1 - 1);
            j[q] = in.col[at] - c0;
            xe[q] = x[at];
            ge[q] = in.g ? in.g[at] : 1.0f;
          }
#pragma unroll
          for (int q = 0; q < kEntries; ++q)
            if (e + q * kRowLanes < e1 && (unsigned)j[q] < (unsigned)kCols) tile[row][j[q]] = xe[q] * ge[q];
        }
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kSteps; ++u) v[u] = tile[u][c];
      if (OUT) __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int t = t1 - u - 1;
      if (t >= 0) {
        d = fmaf(alpha, d, v[u]);
        if (OUT) tile[u][c] = d;
        else if (valid) y[(size_t)t * step + k] = d;
      }
    }
    if (!IN && t1 - kSteps > 0) load(v, t1 - kSteps);
    if (OUT) {
      __syncthreads();
      if (t1 - row >= 1) {
        const int64_t r = (int64_t)(t1 - row - 1) * B + b;
        const int64_t e1 = clamped(out.row_ptr[r + 1], out.cap);
        for (int64_t e = clamped(out.row_ptr[r], out.cap) + lane; e < e1; e += kEntries * kRowLanes) {
          int j[kEntries];
#pragma unroll
          for (int q = 0; q < kEntries; ++q) j[q] = out.col[min(e + q * kRowLanes, e1 - 1)] - c0;
#pragma unroll
          for (int q = 0; q < kEntries; ++q)
            if (e + q * kRowLanes < e1 && (unsigned)j[q] < (unsigned)kCols) y[e + q * kRowLanes] = tile[row][j[q]];
        }
      }
      __syncthreads();
    } else if (IN) {
      __syncthreads();  // the tile is cleared next
    }
  }
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" snn_status snn_leak_grad(const float* x, const int32_t* in_row_ptr, const int32_t* in_col_idx,
                                    const float* in_g, int64_t in_cap, int T, int B, int N, float alpha, float* y,
                                    const int32_t* out_row_ptr, const int32_t* out_col_idx, int64_t out_cap,
                                    void* stream) {
  if (bad_dim(T) || bad_dim(B) || bad_dim(N) || too_big(T, B, N) || bad_alpha(alpha)) return SNN_ERR_INVALID_ARG;
  if (in_cap < 0 || out_cap < 0) return SNN_ERR_INVALID_ARG;
  if ((in_row_ptr ? in_cap > 0 && (!x || !in_col_idx) : !x || in_col_idx || in_g)) return SNN_ERR_INVALID_ARG;
  if ((out_row_ptr ? out_cap > 0 && (!y || !out_col_idx) : !y || out_col_idx)) return SNN_ERR_INVALID_ARG;
  const int slabs = (N + kCols - 1) / kCols;
  if ((int64_t)B * slabs >= (int64_t)1 << 24) return SNN_ERR_UNSUPPORTED;  // a dispatch counts threads in 32 bits
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Entries in{in_row_ptr, in_col_idx, in_g, in_cap}, out{out_row_ptr, out_col_idx, nullptr, out_cap};
  const dim3 grid((unsigned)(B * slabs));
#define SNN_L(I, O) \
  hipLaunchKernelGGL((leak_walk<I, O>), grid, dim3(kCols), 0, s, T, B, N, slabs, alpha, x, in, y, out)
  if (in_row_ptr && out_row_ptr) SNN_L(true, true);
  else if (in_row_ptr) SNN_L(true, false);
  else if (out_row_ptr) SNN_L(false, true);
  else SNN_L(false, false);
#undef SNN_L
  return launch_status();
}
