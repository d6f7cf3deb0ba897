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
// in tiles of 32 steps; entries are spread into, or picked from, an LDS tile [step][column] by 8 threads a row, four each
// under way. Loads and stores retire in order, so whatever a tile reads (a dense x, the rows' pointers, their first entries)
// is asked for before the tile before it is stored, pointers a tile earlier still (500 x 256 x 1024, 2% of it entries, to a
// dense y: 154 us otherwise, 124 so, 4.5 TB/s).
//
// Where no compute unit would have a second block, a block is four groups of 256 threads and takes four tiles at a time: each
// group walks its own from 0, and what the tiles above it leave, alpha^32 a tile, is then added as alpha^(u+1) of it to
// step u. us without and with: 100 x 256 x 200 to entries 11.5, 8.6; 500 x 2 x 1000 77, 31; 500 x 1 x 64 33, 17; 239 x 46 x
// 114 19, 10. With two blocks a compute unit it no longer pays (100 x 512 x 200 to a dense y 13.7, 16.7).
#include "common.h"

namespace snn {
namespace {

constexpr int kCols = 256;
constexpr int kSteps = 32;
constexpr int kRowLanes = kCols / kSteps;  // threads that share a row's entries
constexpr int kGroups = 4;

struct Entries {
  const int32_t* row_ptr;
  const int32_t* col;
  const float* g;  // factor of each entry, or NULL
  int64_t cap;
};

constexpr int kEntries = 4;  // of a thread under way

__device__ __forceinline__ int64_t clamped(int32_t e, int64_t cap) { return e < 0 ? 0 : (e > cap ? cap : e); }

// A thread's share of a row's entries: every kRowLanes-th from `lane` on.
struct Range {
  int64_t e, end;
};

__device__ __forceinline__ Range range_of(const Entries& c, int t, int row_of_step, int B, int lane) {
  Range r{0, 0};
  if (t >= 0) {
    const int64_t at = (int64_t)t * B + row_of_step;
    r.end = clamped(c.row_ptr[at + 1], c.cap);
    r.e = clamped(c.row_ptr[at], c.cap) + lane;
  }
  return r;
}

template <bool IN, bool OUT, int G>  // G groups
__global__ __launch_bounds__(kCols * G) void leak_walk(int T, int B, int N, int slabs, float alpha,
                                                   const float* __restrict__ x, Entries in, float* __restrict__ y,
                                                   Entries out) {
  __shared__ __attribute__((aligned(16))) float tiles[G][IN || OUT ? kSteps : 1][kCols];
  __shared__ float ends[G > 1 ? 2 : 1][G][kCols];  // of two rounds in turn
  const int b = blockIdx.x / slabs;
  const int c0 = (int)(blockIdx.x % slabs) * kCols;
  const int c = threadIdx.x % kCols, group = threadIdx.x / kCols;
  auto& tile = tiles[group];
  const bool valid = c0 + c < N;
  const size_t step = (size_t)B * N;
  const size_t k = (size_t)b * N + (valid ? c0 + c : c0);
  const int row = c / kRowLanes, lane = c % kRowLanes;
  // step u of a tile that begins at t1: x[t1 - u] enters y[t1 - u - 1], for t1 - u >= 1
  float v[kSteps], ahead[IN ? 1 : kSteps];
  const auto load = [&](int t1) {
    if constexpr (!IN) {
#pragma unroll
      for (int u = 0; u < kSteps; ++u) ahead[u] = x[(size_t)max(t1 - u, 0) * step + k];
    }
  };
  struct Some {
    int j[kEntries];
    float v[kEntries];
  };
  // loads of places past a row's entries read its last one (or the first of all) and are left out: no branch between them
  const auto some_in = [&](const Range& r, int64_t e) {
    Some s;
    if (in.cap > 0) {
      float ge[kEntries];
#pragma unroll
      for (int q = 0; q < kEntries; ++q) {
        const int64_t at = max(min(e + q * kRowLanes, r.end - 1), (int64_t)0);
        s.j[q] = in.col[at];
        s.v[q] = x[at];
        ge[q] = 1.0f;
        if (in.g) ge[q] = in.g[at];
      }
#pragma unroll
      for (int q = 0; q < kEntries; ++q) {
        s.j[q] = e + q * kRowLanes < r.end ? s.j[q] - c0 : -1;
        s.v[q] *= ge[q];
      }
    } else {
#pragma unroll
      for (int q = 0; q < kEntries; ++q) s.j[q] = -1;
    }
    return s;
  };
  const auto some_out = [&](const Range& r, int64_t e) {
    Some s;
#pragma unroll
    for (int q = 0; q < kEntries; ++q) s.j[q] = -1;
    if (out.cap > 0) {
      int j[kEntries];
#pragma unroll
      for (int q = 0; q < kEntries; ++q) j[q] = out.col[max(min(e + q * kRowLanes, r.end - 1), (int64_t)0)];
#pragma unroll
      for (int q = 0; q < kEntries; ++q)
        if (e + q * kRowLanes < r.end) s.j[q] = j[q] - c0;
    }
    return s;
  };
  const auto spread = [&](const Some& s) {
#pragma unroll
    for (int q = 0; q < kEntries; ++q)
      if ((unsigned)s.j[q] < (unsigned)kCols) tile[row][s.j[q]] = s.v[q];
  };
  const auto pick = [&](const Some& s, int64_t e) {
#pragma unroll
    for (int q = 0; q < kEntries; ++q)
      if ((unsigned)s.j[q] < (unsigned)kCols) y[e + q * kRowLanes] = tile[row][s.j[q]];
  };
  // y[T-1] = 0
  if (group > 0) {
  } else if (OUT) {
    const int64_t r = (int64_t)(T - 1) * B + b;
    const int64_t e1 = clamped(out.row_ptr[r + 1], out.cap);
    for (int64_t e = clamped(out.row_ptr[r], out.cap) + c; e < e1; e += kCols)
      if ((unsigned)(out.col[e] - c0) < (unsigned)kCols) y[e] = 0.0f;
  } else if (valid) {
    y[(size_t)(T - 1) * step + k] = 0.0f;
  }
  Range ri{0, 0}, ri_next{0, 0}, ro{0, 0}, ro_next{0, 0};
  Some si, so;
  constexpr int kRound = kSteps * G;
  if (T > 1) {
    const int t1 = T - 1 - kSteps * group, t2 = t1 - kRound;
    load(t1);
    if (IN) {
      ri = range_of(in, t1 - row >= 1 ? t1 - row : -1, b, B, lane);
      ri_next = range_of(in, t2 - row >= 1 ? t2 - row : -1, b, B, lane);
      si = some_in(ri, ri.e);
    }
    if (OUT) {
      ro = range_of(out, t1 - 1 - row, b, B, lane);
      ro_next = range_of(out, t2 - 1 - row, b, B, lane);
      so = some_out(ro, ro.e);
    }
  }
  float d = 0.0f, far = alpha;  // alpha^kSteps
#pragma unroll
  for (int k = 1; k < kSteps; k *= 2) far *= far;
  int round = 0;
  for (int t0 = T - 1; t0 > 0; t0 -= kRound, round ^= 1) {
    const int t1 = t0 - kSteps * group, t2 = t1 - kRound, t3 = t2 - kRound;  // where this tile and the next ones begin
    if constexpr (IN) {
      float4* clear = reinterpret_cast<float4*>(&tile[0][0]);
#pragma unroll
      for (int u = 0; u < kSteps / 4; ++u) clear[u * kCols + c] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      __syncthreads();
      spread(si);
      for (int64_t e = ri.e + kEntries * kRowLanes; e < ri.end; e += kEntries * kRowLanes) spread(some_in(ri, e));
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kSteps; ++u) v[u] = tile[u][c];
      if (OUT) __syncthreads();
      ri = ri_next;
      ri_next = range_of(in, t3 - row >= 1 ? t3 - row : -1, b, B, lane);
      si = some_in(ri, ri.e);
    } else {
#pragma unroll
      for (int u = 0; u < kSteps; ++u) v[u] = ahead[u];
      if (t2 > 0) load(t2);
    }
    if constexpr (G > 1) {
      float end = 0.0f;
#pragma unroll
      for (int u = 0; u < kSteps; ++u) v[u] = end = fmaf(alpha, end, v[u]);
      ends[round][group][c] = end;
      __syncthreads();
      float from = d;  // where this tile begins, and the next round
#pragma unroll
      for (int q = 0; q < G; ++q) {
        if (q == group) from = d;
        d = fmaf(far, d, ends[round][q][c]);
      }
#pragma unroll
      for (int u = 0; u < kSteps; ++u) {
        from *= alpha;
        v[u] += from;
      }
    } else {
#pragma unroll
      for (int u = 0; u < kSteps; ++u) v[u] = d = fmaf(alpha, d, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int t = t1 - u - 1;
      if (t >= 0) {
        if (OUT) tile[u][c] = v[u];
        else if (valid) __builtin_nontemporal_store(v[u], y + (size_t)t * step + k);
      }
    }
    if constexpr (OUT) {
      __syncthreads();
      const Range r = ro;
      const Some s = so;
      ro = ro_next;
      ro_next = range_of(out, t3 - 1 - row, b, B, lane);
      so = some_out(ro, ro.e);
      pick(s, r.e);
      for (int64_t e = r.e + kEntries * kRowLanes; e < r.end; e += kEntries * kRowLanes) pick(some_out(r, e), e);
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
  const bool groups = T > kSteps + 1 && B * slabs <= cu_count();
#define SNN_L(I, O)                                                                                                    \
  if (groups)                                                                                                          \
    hipLaunchKernelGGL((leak_walk<I, O, kGroups>), grid, dim3(kCols * kGroups), 0, s, T, B, N, slabs, alpha, x, in, y, out); \
  else                                                                                                                 \
    hipLaunchKernelGGL((leak_walk<I, O, 1>), grid, dim3(kCols), 0, s, T, B, N, slabs, alpha, x, in, y, out)
  if (in_row_ptr && out_row_ptr) {
    SNN_L(true, true);
  } else if (in_row_ptr) {
    SNN_L(true, false);
  } else if (out_row_ptr) {
    SNN_L(false, true);
  } else {
    SNN_L(false, false);
  }
#undef SNN_L
  return launch_status();
}
