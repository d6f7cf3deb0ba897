// Layer norm of rows and its backward pass.
//
//   y = h gamma + beta,  h = (x - mean) rstd,  mean = sum x / N,  rstd = 1 / sqrt(sum (x - mean)^2 / N + eps)
//   a = dy gamma,  dx = rstd (a - mean(a) - h mean(a h)),  dgamma = sum over rows of dy h,  dbeta = sum over rows of dy
//
// Bound: memory. A row is read once into the registers of its lanes (16 lanes, a wavefront, or a block of 256 to 1024
// threads by its width), the squares are summed about the mean that is already known, and the results are written from
// the registers. The backward pass reads x and dy once; each group of lanes walks many rows and keeps its columns' shares
// of dgamma and dbeta in registers, a block adds its groups' shares and writes one partial row, and norm_columns adds the
// partial rows in a fixed order in float64. Rows beyond a block's registers are read once more for every sum. 128000 x 1024
// float32: forward 186 us (5.6 TB/s), backward 288 (5.5); 8192 x 2048 bfloat16 14 and 27, x 2050 21 and 33.
#include <algorithm>

#include "vectors.h"

namespace snn {
namespace {

using namespace vectors;

constexpr int kMaxWidth = 1 << 20;

// Sum over a group of L lanes (16 or 64) or a block of L threads, the same in every lane; red holds a value a wavefront.
template <int L>
__device__ __forceinline__ float group_sum(float v, float* red) {
#pragma unroll
  for (int off = (L < kWave ? L : kWave) / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  if constexpr (L > kWave) {
    const int w = threadIdx.x / kWave;
    __syncthreads();  // the sums before these have been read
    if (lane_id() == 0) red[w] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < L / kWave; ++k) v += red[k];
  }
  return v;
}

template <int L>
__device__ __forceinline__ void group_sum2(float& a, float& b, float2* red) {
#pragma unroll
  for (int off = (L < kWave ? L : kWave) / 2; off > 0; off >>= 1) {
    a += __shfl_xor(a, off, kWave);
    b += __shfl_xor(b, off, kWave);
  }
  if constexpr (L > kWave) {
    __syncthreads();
    if (lane_id() == 0) red[threadIdx.x / kWave] = make_float2(a, b);
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int k = 0; k < L / kWave; ++k) {
      a += red[k].x;
      b += red[k].y;
    }
  }
}

// What the launches share. E elements a vector, Q vectors a lane, L lanes a row, B threads a block.
template <int L>
constexpr int kBlock = L > 256 ? L : 256;

// Whether a row may be shorter than a vector: only the narrowest rows are.
template <int L>
constexpr bool kShort = L == 16;

template <class TX, class TY>
constexpr int kE = sizeof(TX) == 4 || sizeof(TY) == 4 ? 4 : 8;

// A row's values stay in registers as they were read: the compiler would keep their float32 forms as well, twice the
// registers in 16 bits, and so half the rows under way.
template <class T, int E, int Q>
__device__ __forceinline__ void kept(Raw<T, E> (&raw)[Q]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int u = 0; u < E / 2; ++u) asm volatile("" : "+v"(raw[q].w[u]));
  }
}

// Whether a row may end in its lanes' vector q, or before it: shape_of takes as few vectors as there can be.
template <int L, int Q>
__device__ __forceinline__ constexpr bool ragged(int q) {
  return q == Q - 1 || (L == 1024 && Q == 4 && q >= 2);
}

// Whether a wavefront holds anything of its vector q: the last vectors of most of a block's wavefronts may lie past the row.
template <int L, int E>
__device__ __forceinline__ bool any_of(int q, int N) {
  return L <= kWave || (q * L + __builtin_amdgcn_readfirstlane((int)threadIdx.x & ~(kWave - 1))) * E < N;
}

template <class TX, class TY, int L, int Q>
__global__ __launch_bounds__(kBlock<L>) void norm_forward(const TX* __restrict__ x, int64_t ld_x, int64_t R, int N,
                                                          const float* __restrict__ gamma,
                                                          const float* __restrict__ beta, float eps, TY* __restrict__ y,
                                                          int64_t ld_y, float* __restrict__ mean,
                                                          float* __restrict__ rstd) {
  constexpr int E = kE<TX, TY>;
  constexpr int G = kBlock<L> / L;  // rows of a block at a time
  __shared__ float red[kBlock<L> / kWave];
  const int l = threadIdx.x % L;
  float g[Q][E], b[Q][E];
  bool own[Q][E];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int i = (q * L + l) * E;
    if (gamma) span_load<float, E, kShort<L>>(gamma, i, N).to(g[q]);
    if (beta) span_load<float, E, kShort<L>>(beta, i, N).to(b[q]);
#pragma unroll
    for (int u = 0; u < E; ++u) {
      if (!gamma) g[q][u] = 1.0f;
      if (!beta) b[q][u] = -0.0f;  // h + -0 is h
    }
    span_own<E, kShort<L>>(i, N, own[q]);
  }
  // with L > kWave a block is one row: all its threads or none
  const int64_t step = (int64_t)gridDim.x * G;
  int64_t r = (int64_t)blockIdx.x * G + threadIdx.x / L;
  if (r >= R) return;
  Raw<TX, E> raw[Q], next[Q];
  const auto fetch = [&](Raw<TX, E> (&to)[Q], int64_t row) {
#pragma unroll
    for (int q = 0; q < Q; ++q) to[q] = span_load<TX, E, kShort<L>>(x + row * ld_x, (q * L + l) * E, N);
  };
  fetch(raw, r);
  for (; r < R; r += step) {
    if (r + step < R) fetch(next, r + step);
    float s = 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (!any_of<L, E>(q, N)) continue;
      float v[E];
      raw[q].to(v);
#pragma unroll
      for (int u = 0; u < E; ++u) s += !ragged<L, Q>(q) || own[q][u] ? v[u] : 0.0f;
    }
    const float m = group_sum<L>(s, red) / (float)N;
    kept(raw);
    float d2 = 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (!any_of<L, E>(q, N)) continue;
      float v[E];
      raw[q].to(v);
#pragma unroll
      for (int u = 0; u < E; ++u) {
        const float d = !ragged<L, Q>(q) || own[q][u] ? v[u] - m : 0.0f;
        d2 = fmaf(d, d, d2);
      }
    }
    const float k = 1.0f / sqrtf(group_sum<L>(d2, red) / (float)N + eps);
    kept(raw);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (!any_of<L, E>(q, N)) continue;
      float v[E];
      raw[q].to(v);
#pragma unroll
      for (int u = 0; u < E; ++u) v[u] = fmaf((v[u] - m) * k, g[q][u], b[q][u]);
      span_store<TY, E, true, kShort<L>>(y + r * ld_y, (q * L + l) * E, N, v);
    }
    if (l == 0) {
      if (mean) mean[r] = m;
      if (rstd) rstd[r] = k;
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) raw[q] = next[q];
  }
}

// dx, and a block's shares of dgamma and dbeta to part[block][2][N] (part NULL: none are wanted).
template <class TX, class TY, int L, int Q>
__global__ __launch_bounds__(kBlock<L>) void norm_backward(const TY* __restrict__ dy, int64_t ld_dy,
                                                           const TX* __restrict__ x, int64_t ld_x, int64_t R, int N,
                                                           const float* __restrict__ gamma,
                                                           const float* __restrict__ mean,
                                                           const float* __restrict__ rstd, TX* __restrict__ dx,
                                                           int64_t ld_dx, float* __restrict__ part) {
  constexpr int E = kE<TX, TY>;
  constexpr int G = kBlock<L> / L;
  __shared__ float2 red[kBlock<L> / kWave];
  extern __shared__ float share[];  // [G][L * E] of one vector of the groups' shares
  const int g = threadIdx.x / L, l = threadIdx.x % L;
  float dg[Q][E], db[Q][E], w[Q][E];
  bool own[Q][E];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int i = (q * L + l) * E;
    if (gamma) span_load<float, E, kShort<L>>(gamma, i, N).to(w[q]);
#pragma unroll
    for (int u = 0; u < E; ++u) {
      dg[q][u] = db[q][u] = 0.0f;
      if (!gamma) w[q][u] = 1.0f;
    }
    span_own<E, kShort<L>>(i, N, own[q]);
  }
  // with L > kWave a block is one row: all its threads or none
  const int64_t step = (int64_t)gridDim.x * G;
  Raw<TX, E> rx[Q], nx[Q];
  Raw<TY, E> ry[Q], ny[Q];
  float m = 0.0f, k = 0.0f, nm = 0.0f, nk = 0.0f;
  const auto fetch = [&](int64_t row) {
    nm = mean[row];
    nk = rstd[row];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      nx[q] = span_load<TX, E, kShort<L>>(x + row * ld_x, (q * L + l) * E, N);
      ny[q] = span_load<TY, E, kShort<L>>(dy + row * ld_dy, (q * L + l) * E, N);
    }
  };
  int64_t r = (int64_t)blockIdx.x * G + g;
  if (r < R) fetch(r);
  for (; r < R; r += step) {
    m = nm;
    k = nk;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      rx[q] = nx[q];
      ry[q] = ny[q];
    }
    if (r + step < R) fetch(r + step);
    float s = 0.0f, sh = 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (!any_of<L, E>(q, N)) continue;
      float h[E], a[E];
      rx[q].to(h);
      ry[q].to(a);
#pragma unroll
      for (int u = 0; u < E; ++u) {
        h[u] = (h[u] - m) * k;
        if (part) {
          dg[q][u] = fmaf(a[u], h[u], dg[q][u]);
          db[q][u] += a[u];
        }
        // others' elements enter neither sum (the dgamma, dbeta and dx that the lane makes of them are not stored); as 0
        // times one that is infinite they would
        const bool mine = !ragged<L, Q>(q) || own[q][u];
        a[u] *= w[q][u];
        s += mine ? a[u] : 0.0f;
        sh = mine ? fmaf(a[u], h[u], sh) : sh;
      }
    }
    if (dx) {
      group_sum2<L>(s, sh, red);
      s /= (float)N;
      sh /= (float)N;
      kept(rx);
      kept(ry);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (!any_of<L, E>(q, N)) continue;
        float h[E], a[E];
        rx[q].to(h);
        ry[q].to(a);
#pragma unroll
        for (int u = 0; u < E; ++u) a[u] = k * (a[u] * w[q][u] - s - (h[u] - m) * k * sh);
        span_store<TX, E, true, kShort<L>>(dx + r * ld_dx, (q * L + l) * E, N, a);
      }
    }
  }
  if (!part) return;
  float* mine = part + (size_t)blockIdx.x * 2 * N;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int i = (q * L + l) * E;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float t[E];
#pragma unroll
      for (int u = 0; u < E; ++u) t[u] = which ? db[q][u] : dg[q][u];
      if constexpr (G > 1) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < E; ++u) share[(g * L + l) * E + u] = t[u];
        __syncthreads();
        if (g == 0) {
          for (int o = 1; o < G; ++o)
#pragma unroll
            for (int u = 0; u < E; ++u) t[u] += share[(o * L + l) * E + u];
        }
      }
      if (g == 0) span_store<float, E, false, kShort<L>>(mine + (size_t)which * N, i, N, t);
    }
  }
}

// dgamma and dbeta: the sums of the parts' columns, in float64. A block takes 32 columns, each half of its wavefronts every
// kStreams-th part, 16 of them under way together.
constexpr int kColumns = 32, kStreams = 32;
__global__ __launch_bounds__(kColumns * kStreams) void norm_columns(const float* __restrict__ part, int n, int N,
                                                                    float* __restrict__ dgamma,
                                                                    float* __restrict__ dbeta) {
  __shared__ double sum[kStreams][kColumns];
  const int w = threadIdx.x / kColumns, l = threadIdx.x % kColumns;
  const int64_t j = (int64_t)blockIdx.x * kColumns + l;  // of 2 N: dgamma, then dbeta
  double s = 0.0;
  if (j < 2 * (int64_t)N) {
#pragma unroll 16
    for (int p = w; p < n; p += kStreams) s += (double)part[(size_t)p * 2 * N + j];
  }
  sum[w][l] = s;
  __syncthreads();
  if (w == 0 && j < 2 * (int64_t)N) {
    for (int o = 1; o < kStreams; ++o) s += sum[o][l];
    float* out = j < N ? dgamma : dbeta;
    if (out) out[j < N ? j : j - N] = (float)s;
  }
}

// Rows beyond a block's registers: a block walks its row three times.
constexpr int kLong = 1024;
template <class TX, class TY>
__global__ __launch_bounds__(kLong) void norm_forward_long(const TX* __restrict__ x, int64_t ld_x, int N,
                                                           const float* __restrict__ gamma,
                                                           const float* __restrict__ beta, float eps, TY* __restrict__ y,
                                                           int64_t ld_y, float* __restrict__ mean,
                                                           float* __restrict__ rstd) {
  constexpr int E = kE<TX, TY>;
  __shared__ float red[kLong / kWave];
  const int64_t r = blockIdx.x;
  const TX* row = x + r * ld_x;
  float s = 0.0f;
  for (int i = threadIdx.x * E; i < N; i += kLong * E) {
    float v[E];
    load_in<TX, E>(row, i, N, v);
#pragma unroll
    for (int u = 0; u < E; ++u) s += v[u];
  }
  const float m = group_sum<kLong>(s, red) / (float)N;
  float d2 = 0.0f;
  for (int i = threadIdx.x * E; i < N; i += kLong * E) {
    float v[E];
    load_in<TX, E>(row, i, N, v);
#pragma unroll
    for (int u = 0; u < E; ++u)
      if (i + u < N) d2 = fmaf(v[u] - m, v[u] - m, d2);
  }
  const float k = 1.0f / sqrtf(group_sum<kLong>(d2, red) / (float)N + eps);
  for (int i = threadIdx.x * E; i < N; i += kLong * E) {
    float v[E], g[E], b[E];
    load_in<TX, E>(row, i, N, v);
    if (gamma) load_in<float, E>(gamma, i, N, g);
    if (beta) load_in<float, E>(beta, i, N, b);
#pragma unroll
    for (int u = 0; u < E; ++u) {
      const float h = (v[u] - m) * k;
      v[u] = gamma ? (beta ? fmaf(h, g[u], b[u]) : h * g[u]) : (beta ? h + b[u] : h);
    }
    store_in<TY, E>(y + r * ld_y, i, N, v);
  }
  if (threadIdx.x == 0) {
    if (mean) mean[r] = m;
    if (rstd) rstd[r] = k;
  }
}

template <class TX, class TY>
__global__ __launch_bounds__(kLong) void norm_backward_long(const TY* __restrict__ dy, int64_t ld_dy,
                                                            const TX* __restrict__ x, int64_t ld_x, int N,
                                                            const float* __restrict__ gamma,
                                                            const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, TX* __restrict__ dx,
                                                            int64_t ld_dx) {
  constexpr int E = kE<TX, TY>;
  __shared__ float red[kLong / kWave];
  const int64_t r = blockIdx.x;
  const float m = mean[r], k = rstd[r];
  float s = 0.0f, sh = 0.0f;
  for (int pass = 0; pass < 2; ++pass) {
    for (int i = threadIdx.x * E; i < N; i += kLong * E) {
      float h[E], a[E], w[E];
      load_in<TX, E>(x + r * ld_x, i, N, h);
      load_in<TY, E>(dy + r * ld_dy, i, N, a);
      if (gamma) load_in<float, E>(gamma, i, N, w);
#pragma unroll
      for (int u = 0; u < E; ++u) {
        h[u] = (h[u] - m) * k;
        if (gamma) a[u] *= w[u];
        if (pass == 0) {
          s += a[u];
          sh = fmaf(a[u], h[u], sh);
        } else {
          a[u] = k * (a[u] - s - h[u] * sh);
        }
      }
      if (pass) store_in<TX, E>(dx + r * ld_dx, i, N, a);
    }
    if (pass == 0) {
      s = group_sum<kLong>(s, red) / (float)N;
      sh = group_sum<kLong>(sh, red) / (float)N;
    }
  }
}

// Long rows' shares of dgamma and dbeta: a thread a column, part p the rows p, p + gridDim.y, ...
template <class TX, class TY>
__global__ __launch_bounds__(256) void norm_columns_long(const TY* __restrict__ dy, int64_t ld_dy,
                                                         const TX* __restrict__ x, int64_t ld_x, int64_t R, int N,
                                                         const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, float* __restrict__ part) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= N) return;
  float dg = 0.0f, db = 0.0f;
  for (int64_t r = blockIdx.y; r < R; r += gridDim.y) {
    const float d = to_float(dy[r * ld_dy + j]);
    dg = fmaf(d, (to_float(x[r * ld_x + j]) - mean[r]) * rstd[r], dg);
    db += d;
  }
  part[(size_t)blockIdx.y * 2 * N + j] = dg;
  part[(size_t)blockIdx.y * 2 * N + N + j] = db;
}

// How a row of N is spread: lanes and vectors a lane. L 0: beyond a block's registers. A wavefront alone needs no barrier
// between its sums; with more than 20 values a lane (gamma, beta and their gradients are held beside the row's) too few
// wavefronts fit, and a block takes the row: of 256 threads up to 384 vectors (8192 x 2050 bfloat16, 257 vectors, backward:
// two each of 256 threads 33 us, one each of 384 41), of 512 and 1024 beyond.
struct Shape {
  int L, Q;
};
Shape shape_of(int N, int E) {
  const int v = (N + E - 1) / E;
  if (v <= 16) return {16, 1};
  for (int q = 1; q * E <= 20; ++q)
    if (v <= 64 * q) return {64, q};
  if (v <= 256) return {256, 1};
  if (v <= 384) return {256, 2};
  if (v <= 512) return {512, 1};
  if (v <= 1024) return {512, 2};
  if (v <= 2048) return {1024, 2};
  if (v <= 4096) return {1024, 4};
  return {0, 0};
}

int vector_of(int x_dtype, int y_dtype) { return x_dtype == SNN_F32 || y_dtype == SNN_F32 ? 4 : 8; }

// Blocks of the backward pass, each with a partial row: as many as are resident, that none is left for a second turn and
// the partial rows are few. A wavefront's rows of several vectors, and the blocks of 512 and 1024 threads, leave room for
// two blocks a compute unit (backward of 64000 x 2048 float32 with 1024 blocks 329 us, with 512 277; backward
// of 8192 x 1024 bfloat16 22.8 and 18.3), the others for four (100000 x 100 float32 34 us, with 512 45; 8192 x 2050
// bfloat16 32 and 37, 256000 x 300 130 and 164).
int parts_of(int64_t R, int N, int E) {
  const Shape sh = shape_of(N, E);
  if (!sh.L) return (int)std::min<int64_t>(R, 64);
  const int G = sh.L >= 256 ? 1 : 256 / sh.L;
  const int64_t blocks = (R + G - 1) / G;
  return (int)std::min<int64_t>(blocks, sh.L >= 512 || (sh.L == 64 && sh.Q > 1) ? 512 : 1024);
}

constexpr int64_t kLaunchRows = (int64_t)1 << 21;  // a dispatch counts threads in 32 bits

template <class TX, class TY>
void forward(const void* x, int64_t ld_x, int64_t R, int N, const float* gamma, const float* beta, float eps, void* y,
             int64_t ld_y, float* mean, float* rstd, hipStream_t s) {
  const Shape sh = shape_of(N, kE<TX, TY>);
  for (int64_t r = 0; r < R; r += kLaunchRows) {
    const int64_t n = std::min(kLaunchRows, R - r);
    const TX* px = static_cast<const TX*>(x) + r * ld_x;
    TY* py = static_cast<TY*>(y) + r * ld_y;
    float *pm = mean ? mean + r : nullptr, *pr = rstd ? rstd + r : nullptr;
    const int64_t most = (int64_t)8 * cu_count();  // blocks; beyond, a block walks several rows with one gamma and beta
#define SNN_N(L_, Q_)                                                                                            \
  hipLaunchKernelGGL((norm_forward<TX, TY, L_, Q_>), dim3((unsigned)std::min(most, (n + kBlock<L_> / L_ - 1) / (kBlock<L_> / L_))), \
                     dim3(kBlock<L_>), 0, s, px, ld_x, n, N, gamma, beta, eps, py, ld_y, pm, pr)
    if (sh.L == 16) SNN_N(16, 1);
    else if (sh.L == 64 && sh.Q == 1) SNN_N(64, 1);
    else if (sh.L == 64 && sh.Q == 2) SNN_N(64, 2);
    else if (sh.L == 64 && sh.Q == 3) SNN_N(64, 3);
    else if (sh.L == 64 && sh.Q == 4) SNN_N(64, 4);
    else if (sh.L == 64) SNN_N(64, 5);
    else if (sh.L == 256 && sh.Q == 1) SNN_N(256, 1);
    else if (sh.L == 256) SNN_N(256, 2);
    else if (sh.L == 512 && sh.Q == 1) SNN_N(512, 1);
    else if (sh.L == 512) SNN_N(512, 2);
    else if (sh.L == 1024 && sh.Q == 2) SNN_N(1024, 2);
    else if (sh.L == 1024) SNN_N(1024, 4);
    else
      hipLaunchKernelGGL((norm_forward_long<TX, TY>), dim3((unsigned)n), dim3(kLong), 0, s, px, ld_x, N, gamma, beta, eps,
                         py, ld_y, pm, pr);
#undef SNN_N
  }
}

template <class TX, class TY>
void backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, int64_t R, int N, const float* gamma,
              const float* mean, const float* rstd, void* dx, int64_t ld_dx, float* part, int parts, hipStream_t s) {
  constexpr int E = kE<TX, TY>;
  const Shape sh = shape_of(N, E);
  const TY* pdy = static_cast<const TY*>(dy);
  const TX* px = static_cast<const TX*>(x);
  TX* pdx = static_cast<TX*>(dx);
#define SNN_N(L_, Q_)                                                                                                \
  hipLaunchKernelGGL((norm_backward<TX, TY, L_, Q_>), dim3((unsigned)parts), dim3(kBlock<L_>),                        \
                     L_ < 256 ? 256 * E * sizeof(float) : 0, s, pdy, ld_dy, px, ld_x, R, N, gamma, mean, rstd, pdx,  \
                     ld_dx, part)
  if (sh.L == 16) SNN_N(16, 1);
  else if (sh.L == 64 && sh.Q == 1) SNN_N(64, 1);
  else if (sh.L == 64 && sh.Q == 2) SNN_N(64, 2);
  else if (sh.L == 64 && sh.Q == 3) SNN_N(64, 3);
  else if (sh.L == 64 && sh.Q == 4) SNN_N(64, 4);
  else if (sh.L == 64) SNN_N(64, 5);
  else if (sh.L == 256 && sh.Q == 1) SNN_N(256, 1);
  else if (sh.L == 256) SNN_N(256, 2);
  else if (sh.L == 512 && sh.Q == 1) SNN_N(512, 1);
  else if (sh.L == 512) SNN_N(512, 2);
  else if (sh.L == 1024 && sh.Q == 2) SNN_N(1024, 2);
  else if (sh.L == 1024) SNN_N(1024, 4);
  else {
    for (int64_t r = 0; pdx && r < R; r += kLaunchRows)
      hipLaunchKernelGGL((norm_backward_long<TX, TY>), dim3((unsigned)std::min(kLaunchRows, R - r)), dim3(kLong), 0, s,
                         pdy + r * ld_dy, ld_dy, px + r * ld_x, ld_x, N, gamma, mean + r, rstd + r, pdx + r * ld_dx, ld_dx);
    if (part)
      hipLaunchKernelGGL((norm_columns_long<TX, TY>), dim3((unsigned)((N + 255) / 256), (unsigned)parts), dim3(256), 0, s,
                         pdy, ld_dy, px, ld_x, R, N, mean, rstd, part);
  }
#undef SNN_N
}

snn_status check_sizes(int x_dtype, int y_dtype, int64_t R, int N) {
  if (!dtype_size(x_dtype) || !dtype_size(y_dtype) || R <= 0 || N <= 0) return SNN_ERR_INVALID_ARG;
  if (R > INT32_MAX || N > kMaxWidth) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

// The pairs of types: F(TX, TY).
#define SNN_PAIRS(F)                                                                          \
  if (x_dtype == SNN_F32 && y_dtype == SNN_F32) F(float, float);                              \
  else if (x_dtype == SNN_F32 && y_dtype == SNN_BF16) F(float, Bf16);                         \
  else if (x_dtype == SNN_F32) F(float, F16);                                                 \
  else if (x_dtype == SNN_BF16 && y_dtype == SNN_F32) F(Bf16, float);                         \
  else if (x_dtype == SNN_BF16 && y_dtype == SNN_BF16) F(Bf16, Bf16);                         \
  else if (x_dtype == SNN_BF16) F(Bf16, F16);                                                 \
  else if (y_dtype == SNN_F32) F(F16, float);                                                 \
  else if (y_dtype == SNN_BF16) F(F16, Bf16);                                                 \
  else F(F16, F16)

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" snn_status snn_layer_norm(const void* x, int x_dtype, int64_t R, int N, int64_t ld_x, const float* gamma,
                                     const float* beta, float eps, void* y, int y_dtype, int64_t ld_y, float* mean,
                                     float* rstd, void* stream) {
  if (!x || !y) return SNN_ERR_INVALID_ARG;
  if (const snn_status st = check_sizes(x_dtype, y_dtype, R, N)) return st;
  if (ld_x < N || ld_y < N || !(eps >= 0.0f) || isinf(eps)) return SNN_ERR_INVALID_ARG;
  if (misaligned(x, x_dtype) || misaligned(y, y_dtype)) return SNN_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define SNN_F(TX, TY) forward<TX, TY>(x, ld_x, R, N, gamma, beta, eps, y, ld_y, mean, rstd, s)
  SNN_PAIRS(SNN_F);
#undef SNN_F
  return launch_status();
}

extern "C" size_t snn_layer_norm_grad_workspace(int x_dtype, int y_dtype, int64_t R, int N) {
  if (check_sizes(x_dtype, y_dtype, R, N) != SNN_OK) return 0;
  return align256((size_t)parts_of(R, N, vector_of(x_dtype, y_dtype)) * 2 * N * sizeof(float));
}

extern "C" snn_status snn_layer_norm_grad(const void* dy, int y_dtype, int64_t ld_dy, const void* x, int x_dtype,
                                          int64_t ld_x, int64_t R, int N, const float* gamma, const float* mean,
                                          const float* rstd, void* dx, int64_t ld_dx, float* dgamma, float* dbeta,
                                          void* workspace, size_t workspace_bytes, void* stream) {
  if (!dy || !x || !mean || !rstd || (!dx && !dgamma && !dbeta)) return SNN_ERR_INVALID_ARG;
  if (const snn_status st = check_sizes(x_dtype, y_dtype, R, N)) return st;
  if (ld_dy < N || ld_x < N || (dx && ld_dx < N)) return SNN_ERR_INVALID_ARG;
  if (misaligned(dy, y_dtype) || misaligned(x, x_dtype) || misaligned(dx, x_dtype)) return SNN_ERR_INVALID_ARG;
  const bool columns = dgamma || dbeta;
  if (columns && (!workspace || workspace_bytes < snn_layer_norm_grad_workspace(x_dtype, y_dtype, R, N)))
    return SNN_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  float* part = columns ? static_cast<float*>(workspace) : nullptr;
  const int parts = parts_of(R, N, vector_of(x_dtype, y_dtype));
#define SNN_F(TX, TY) backward<TX, TY>(dy, ld_dy, x, ld_x, R, N, gamma, mean, rstd, dx, ld_dx, part, parts, s)
  SNN_PAIRS(SNN_F);
#undef SNN_F
  if (columns)
    hipLaunchKernelGGL(norm_columns, dim3((unsigned)((2 * (int64_t)N + kColumns - 1) / kColumns)),
                       dim3(kColumns * kStreams), 0, s, part, parts, N, dgamma, dbeta);
  return launch_status();
}
