// Softmax cross entropy of linear logits against one target a row, with the gradients of both factors.
//
//   z = x W  [R,C],  lse_r = log sum_c exp z_rc,  L_r = lse_r - z_r,target,  loss = sum_r w_r L_r
//   dz_rc = w_r (exp(z_rc - lse_r) - [c = target_r]),  dx = dz W^T,  dW = x^T dz
//
// The logits of all classes are never in memory together: the classes are taken in pieces, each piece's logits are formed,
// give their share of every row's sum of exponentials and are dropped; with the rows' lse known a piece's logits are formed
// again (unless there is one piece) and turned into its columns of dz, from which its share of dx and its columns of dW
// follow. Rows without a target (or of weight 0) are taken out first: the others lie packed, in their order, before rows of
// zeros, so that nothing of the former is read again.
#include <algorithm>

#include "gemm16.h"

namespace snn {
namespace {

using namespace vectors;

constexpr int kMaxRows = 1 << 24;
constexpr int kMaxHidden = 1 << 16;
constexpr int64_t kPiece = (int64_t)1 << 27;  // logits of a piece
constexpr int kWaves = 4;                     // rows of a block in the kernels with a wavefront a row

__device__ __forceinline__ bool has_target(int32_t t, int C) { return t >= 0 && t < C; }

// live[r]: whether row r takes part.
__global__ void ce_live(const int32_t* __restrict__ targets, const float* __restrict__ weight, int R, int C,
                        int32_t* __restrict__ live) {
  const int r = blockIdx.x * blockDim.x + threadIdx.x;
  if (r < R) live[r] = has_target(targets[r], C) && (!weight || weight[r] != 0.0f);
}

// Rows to their packed places: pos[r] = live rows before r, pos[R] = their number. Row r of x as float32, a row of zeros
// for one that takes no part (these lie behind the others).
__global__ __launch_bounds__(kWaves * kWave) void ce_pack(const float* __restrict__ x, int64_t ld, int R, int H,
                                                          const int32_t* __restrict__ targets,
                                                          const float* __restrict__ weight,
                                                          const int32_t* __restrict__ pos, float* __restrict__ X,
                                                          int32_t* __restrict__ target, float* __restrict__ w) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R) return;
  const int n = pos[R], p0 = pos[r];
  const bool live = pos[r + 1] > p0;
  const int p = live ? p0 : n + (r - p0);
  for (int i = lane_id(); i < H; i += kWave) X[(size_t)p * H + i] = live ? x[(int64_t)r * ld + i] : 0.0f;
  if (lane_id() == 0) {
    target[p] = live ? targets[r] : -1;
    w[p] = !live ? 0.0f : weight ? weight[r] : 1.0f / (float)n;
  }
}

// A piece's share of every row's largest logit and sum of exponentials, and the target's logit.
__global__ __launch_bounds__(kWaves * kWave) void ce_sums(const float* __restrict__ z, int R, int n, int c0,
                                                          const int32_t* __restrict__ target, float* __restrict__ top,
                                                          float* __restrict__ sum, float* __restrict__ at_target) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R) return;
  const float* row = z + (size_t)r * n;
  const int l = lane_id();
  float m = -INFINITY;
  for (int i = l; i < n; i += kWave) m = fmaxf(m, row[i]);  // a NaN is left to the sum
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
  const float ref = m > -INFINITY ? m : 0.0f;
  float s = 0.0f;
  for (int i = l; i < n; i += kWave) s += expf(row[i] - ref);
  s = wave_sum(s);
  if (l == 0) {
    if (c0 > 0) {
      const float m0 = top[r], s0 = sum[r];
      const float both = fmaxf(m0, m), from = both > -INFINITY ? both : 0.0f;
      s = s0 * expf(m0 - from) + s * expf(m - from);
      m = both;
    }
    top[r] = m;
    sum[r] = s;
    const int t = target[r] - c0;
    if (target[r] >= 0 && t >= 0 && t < n) at_target[r] = row[t];
  }
}

// Each row's log-sum-exp and loss; loss parts of a block in float64. Rows that take no part have loss 0.
__global__ __launch_bounds__(256) void ce_losses(int R, const int32_t* __restrict__ pos, const float* __restrict__ top,
                                                 const float* __restrict__ sum, const float* __restrict__ at_target,
                                                 const float* __restrict__ w, float* __restrict__ lse,
                                                 float* __restrict__ row_loss, double* __restrict__ parts) {
  double s = 0.0;
  for (int r = blockIdx.x * 256 + threadIdx.x; r < R; r += gridDim.x * 256) {
    const int p = pos[r];
    float loss = 0.0f;
    if (pos[r + 1] > p) {
      const float log_sum = logf(sum[p]);
      lse[p] = top[p] + log_sum;
      loss = (top[p] - at_target[p]) + log_sum;
      s += (double)w[p] * (double)loss;
    }
    if (row_loss) row_loss[r] = loss;
  }
  __shared__ double all[256];
  all[threadIdx.x] = s;
  __syncthreads();
  for (int off = 128; off > 0; off >>= 1) {
    if ((int)threadIdx.x < off) all[threadIdx.x] += all[threadIdx.x + off];
    __syncthreads();
  }
  if (threadIdx.x == 0) parts[blockIdx.x] = all[0];
}

__global__ void ce_total(const double* __restrict__ parts, int n, float* __restrict__ loss) {
  double s = 0.0;
  for (int k = 0; k < n; ++k) s += parts[k];
  *loss = (float)s;
}

// z to dz in place; rows behind the live ones to 0.
__global__ __launch_bounds__(kWaves * kWave) void ce_dz(float* __restrict__ z, int R, int n, int c0,
                                                        const int32_t* __restrict__ target, const float* __restrict__ w,
                                                        const float* __restrict__ lse) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R) return;
  float* row = z + (size_t)r * n;
  const int t = target[r];
  const float k = w[r], ref = t >= 0 ? lse[r] : 0.0f;
  for (int i = lane_id(); i < n; i += kWave)
    row[i] = t >= 0 ? k * (expf(row[i] - ref) - (c0 + i == t ? 1.0f : 0.0f)) : 0.0f;
}

__global__ __launch_bounds__(kWaves * kWave) void ce_dx(const float* __restrict__ dX, int R, int H,
                                                        const int32_t* __restrict__ pos, float* __restrict__ dx,
                                                        int64_t ld) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R) return;
  const int p = pos[r];
  const bool live = pos[r + 1] > p;
  for (int i = lane_id(); i < H; i += kWave) dx[(int64_t)r * ld + i] = live ? dX[(size_t)p * H + i] : 0.0f;
}

// A piece's columns of dW from its K slices, summed in order.
__global__ void ce_dw(const float* __restrict__ part, int slices, int H, int n, float* __restrict__ dW, int64_t ld) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= n) return;
  for (int h = blockIdx.y; h < H; h += gridDim.y) {
    double s = 0.0;
    for (int k = 0; k < slices; ++k) s += (double)part[((size_t)k * H + h) * n + c];
    dW[(int64_t)h * ld + c] = (float)s;
  }
}

struct Plan {
  int width, pieces, slices;  // classes of a piece; K slices of dW
};

Plan plan_of(int R, int H, int C) {
  Plan p;
  p.width = (int)std::min<int64_t>(C, std::max<int64_t>(256, kPiece / R / 128 * 128));
  p.pieces = (C + p.width - 1) / p.width;
  p.slices = plan_splits(H, p.width, R, 88e12).splits;
  return p;
}

constexpr int kLossParts = 256;

struct Workspace {
  int32_t *live, *pos, *temp, *target;
  int64_t* total;
  float *X, *z, *dX, *dW, *w, *top, *sum, *at_target, *lse;
  double* parts;
  size_t bytes;
};

Workspace carve(void* ws, int R, int H, int C, bool grad, const Plan& p) {
  Carve c(ws);
  Workspace g;
  g.live = c.take<int32_t>(R);
  g.pos = c.take<int32_t>((size_t)R + 1);
  g.temp = c.take<int32_t>(scan_temp_elems(R));
  g.total = c.take<int64_t>(1);
  g.target = c.take<int32_t>(R);
  g.w = c.take<float>(R);
  g.top = c.take<float>(R);
  g.sum = c.take<float>(R);
  g.at_target = c.take<float>(R);
  g.lse = c.take<float>(R);
  g.parts = c.take<double>(kLossParts);
  g.X = c.take<float>((size_t)R * H);
  g.z = c.take<float>((size_t)R * p.width);
  g.dX = c.take<float>(grad ? (size_t)R * H : 0);
  g.dW = c.take<float>(grad ? (size_t)p.slices * H * p.width : 0);
  g.bytes = c.off;
  return g;
}

void run(const float* x, int64_t ld_x, const float* W, int64_t ld_w, int R, int H, int C, const int32_t* targets,
         const float* weight, float* loss, float* row_loss, float* dx, int64_t ld_dx, float* dW, int64_t ld_dw,
         const Plan& p, const Workspace& g, hipStream_t s) {
  const dim3 rows((unsigned)((R + kWaves - 1) / kWaves)), waves(kWaves * kWave);
  const int ld = (int)ld_w;
  hipLaunchKernelGGL(ce_live, dim3((unsigned)((R + 255) / 256)), dim3(256), 0, s, targets, weight, R, C, g.live);
  launch_exclusive_scan(g.live, R, g.pos, g.total, g.temp, s);
  hipLaunchKernelGGL(ce_pack, rows, waves, 0, s, x, ld_x, R, H, targets, weight, g.pos, g.X, g.target, g.w);
  for (int c0 = 0; c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0);
    gemm_split_kr(R, n, H, g.X, H, W + c0, ld, g.z, n, s);
    hipLaunchKernelGGL(ce_sums, rows, waves, 0, s, g.z, R, n, c0, g.target, g.top, g.sum, g.at_target);
  }
  hipLaunchKernelGGL(ce_losses, dim3(kLossParts), dim3(256), 0, s, R, g.pos, g.top, g.sum, g.at_target, g.w, g.lse,
                     row_loss, g.parts);
  hipLaunchKernelGGL(ce_total, dim3(1), dim3(1), 0, s, g.parts, kLossParts, loss);
  if (!dx && !dW) return;
  for (int c0 = 0; c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0);
    if (p.pieces > 1) gemm_split_kr(R, n, H, g.X, H, W + c0, ld, g.z, n, s);
    hipLaunchKernelGGL(ce_dz, rows, waves, 0, s, g.z, R, n, c0, g.target, g.w, g.lse);
    if (dx) gemm_split_kc(R, H, n, g.z, n, W + c0, ld, g.dX, H, s, c0 > 0);
    if (dW) {
      gemm_split_km(H, n, R, g.X, H, g.z, n, g.dW, n, p.slices, (size_t)H * n, s);
      hipLaunchKernelGGL(ce_dw, dim3((unsigned)((n + 255) / 256), (unsigned)std::min(H, 1024)), dim3(256), 0, s, g.dW,
                         p.slices, H, n, dW + c0, ld_dw);
    }
  }
  if (dx) hipLaunchKernelGGL(ce_dx, rows, waves, 0, s, g.dX, R, H, g.pos, dx, ld_dx);
}

// ------------------------------------------------------------------ 16-bit operands

// x and dz of 16-bit calls are multiplied in that type. dz enters as ref times (w / ref)(softmax - onehot), ref the
// largest weight, so that one weight for all rows costs no rounding; float16's numbers are also raised by 2^15, since
// those below 2^-14 have few bits. Both come off the float32 sums.
template <class T>
constexpr float kRaise = std::is_same<T, F16>::value ? 32768.0f : 1.0f;

constexpr int kTile = gemm16::kTile;
constexpr int kPart = 128;  // classes of a partial sum of exponentials: a wavefront's

__global__ __launch_bounds__(1024) void ce_ref(const float* __restrict__ weight, const int32_t* __restrict__ pos, int R,
                                               float* __restrict__ ref) {
  __shared__ float top[1024 / kWave];
  float m = 0.0f;
  if (weight) {
    for (int r = threadIdx.x; r < R; r += 1024)
      if (pos[r + 1] > pos[r]) m = fmaxf(m, fabsf(weight[r]));
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
    if (lane_id() == 0) top[threadIdx.x / kWave] = m;
    __syncthreads();
    for (int k = 0; k < 1024 / kWave; ++k) m = fmaxf(m, top[k]);
  } else if (pos[R] > 0) {
    m = 1.0f / (float)pos[R];
  }
  if (threadIdx.x == 0) *ref = m;
}

// ce_pack in the type itself: rows of Hp, zeros behind H and in the rows behind the live ones up to a whole tile.
template <class T>
__global__ __launch_bounds__(kWaves * kWave) void ce_pack16(const T* __restrict__ x, int64_t ld, int R, int Rp, int H,
                                                            int Hp, const int32_t* __restrict__ targets,
                                                            const float* __restrict__ weight,
                                                            const int32_t* __restrict__ pos, T* __restrict__ X,
                                                            int32_t* __restrict__ target, float* __restrict__ w) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= Rp) return;
  const int n = pos[R], p0 = r < R ? pos[r] : n;
  const bool live = r < R && pos[r + 1] > p0;
  const int p = live ? p0 : n + (r - p0);
  if (p >= (n + kTile - 1) / kTile * kTile) return;
  for (int i = lane_id() * 8; i < Hp; i += kWave * 8) {
    T v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = T{0};
    if (live) {
      const T* s = x + (int64_t)r * ld + i;
      if (i + 8 <= H) {
        __builtin_memcpy(v, s, 16);
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (i + u < H) v[u] = s[u];
      }
    }
    *reinterpret_cast<uint4*>(X + (size_t)p * Hp + i) = __builtin_bit_cast(uint4, v);
  }
  if (lane_id() == 0) {
    target[p] = live ? targets[r] : -1;
    w[p] = !live ? 0.0f : weight ? weight[r] : 1.0f / (float)n;
  }
}

// n columns of W in lines of `width`, zeros behind them and in the lines from H on.
template <class T>
__global__ __launch_bounds__(256) void ce_weights16(const T* __restrict__ W, int64_t ld, int H, int n, int width,
                                                    T* __restrict__ out) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8, h = blockIdx.y;
  if (c >= width) return;
  T v[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) v[u] = T{0};
  if (h < H) {
    const T* s = W + (int64_t)h * ld + c;
    if (c + 8 <= n) {
      __builtin_memcpy(v, s, 16);
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c + u < n) v[u] = s[u];
    }
  }
  *reinterpret_cast<uint4*>(out + (size_t)h * width + c) = __builtin_bit_cast(uint4, v);
}

// Logits of a tile of classes (m) and rows (n). GRAD false: every row's largest logit and sum of exponentials over the
// 128 classes of a wavefront, to part[class / 128][row], and the target's logit. GRAD true: dz to G[row][class].
template <class T, bool GRAD>
__global__ __launch_bounds__(gemm16::kThreads, 2) void ce_logits16(
    const T* __restrict__ W, int64_t ldw, const T* __restrict__ X, int Hp, int stages, int c0, int C, int R, int Rp,
    int tiles_m, int tiles_n, const int32_t* __restrict__ pos, const int32_t* __restrict__ target,
    float2* __restrict__ part, float* __restrict__ at_target, const float* __restrict__ lse, const float* __restrict__ w,
    const float* __restrict__ ref, T* __restrict__ G, int64_t ldg) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const gemm16::Tiles t = gemm16::tile_of(tiles_m, tiles_n, 1);
  if (!t.ok || t.n * kTile >= pos[R]) return;
  gemm16::Product<T, true, false> z;
  z.run(W, ldw, t.m * kTile, X, Hp, t.n * kTile, 0, stages, smem);
  const int l = lane_id(), g = l / 16;
  const int m0 = t.m * kTile + z.m_of_wave();
  const int first = c0 + m0;  // class of the wavefront's first m
  const int n0 = t.n * kTile + z.n_of_wave() + l % 16;
  constexpr float kLog2e = 1.44269504088896340736f;
  const bool ragged = first + kPart > C;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int n = n0 + 16 * b;
    const int at = target[n] - first;  // the target among this wavefront's classes
    const bool here = target[n] >= 0 && (unsigned)at < (unsigned)kPart;
    if (ragged) {
#pragma unroll
      for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (first + 16 * a + 4 * g + v >= C) z.acc[a][b][v] = -INFINITY;
    }
    if constexpr (!GRAD) {
      if (here && (at / 4) % 4 == g) {
#pragma unroll
        for (int a = 0; a < 8; ++a)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (at == 16 * a + 4 * g + v) at_target[n] = z.acc[a][b][v];
      }
      float m = -INFINITY;
#pragma unroll
      for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, z.acc[a][b][v]);
      m = fmaxf(m, __shfl_xor(m, 16, kWave));
      m = fmaxf(m, __shfl_xor(m, 32, kWave));
      const float from = m > -INFINITY ? m : 0.0f;
      float s = 0.0f;
#pragma unroll
      for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int v = 0; v < 4; ++v) s += __builtin_amdgcn_exp2f((z.acc[a][b][v] - from) * kLog2e);
      s += __shfl_xor(s, 16, kWave);
      s += __shfl_xor(s, 32, kWave);
      if (g == 0) part[(size_t)(first / kPart) * Rp + n] = make_float2(m, s);
    } else {
      const bool live = target[n] >= 0;
      const float k = live ? w[n] / *ref * kRaise<T> : 0.0f;
      const float from = live ? lse[n] : 0.0f;
#pragma unroll
      for (int a = 0; a < 8; ++a) {
        T d[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float p = __builtin_amdgcn_exp2f((z.acc[a][b][v] - from) * kLog2e);
          d[v] = from_float<T>(live ? k * (p - (here && at == 16 * a + 4 * g + v ? 1.0f : 0.0f)) : 0.0f);
        }
        *reinterpret_cast<uint2*>(G + (size_t)n * ldg + m0 + 16 * a + 4 * g) = __builtin_bit_cast(uint2, d);
      }
    }
  }
}

// top and sum of every live row from the parts of its classes. A block takes 32 rows, 32 threads share a row's parts.
__global__ __launch_bounds__(1024) void ce_join16(const float2* __restrict__ part, int parts, int R, int Rp,
                                                  const int32_t* __restrict__ pos, float* __restrict__ top,
                                                  float* __restrict__ sum) {
  __shared__ float2 all[32][33];
  const int x = threadIdx.x % 32, y = threadIdx.x / 32;
  const int r = blockIdx.x * 32 + x;
  if (blockIdx.x * 32 >= pos[R]) return;
  float m = -INFINITY, s = 0.0f;
  const auto add = [&](float m1, float s1) {
    const float both = fmaxf(m, m1), from = both > -INFINITY ? both : 0.0f;
    s = s * expf(m - from) + s1 * expf(m1 - from);
    m = both;
  };
#pragma unroll 4
  for (int p = y; p < parts; p += 32) {
    const float2 q = part[(size_t)p * Rp + r];
    add(q.x, q.y);
  }
  all[y][x] = make_float2(m, s);
  __syncthreads();
  if (y == 0) {
    for (int k = 1; k < 32; ++k) add(all[k][x].x, all[k][x].y);
    if (r < pos[R]) {
      top[r] = m;
      sum[r] = s;
    }
  }
}

// A K slice's dx of a piece: dX[slice][row][h] (+)= sum over its classes of G W.
template <class T>
__global__ __launch_bounds__(gemm16::kThreads, 2) void ce_dx16(const T* __restrict__ W, int64_t ldw, const T* __restrict__ G,
                                                               int64_t ldg, int stages, int per, int R, int Rp, int Hp,
                                                               int tiles_m, int tiles_n, int slices,
                                                               const int32_t* __restrict__ pos, int accumulate,
                                                               float* __restrict__ dX) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const gemm16::Tiles t = gemm16::tile_of(tiles_m, tiles_n, slices);
  if (!t.ok || t.n * kTile >= pos[R]) return;
  gemm16::Product<T, false, false> d;
  const int from = t.slice * per;
  d.run(W, ldw, t.m * kTile, G, ldg, t.n * kTile, (int64_t)from * gemm16::kK, max(0, min(per, stages - from)), smem);
  const int l = lane_id();
  float* out = dX + ((size_t)t.slice * Rp + t.n * kTile + d.n_of_wave() + l % 16) * Hp + t.m * kTile + d.m_of_wave() + l / 16 * 4;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int a = 0; a < 8; ++a) {
      gemm16::f32x4* o = reinterpret_cast<gemm16::f32x4*>(out + (size_t)16 * b * Hp + 16 * a);
      *o = accumulate ? *o + d.acc[a][b] : d.acc[a][b];
    }
}

template <class T>
__global__ __launch_bounds__(kWaves * kWave) void ce_dx_out16(const float* __restrict__ dX, int slices, int R, int Rp, int H,
                                                              int Hp, const int32_t* __restrict__ pos,
                                                              const float* __restrict__ ref, T* __restrict__ dx,
                                                              int64_t ld) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R) return;
  const int p = pos[r];
  const bool live = pos[r + 1] > p;
  const float k = *ref / kRaise<T>;
  for (int i = lane_id() * 4; i < H; i += kWave * 4) {
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (live)
      for (int q = 0; q < slices; ++q) {
        const float4 v = *reinterpret_cast<const float4*>(dX + ((size_t)q * Rp + p) * Hp + i);
        s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
      }
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] *= k;
    store_in<T, 4>(dx + (int64_t)r * ld, i, H, s);
  }
}

// dW of a piece's n columns: the tile itself with one slice, else its share to part[slice][h][width].
template <class T>
__global__ __launch_bounds__(gemm16::kThreads, 2) void ce_dw16(const T* __restrict__ G, int64_t ldg, const T* __restrict__ X,
                                                               int Hp, int R, int H, int n, int width, int tiles_m,
                                                               int tiles_n, int slices, const int32_t* __restrict__ pos,
                                                               const float* __restrict__ ref, T* __restrict__ dW,
                                                               int64_t ld, float* __restrict__ part) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const gemm16::Tiles t = gemm16::tile_of(tiles_m, tiles_n, slices);
  if (!t.ok) return;
  const int stages = (pos[R] + gemm16::kK - 1) / gemm16::kK;
  const int per = (stages + slices - 1) / slices, from = t.slice * per;
  gemm16::Product<T, true, true> d;
  d.run(G, ldg, t.m * kTile, X, Hp, t.n * kTile, (int64_t)from * gemm16::kK, max(0, min(per, stages - from)), smem);
  const int l = lane_id();
  const int m0 = t.m * kTile + d.m_of_wave() + l / 16 * 4, n0 = t.n * kTile + d.n_of_wave() + l % 16;
  const float k = *ref / kRaise<T>;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int h = n0 + 16 * b;
    if (h >= H) continue;
#pragma unroll
    for (int a = 0; a < 8; ++a) {
      const int c = m0 + 16 * a;
      if (slices > 1) {
        *reinterpret_cast<gemm16::f32x4*>(part + ((size_t)t.slice * H + h) * width + c) = d.acc[a][b];
      } else if (c < n) {
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = d.acc[a][b][u] * k;
        store_in<T, 4>(dW + (int64_t)h * ld, c, n, v);
      }
    }
  }
}

template <class T>
__global__ void ce_dw_out16(const float* __restrict__ part, int slices, int H, int n, int width,
                            const float* __restrict__ ref, T* __restrict__ dW, int64_t ld) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= n) return;
  const float k = *ref / kRaise<T>;
  for (int h = blockIdx.y; h < H; h += gridDim.y) {
    float s = 0.0f;
    for (int q = 0; q < slices; ++q) s += part[((size_t)q * H + h) * width + c];
    dW[(int64_t)h * ld + c] = from_float<T>(s * k);
  }
}

constexpr int64_t kPiece16 = (int64_t)1 << 28;  // dz values of a piece

// K slices of a product of `tiles` tiles and `stages` stages: a block a compute unit and round, a stage about a
// microsecond, a slice's share of a tile (written and read) a quarter of one.
int slices_of(int64_t tiles, int stages) {
  const int64_t cus = cu_count();
  int best = 1;
  double least = 0.0;
  for (int s = 1; s <= 64 && (s == 1 || s * 4 <= stages); ++s) {
    const double rounds = (double)((tiles * s + cus - 1) / cus);
    const double t = rounds * ((stages + s - 1) / s + 3) + (s > 1 ? 0.25 * rounds + 0.1 * s * tiles / cus : 0.0);
    if (s == 1 || t < least) {
      best = s;
      least = t;
    }
  }
  return best;
}

int padded(int n, int to) { return (n + to - 1) / to * to; }

struct Plan16 {
  int Rp, Hp, width, pieces, dx_slices, dw_slices;
  size_t parts;  // partial sums of exponentials a row
};

Plan16 plan16_of(int R, int H, int C) {
  Plan16 p;
  p.Rp = padded(R, kTile);
  p.Hp = padded(H, kTile);
  const int most = (int)std::min<int64_t>(padded(C, kTile), std::max<int64_t>(kTile, kPiece16 / p.Rp / kTile * kTile));
  p.pieces = (C + most - 1) / most;
  p.width = padded((C + p.pieces - 1) / p.pieces, kTile);
  p.pieces = (C + p.width - 1) / p.width;
  p.dx_slices = slices_of((int64_t)(p.Hp / kTile) * (p.Rp / kTile), p.width / gemm16::kK);
  p.dw_slices = slices_of((int64_t)(p.width / kTile) * (p.Hp / kTile), p.Rp / gemm16::kK);
  p.parts = (size_t)p.pieces * p.width / kPart;
  return p;
}

struct Workspace16 {
  int32_t *live, *pos, *temp, *target;
  int64_t* total;
  uint16_t *X, *W, *G;
  float *w, *top, *sum, *at_target, *lse, *ref, *dX, *dW;
  float2* part;
  double* parts;
  size_t bytes;
};

// W is always given room, so that the size does not depend on its address.
Workspace16 carve16(void* ws, int R, int H, int C, bool grad, const Plan16& p) {
  Carve c(ws);
  Workspace16 g;
  g.live = c.take<int32_t>(R);
  g.pos = c.take<int32_t>((size_t)R + 1);
  g.temp = c.take<int32_t>(scan_temp_elems(R));
  g.total = c.take<int64_t>(1);
  g.target = c.take<int32_t>(p.Rp);
  g.w = c.take<float>(p.Rp);
  g.top = c.take<float>(p.Rp);
  g.sum = c.take<float>(p.Rp);
  g.at_target = c.take<float>(p.Rp);
  g.lse = c.take<float>(p.Rp);
  g.ref = c.take<float>(1);
  g.parts = c.take<double>(kLossParts);
  g.part = c.take<float2>(p.parts * p.Rp);
  g.X = c.take<uint16_t>((size_t)p.Rp * p.Hp);
  g.W = c.take<uint16_t>((size_t)p.Hp * p.width);
  g.G = c.take<uint16_t>(grad ? (size_t)p.Rp * p.width : 0);
  g.dX = c.take<float>(grad ? (size_t)p.dx_slices * p.Rp * p.Hp : 0);
  g.dW = c.take<float>(grad && p.dw_slices > 1 ? (size_t)p.dw_slices * H * p.width : 0);
  g.bytes = c.off;
  return g;
}

template <class T>
void run16(const T* x, int64_t ld_x, const T* W, int64_t ld_w, int R, int H, int C, const int32_t* targets,
           const float* weight, float* loss, float* row_loss, T* dx, int64_t ld_dx, T* dW, int64_t ld_dw,
           const Plan16& p, const Workspace16& g, hipStream_t s) {
  T *X = reinterpret_cast<T*>(g.X), *Wp = reinterpret_cast<T*>(g.W), *G = reinterpret_cast<T*>(g.G);
  const dim3 waves(kWaves * kWave), block(gemm16::kThreads);
  const auto rows_of = [](int n) { return dim3((unsigned)((n + kWaves - 1) / kWaves)); };
  for (const void* f : {(const void*)ce_logits16<T, false>, (const void*)ce_logits16<T, true>, (const void*)ce_dx16<T>,
                        (const void*)ce_dw16<T>})
    ensure_dynamic_lds(f, gemm16::kLds);
  hipLaunchKernelGGL(ce_live, dim3((unsigned)((R + 255) / 256)), dim3(256), 0, s, targets, weight, R, C, g.live);
  launch_exclusive_scan(g.live, R, g.pos, g.total, g.temp, s);
  hipLaunchKernelGGL(ce_pack16<T>, rows_of(p.Rp), waves, 0, s, x, ld_x, R, p.Rp, H, p.Hp, targets, weight, g.pos, X,
                     g.target, g.w);
  // W in place where its rows are whole tiles at 16-byte addresses
  const bool whole = H % kTile == 0 && C % kTile == 0 && ld_w % 8 == 0 && ld_w < (1 << 22) &&
                     reinterpret_cast<uintptr_t>(W) % 16 == 0;
  const T* w = nullptr;
  int64_t ldw = 0;
  const auto weights = [&](int c0, int n) {
    if (whole) {
      w = W + c0;
      ldw = ld_w;
    } else {
      hipLaunchKernelGGL(ce_weights16<T>, dim3((unsigned)((p.width / 8 + 255) / 256), (unsigned)p.Hp), dim3(256), 0, s,
                         W + c0, ld_w, H, n, p.width, Wp);
      w = Wp;
      ldw = p.width;
    }
  };
  const int tiles_n = p.Rp / kTile, tiles_h = p.Hp / kTile, stages_h = padded(H, gemm16::kK) / gemm16::kK;
  for (int c0 = 0; c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0), tiles_m = (n + kTile - 1) / kTile;
    weights(c0, n);
    hipLaunchKernelGGL((ce_logits16<T, false>), dim3(gemm16::grid_of(tiles_m, tiles_n, 1)), block, gemm16::kLds, s, w, ldw,
                       X, p.Hp, stages_h, c0, C, R, p.Rp, tiles_m, tiles_n, g.pos, g.target, g.part, g.at_target, nullptr,
                       nullptr, nullptr, (T*)nullptr, 0);
  }
  hipLaunchKernelGGL(ce_join16, dim3((unsigned)(p.Rp / 32)), dim3(1024), 0, s, g.part, (int)((padded(C, kTile)) / kPart), R,
                     p.Rp, g.pos, g.top, g.sum);
  hipLaunchKernelGGL(ce_losses, dim3(kLossParts), dim3(256), 0, s, R, g.pos, g.top, g.sum, g.at_target, g.w, g.lse,
                     row_loss, g.parts);
  hipLaunchKernelGGL(ce_total, dim3(1), dim3(1), 0, s, g.parts, kLossParts, loss);
  if (!dx && !dW) return;
  hipLaunchKernelGGL(ce_ref, dim3(1), dim3(1024), 0, s, weight, g.pos, R, g.ref);
  for (int c0 = 0; c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0), tiles_m = (n + kTile - 1) / kTile;
    if (p.pieces > 1) weights(c0, n);
    hipLaunchKernelGGL((ce_logits16<T, true>), dim3(gemm16::grid_of(tiles_m, tiles_n, 1)), block, gemm16::kLds, s, w, ldw,
                       X, p.Hp, stages_h, c0, C, R, p.Rp, tiles_m, tiles_n, g.pos, g.target, nullptr, nullptr, g.lse, g.w,
                       g.ref, G, (int64_t)p.width);
    if (dx) {
      const int stages = tiles_m * (kTile / gemm16::kK), per = (stages + p.dx_slices - 1) / p.dx_slices;
      hipLaunchKernelGGL(ce_dx16<T>, dim3(gemm16::grid_of(tiles_h, tiles_n, p.dx_slices)), block, gemm16::kLds, s, w, ldw,
                         G, (int64_t)p.width, stages, per, R, p.Rp, p.Hp, tiles_h, tiles_n, p.dx_slices, g.pos, c0 > 0,
                         g.dX);
    }
    if (dW) {
      hipLaunchKernelGGL(ce_dw16<T>, dim3(gemm16::grid_of(tiles_m, tiles_h, p.dw_slices)), block, gemm16::kLds, s, G,
                         (int64_t)p.width, X, p.Hp, R, H, n, p.width, tiles_m, tiles_h, p.dw_slices, g.pos, g.ref, dW + c0,
                         ld_dw, g.dW);
      if (p.dw_slices > 1)
        hipLaunchKernelGGL(ce_dw_out16<T>, dim3((unsigned)((n + 255) / 256), (unsigned)std::min(H, 1024)), dim3(256), 0, s,
                           g.dW, p.dw_slices, H, n, p.width, g.ref, dW + c0, ld_dw);
    }
  }
  if (dx)
    hipLaunchKernelGGL(ce_dx_out16<T>, rows_of(R), waves, 0, s, g.dX, p.dx_slices, R, p.Rp, H, p.Hp, g.pos, g.ref, dx,
                       ld_dx);
}

snn_status check_sizes(int dtype, int64_t R, int H, int C) {
  if (!dtype_size(dtype) || R <= 0 || H <= 0 || C <= 0) return SNN_ERR_INVALID_ARG;
  if (R > kMaxRows || H > kMaxHidden || C > rows::kMaxClasses) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" size_t snn_linear_ce_workspace(int dtype, int64_t R, int H, int C, int grad) {
  if (check_sizes(dtype, R, H, C) != SNN_OK) return 0;
  if (dtype == SNN_F32) return carve(nullptr, (int)R, H, C, grad != 0, plan_of((int)R, H, C)).bytes;
  return carve16(nullptr, (int)R, H, C, grad != 0, plan16_of((int)R, H, C)).bytes;
}

extern "C" snn_status snn_linear_ce(const void* x, const void* W, int dtype, int64_t R, int H, int C, int64_t ld_x,
                                    int64_t ld_w, const int32_t* targets, const float* weight, float* loss,
                                    float* row_loss, void* dx, int64_t ld_dx, void* dW, int64_t ld_dw, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  if (!x || !W || !targets || !loss || !workspace) return SNN_ERR_INVALID_ARG;
  if (const snn_status st = check_sizes(dtype, R, H, C)) return st;
  if (ld_x < H || ld_w < C || (dx && ld_dx < H) || (dW && ld_dw < C)) return SNN_ERR_INVALID_ARG;
  if (misaligned(x, dtype) || misaligned(W, dtype) || misaligned(dx, dtype) || misaligned(dW, dtype))
    return SNN_ERR_INVALID_ARG;
  if (ld_w > INT32_MAX) return SNN_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == SNN_F32) {
    const Plan p = plan_of((int)R, H, C);
    const Workspace g = carve(workspace, (int)R, H, C, dx || dW, p);
    if (workspace_bytes < g.bytes) return SNN_ERR_INVALID_ARG;
    run(static_cast<const float*>(x), ld_x, static_cast<const float*>(W), ld_w, (int)R, H, C, targets, weight, loss,
        row_loss, static_cast<float*>(dx), ld_dx, static_cast<float*>(dW), ld_dw, p, g, s);
    return launch_status();
  }
  const Plan16 p = plan16_of((int)R, H, C);
  const Workspace16 g = carve16(workspace, (int)R, H, C, dx || dW, p);
  if (workspace_bytes < g.bytes) return SNN_ERR_INVALID_ARG;
#define SNN_CE(T)                                                                                                   \
  run16<T>(static_cast<const T*>(x), ld_x, static_cast<const T*>(W), ld_w, (int)R, H, C, targets, weight, loss,     \
           row_loss, static_cast<T*>(dx), ld_dx, static_cast<T*>(dW), ld_dw, p, g, s)
  if (dtype == SNN_BF16) SNN_CE(Bf16);
  else SNN_CE(F16);
#undef SNN_CE
  return launch_status();
}
