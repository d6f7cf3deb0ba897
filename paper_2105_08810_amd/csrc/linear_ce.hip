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

#include "vectors.h"

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
template <class T>
__global__ __launch_bounds__(kWaves * kWave) void ce_pack(const T* __restrict__ x, int64_t ld, int R, int H,
                                                          const int32_t* __restrict__ targets,
                                                          const float* __restrict__ weight,
                                                          const int32_t* __restrict__ pos, float* __restrict__ X,
                                                          int32_t* __restrict__ target, float* __restrict__ w) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R) return;
  const int n = pos[R], p0 = pos[r];
  const bool live = pos[r + 1] > p0;
  const int p = live ? p0 : n + (r - p0);
  for (int i = lane_id(); i < H; i += kWave) X[(size_t)p * H + i] = live ? to_float(x[(int64_t)r * ld + i]) : 0.0f;
  if (lane_id() == 0) {
    target[p] = live ? targets[r] : -1;
    w[p] = !live ? 0.0f : weight ? weight[r] : 1.0f / (float)n;
  }
}

// A piece of W as float32.
template <class T>
__global__ void ce_weights(const T* __restrict__ W, int64_t ld, int H, int n, float* __restrict__ out) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c < n)
    for (int h = blockIdx.y; h < H; h += gridDim.y) out[(size_t)h * n + c] = to_float(W[(int64_t)h * ld + c]);
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

template <class T>
__global__ __launch_bounds__(kWaves * kWave) void ce_dx(const float* __restrict__ dX, int R, int H,
                                                        const int32_t* __restrict__ pos, T* __restrict__ dx, int64_t ld) {
  const int r = blockIdx.x * kWaves + threadIdx.x / kWave;
  if (r >= R) return;
  const int p = pos[r];
  const bool live = pos[r + 1] > p;
  for (int i = lane_id(); i < H; i += kWave) dx[(int64_t)r * ld + i] = from_float<T>(live ? dX[(size_t)p * H + i] : 0.0f);
}

// A piece's columns of dW from its K slices, summed in order.
template <class T>
__global__ void ce_dw(const float* __restrict__ part, int slices, int H, int n, T* __restrict__ dW, int64_t ld) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= n) return;
  for (int h = blockIdx.y; h < H; h += gridDim.y) {
    double s = 0.0;
    for (int k = 0; k < slices; ++k) s += (double)part[((size_t)k * H + h) * n + c];
    dW[(int64_t)h * ld + c] = from_float<T>((float)s);
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
  float *X, *W, *z, *dX, *dW, *w, *top, *sum, *at_target, *lse;
  double* parts;
  size_t bytes;
};

Workspace carve(void* ws, int dtype, int R, int H, int C, bool grad, const Plan& p) {
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
  g.W = c.take<float>(dtype == SNN_F32 ? 0 : (size_t)H * p.width);
  g.z = c.take<float>((size_t)R * p.width);
  g.dX = c.take<float>(grad ? (size_t)R * H : 0);
  g.dW = c.take<float>(grad ? (size_t)p.slices * H * p.width : 0);
  g.bytes = c.off;
  return g;
}

template <class T>
void run(const T* x, int64_t ld_x, const T* W, int64_t ld_w, int R, int H, int C, const int32_t* targets,
         const float* weight, float* loss, float* row_loss, T* dx, int64_t ld_dx, T* dW, int64_t ld_dw, const Plan& p,
         const Workspace& g, hipStream_t s) {
  const dim3 rows((unsigned)((R + kWaves - 1) / kWaves)), waves(kWaves * kWave);
  hipLaunchKernelGGL(ce_live, dim3((unsigned)((R + 255) / 256)), dim3(256), 0, s, targets, weight, R, C, g.live);
  launch_exclusive_scan(g.live, R, g.pos, g.total, g.temp, s);
  hipLaunchKernelGGL(ce_pack<T>, rows, waves, 0, s, x, ld_x, R, H, targets, weight, g.pos, g.X, g.target, g.w);
  const auto logits = [&](int c0, int n, const float*& w, int64_t& ld) {
    if constexpr (sizeof(T) == 4) {
      w = reinterpret_cast<const float*>(W) + c0;
      ld = ld_w;
    } else {
      hipLaunchKernelGGL(ce_weights<T>, dim3((unsigned)((n + 255) / 256), (unsigned)std::min(H, 1024)), dim3(256), 0, s,
                         W + c0, ld_w, H, n, g.W);
      w = g.W;
      ld = n;
    }
  };
  const float* w = nullptr;
  int64_t ld = 0;
  for (int c0 = 0; c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0);
    logits(c0, n, w, ld);
    gemm_split_kr(R, n, H, g.X, H, w, (int)ld, g.z, n, s);
    hipLaunchKernelGGL(ce_sums, rows, waves, 0, s, g.z, R, n, c0, g.target, g.top, g.sum, g.at_target);
  }
  hipLaunchKernelGGL(ce_losses, dim3(kLossParts), dim3(256), 0, s, R, g.pos, g.top, g.sum, g.at_target, g.w, g.lse,
                     row_loss, g.parts);
  hipLaunchKernelGGL(ce_total, dim3(1), dim3(1), 0, s, g.parts, kLossParts, loss);
  if (!dx && !dW) return;
  for (int c0 = 0; c0 < C; c0 += p.width) {
    const int n = std::min(p.width, C - c0);
    if (p.pieces > 1) {
      logits(c0, n, w, ld);
      gemm_split_kr(R, n, H, g.X, H, w, (int)ld, g.z, n, s);
    }
    hipLaunchKernelGGL(ce_dz, rows, waves, 0, s, g.z, R, n, c0, g.target, g.w, g.lse);
    if (dx) gemm_split_kc(R, H, n, g.z, n, w, (int)ld, g.dX, H, s, c0 > 0);
    if (dW) {
      gemm_split_km(H, n, R, g.X, H, g.z, n, g.dW, n, p.slices, (size_t)H * n, s);
      hipLaunchKernelGGL(ce_dw<T>, dim3((unsigned)((n + 255) / 256), (unsigned)std::min(H, 1024)), dim3(256), 0, s, g.dW,
                         p.slices, H, n, dW + c0, ld_dw);
    }
  }
  if (dx) hipLaunchKernelGGL(ce_dx<T>, rows, waves, 0, s, g.dX, R, H, g.pos, dx, ld_dx);
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
  return carve(nullptr, dtype, (int)R, H, C, grad != 0, plan_of((int)R, H, C)).bytes;
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
  const Plan p = plan_of((int)R, H, C);
  const Workspace g = carve(workspace, dtype, (int)R, H, C, dx || dW, p);
  if (workspace_bytes < g.bytes) return SNN_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define SNN_CE(T)                                                                                                 \
  run<T>(static_cast<const T*>(x), ld_x, static_cast<const T*>(W), ld_w, (int)R, H, C, targets, weight, loss,     \
         row_loss, static_cast<T*>(dx), ld_dx, static_cast<T*>(dW), ld_dw, p, g, s)
  if (dtype == SNN_F32) SNN_CE(float);
  else if (dtype == SNN_BF16) SNN_CE(Bf16);
  else SNN_CE(F16);
#undef SNN_CE
  return launch_status();
}
