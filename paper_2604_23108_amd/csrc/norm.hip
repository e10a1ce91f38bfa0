// Root-mean-square norm with the residual's addition for gfx950, forward and backward.
//   forward   h = x + r,  rstd = (mean h^2 + eps)^-1/2,  y = h rstd w
//   backward  n = h rstd, g = w dy, dx = ds + rstd (g - n mean(g n)),  dw = sum over rows of dy n
// Bound by memory: a row is read once into registers (8 elements per thread and piece), its one or two sums
// are folded across the threads that share it, and it is written from the registers.
#include "block.h"

namespace mohge {

// Sums of the wave's lanes in every lane
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
  return v;
}

// TPR threads share a row; a thread has up to NV pieces of it, TPR pieces apart.
template <bool BF16, int TPR, int NV, bool Q8>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) rmsnorm_kernel(
    const void* x, const void* residual, const float* __restrict__ weight, void* sum_out, void* y, float* y_scale,
    float* rstd_out, int T, int pieces, float inv_d, float eps) {
  constexpr int kRows = TPR < 256 ? 256 / TPR : 1;
  constexpr int kWaves = TPR / 64;
  const int t = threadIdx.x % TPR, lane = threadIdx.x & 63;
  const int row = blockIdx.x * kRows + threadIdx.x / TPR;
  if (row >= T) return;                                   // (whole waves, and whole rows)
  const long long base = (long long)row * pieces;
  float h[NV][8], w[NV][8];
  float ss = 0.f, top = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int p = t + i * TPR;
    if (p < pieces) {
      Piece<BF16> a;
      a.load(x, base + p);
      a.get(h[i]);
      if (residual) {
        float r[8];
        a.load(residual, base + p);
        a.get(r);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] += r[j];
      }
      Piece<false> b;
      b.load(weight, p);
      b.get(w[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ss = fmaf(h[i][j], h[i][j], ss);
        if constexpr (Q8) top = fmaxf(top, fabsf(h[i][j] * w[i][j]));
      }
    }
  }
  ss = wave_sum(ss);
  if constexpr (Q8) top = wave_max(top);
  if constexpr (kWaves > 1) {
    __shared__ float red[2 * kWaves];
    if (lane == 0) {
      red[threadIdx.x >> 6] = ss;
      if constexpr (Q8) red[kWaves + (threadIdx.x >> 6)] = top;
    }
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) ss += red[i];
    if constexpr (Q8) {
#pragma unroll
      for (int i = 0; i < kWaves; ++i) top = fmaxf(top, red[kWaves + i]);
    }
  }
  const float rstd = rsqrtf(ss * inv_d + eps);
  float scale = 1.f, inv_scale = 1.f;
  if constexpr (Q8) {
    scale = e4m3_scale(top * rstd);
    inv_scale = 1.f / scale;
    if (t == 0) y_scale[row] = scale;
  }
  if (rstd_out && t == 0) rstd_out[row] = rstd;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int p = t + i * TPR;
    if (p < pieces) {
      Piece<BF16> o;
      if (sum_out) {
        o.set(h[i]);
        o.store(sum_out, base + p);
      }
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = h[i][j] * rstd * w[i][j];
      if constexpr (Q8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= inv_scale;
        static_cast<uint2*>(y)[base + p] = to_e4m3x8(v);
      } else {
        o.set(v);
        o.store(y, base + p);
      }
    }
  }
}

template <bool BF16, bool Q8>
static hipError_t launch_norm(const mohge_norm_config& c, const void* x, const void* residual, const float* weight,
                              void* sum_out, void* y, float* y_scale, float* rstd, hipStream_t s) {
  const int pieces = c.d / 8;
  auto go = [&](auto kern, int tpr) {
    const int rows = tpr < 256 ? 256 / tpr : 1;
    hipLaunchKernelGGL(kern, dim3((unsigned)((c.T + rows - 1) / rows)), dim3(tpr < 256 ? 256 : tpr), 0, s, x, residual,
                       weight, sum_out, y, y_scale, rstd, c.T, pieces, 1.f / c.d, c.eps);
  };
  if (pieces <= 64) go(rmsnorm_kernel<BF16, 64, 1, Q8>, 64);
  else if (pieces <= 128) go(rmsnorm_kernel<BF16, 64, 2, Q8>, 64);
  else if (pieces <= 256) go(rmsnorm_kernel<BF16, 256, 1, Q8>, 256);
  else if (pieces <= 512) go(rmsnorm_kernel<BF16, 256, 2, Q8>, 256);
  else if (pieces <= 1024) go(rmsnorm_kernel<BF16, 512, 2, Q8>, 512);
  else if (pieces <= 2048) go(rmsnorm_kernel<BF16, 1024, 2, Q8>, 1024);
  else go(rmsnorm_kernel<BF16, 1024, 4, Q8>, 1024);
  return hipGetLastError();
}

hipError_t launch_rmsnorm(const mohge_norm_config& c, const void* x, const void* residual, const float* weight,
                          void* sum_out, void* y, float* y_scale, float* rstd, hipStream_t s) {
  const bool bf = c.dtype == MOHGE_BF16, q8 = c.y_dtype == MOHGE_E4M3;
  return bf ? q8 ? launch_norm<true, true>(c, x, residual, weight, sum_out, y, y_scale, rstd, s)
                 : launch_norm<true, false>(c, x, residual, weight, sum_out, y, y_scale, rstd, s)
            : q8 ? launch_norm<false, true>(c, x, residual, weight, sum_out, y, y_scale, rstd, s)
                 : launch_norm<false, false>(c, x, residual, weight, sum_out, y, y_scale, rstd, s);
}

// ---- backward -----------------------------------------------------------------------------------
// A workgroup walks rows, gridDim.x apart, and keeps the part of dw of its rows in registers; its sums
// go to the workspace, and a second kernel adds them in the order of the workgroups.
constexpr int kBwdGroups = 512;

template <bool BF16, int TPR, int NV>
__global__ void __launch_bounds__(TPR) rmsnorm_bwd_kernel(const void* dy, const void* __restrict__ h,
                                                          const float* __restrict__ weight,
                                                          const float* __restrict__ rstd, const void* dsum, void* dx,
                                                          float* __restrict__ partial, int T, int pieces, float inv_d) {
  constexpr int kWaves = TPR / 64;
  const int t = threadIdx.x, lane = t & 63;
  __shared__ float red[2][kWaves];
  float w[NV][8], dw[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[i][j] = dw[i][j] = 0.f;
    if (t + i * TPR < pieces) {
      Piece<false> b;
      b.load(weight, t + i * TPR);
      b.get(w[i]);
    }
  }
  int turn = 0;
  for (int row = blockIdx.x; row < T; row += gridDim.x, turn ^= 1) {
    const long long base = (long long)row * pieces;
    const float r = rstd[row];
    float g[NV][8], n[NV][8], dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int p = t + i * TPR;
      if (p < pieces) {
        Piece<BF16> a, b;
        a.load(dy, base + p);
        b.load(h, base + p);
        a.get(g[i]);
        b.get(n[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          n[i][j] *= r;
          dw[i][j] = fmaf(g[i][j], n[i][j], dw[i][j]);
          g[i][j] *= w[i][j];
          dot = fmaf(g[i][j], n[i][j], dot);
        }
      }
    }
    dot = wave_sum(dot);
    if constexpr (kWaves > 1) {
      if (lane == 0) red[turn][t >> 6] = dot;
      __syncthreads();                       // two buffers: the next row's sums do not meet this row's reads
      dot = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) dot += red[turn][i];
    }
    const float mean = dot * inv_d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int p = t + i * TPR;
      if (p < pieces) {
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = r * (g[i][j] - n[i][j] * mean);
        Piece<BF16> a;
        if (dsum) {
          float e[8];
          a.load(dsum, base + p);
          a.get(e);
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] += e[j];
        }
        a.set(o);
        a.store(dx, base + p);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int p = t + i * TPR;
    if (p < pieces) {
      Piece<false> o;
      o.set(dw[i]);
      o.store(partial, (long long)blockIdx.x * pieces + p);
    }
  }
}

// dw[j] = sum of n rows of the workspace: 64 columns per workgroup, 16 waves that stride the rows
__global__ void __launch_bounds__(1024) rmsnorm_bwd_sum_kernel(const float* __restrict__ partial, float* dweight, int n,
                                                               int d) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int j = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (j < d)
    for (int i = wv; i < n; i += 16) s += partial[(long long)i * d + j];
  red[wv][lane] = s;
  __syncthreads();
  if (wv == 0 && j < d) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += red[i][lane];
    dweight[j] = s;
  }
}

size_t norm_workspace_bytes(const mohge_norm_config& c) { return (size_t)kBwdGroups * c.d * sizeof(float); }

template <bool BF16>
static hipError_t launch_norm_bwd(const mohge_norm_config& c, const void* dy, const void* h, const float* weight,
                                  const float* rstd, const void* dsum, void* dx, float* dweight, float* partial,
                                  hipStream_t s) {
  const int pieces = c.d / 8, groups = c.T < kBwdGroups ? c.T : kBwdGroups;
  auto go = [&](auto kern, int tpr) {
    hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(tpr), 0, s, dy, h, weight, rstd, dsum, dx, partial, c.T, pieces,
                       1.f / c.d);
  };
  if (groups > 0) {
    if (pieces <= 64) go(rmsnorm_bwd_kernel<BF16, 64, 1>, 64);
    else if (pieces <= 128) go(rmsnorm_bwd_kernel<BF16, 128, 1>, 128);
    else if (pieces <= 256) go(rmsnorm_bwd_kernel<BF16, 256, 1>, 256);
    else if (pieces <= 512) go(rmsnorm_bwd_kernel<BF16, 256, 2>, 256);
    else if (pieces <= 1024) go(rmsnorm_bwd_kernel<BF16, 512, 2>, 512);
    else if (pieces <= 2048) go(rmsnorm_bwd_kernel<BF16, 1024, 2>, 1024);
    else go(rmsnorm_bwd_kernel<BF16, 1024, 4>, 1024);
  }
  hipLaunchKernelGGL(rmsnorm_bwd_sum_kernel, dim3((unsigned)((c.d + 63) / 64)), dim3(1024), 0, s, partial, dweight, groups,
                     c.d);
  return hipGetLastError();
}

hipError_t launch_rmsnorm_bwd(const mohge_norm_config& c, const void* dy, const void* h, const float* weight,
                              const float* rstd, const void* dsum, void* dx, float* dweight, void* ws, hipStream_t s) {
  float* partial = static_cast<float*>(ws);
  return c.dtype == MOHGE_BF16 ? launch_norm_bwd<true>(c, dy, h, weight, rstd, dsum, dx, dweight, partial, s)
                               : launch_norm_bwd<false>(c, dy, h, weight, rstd, dsum, dx, dweight, partial, s);
}

}  // namespace mohge
