// Root-mean-square norm with the residual's addition for gfx950, forward and backward.
//   forward   h = x + r,  rstd = (mean h^2 + eps)^-1/2,  y = h rstd w
//   backward  n = h rstd, g = w dy, dx = ds + rstd (g - n mean(g n)),  dw = sum over rows of dy n
// Bound by memory: a row is read once into registers (8 elements per thread and piece), its one or two sums
// are folded across the threads that share it, and it is written from the registers.
#include <type_traits>

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
// TPR threads share a row and walk rows, the next one's elements on the way while the sums of one are folded; a thread keeps the
// part of dw of its columns in registers.  A workgroup's parts are added in LDS and left in the workspace, one row for
// each workgroup, which a second kernel adds in their order.
constexpr int kBwdGroups = 512;          // workgroups at most: two per compute unit

template <bool BF16, int NV>
struct NormRow {
  Piece<BF16> dy[NV], h[NV], ds[NV];
  float rstd;
};

template <bool BF16, int TPR, int NV, bool DSUM>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) rmsnorm_bwd_kernel(const void* dy, const void* __restrict__ h,
                                                                            const float* __restrict__ weight,
                                                                            const float* __restrict__ rstd, const void* dsum,
                                                                            void* dx, float* __restrict__ partial, int T,
                                                                            int pieces, float inv_d) {
  constexpr int kRows = TPR < 256 ? 256 / TPR : 1, kWaves = TPR / 64;
  const int t = threadIdx.x % TPR, mine = threadIdx.x / TPR, lane = threadIdx.x & 63;
  __shared__ float red[2][kRows][kWaves];
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
  // pieces past the row's end hold its last one, with a weight of 0
  auto load = [&](NormRow<BF16, NV>& x, int row) {
    const long long base = (long long)row * pieces;
    x.rstd = rstd[row];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int p = min(t + i * TPR, pieces - 1);
      x.dy[i].load(dy, base + p);
      x.h[i].load(h, base + p);
      if constexpr (DSUM) x.ds[i].load(dsum, base + p);
    }
  };
  const int step = gridDim.x * kRows, row0 = blockIdx.x * kRows + mine;
  const int turns = (T - (int)blockIdx.x * kRows + step - 1) / step;          // the same for the whole workgroup
  NormRow<BF16, NV> cur, next;
  load(cur, min(row0, T - 1));
  for (int k = 0; k < turns; ++k) {
    const int row = row0 + k * step;
    if (k + 1 < turns) load(next, min(row + step, T - 1));
    const float r = row < T ? cur.rstd : 0.f;
    float g[NV][8], n[NV][8], dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      cur.dy[i].get(g[i]);
      cur.h[i].get(n[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[i][j] *= r;
        if (row < T) dw[i][j] = fmaf(g[i][j], n[i][j], dw[i][j]);
        g[i][j] *= w[i][j];
        dot = fmaf(g[i][j], n[i][j], dot);
      }
    }
    dot = wave_sum(dot);
    if constexpr (kWaves > 1) {
      if (lane == 0) red[k & 1][mine][t >> 6] = dot;
      __syncthreads();                       // two buffers: the next row's sums do not meet this row's reads
      dot = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) dot += red[k & 1][mine][i];
    }
    const float mean = dot * inv_d;
    if (row < T) {
      const long long base = (long long)row * pieces;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (t + i * TPR < pieces) {
          float o[8], e[8];
          if constexpr (DSUM) cur.ds[i].get(e);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            o[j] = r * (g[i][j] - n[i][j] * mean);
            if constexpr (DSUM) o[j] += e[j];
          }
          Piece<BF16> a;
          a.set(o);
          a.store(dx, base + t + i * TPR);
        }
      }
    }
    cur = next;
  }
  // the rows' groups of a workgroup, added in their order
  if constexpr (kRows > 1) {
    __shared__ float sums[kRows - 1][NV * 8][TPR];
    if (mine > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[mine - 1][8 * i + j][t] = dw[i][j];
    }
    __syncthreads();
    if (mine > 0) return;
#pragma unroll
    for (int x = 0; x < kRows - 1; ++x)
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] += sums[x][8 * i + j][t];
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

// dw[j] = sum of n rows of the workspace: 32 columns per workgroup, four to a thread, 32 threads along the rows
__global__ void __launch_bounds__(256) rmsnorm_bwd_sum_kernel(const float* __restrict__ partial, float* dweight, int n,
                                                              int d) {
  __shared__ float4 red[32][8];
  const int c = threadIdx.x & 7, part = threadIdx.x >> 3, j = blockIdx.x * 32 + 4 * c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (j < d) {
#pragma unroll 8
    for (int i = part; i < n; i += 32) {
      const float4 v = *reinterpret_cast<const float4*>(partial + (long long)i * d + j);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  red[part][c] = s;
  __syncthreads();
  if (part < 4) {                                  // four threads add eight parts each, then one adds four
    s = red[8 * part][c];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      const float4 v = red[8 * part + i][c];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  __syncthreads();
  if (part < 4) red[part][c] = s;
  __syncthreads();
  if (part == 0 && j < d) {
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      const float4 v = red[i][c];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    *reinterpret_cast<float4*>(dweight + j) = s;
  }
}

size_t norm_workspace_bytes(const mohge_norm_config& c) { return (size_t)kBwdGroups * c.d * sizeof(float); }

template <bool BF16>
static hipError_t launch_norm_bwd(const mohge_norm_config& c, const void* dy, const void* h, const float* weight,
                                  const float* rstd, const void* dsum, void* dx, float* dweight, float* partial,
                                  hipStream_t s) {
  const int pieces = c.d / 8;
  int groups = 0;
  auto go = [&](auto tpr, auto nv) {
    constexpr int kRows = tpr.value < 256 ? 256 / tpr.value : 1;
    groups = (c.T + kRows - 1) / kRows;
    if (groups > kBwdGroups) groups = kBwdGroups;
    if (groups == 0) return;
    auto launch = [&](auto kern) {
      hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(tpr.value < 256 ? 256 : tpr.value), 0, s, dy, h, weight, rstd, dsum,
                         dx, partial, c.T, pieces, 1.f / c.d);
    };
    if (dsum) launch(rmsnorm_bwd_kernel<BF16, tpr.value, nv.value, true>);
    else launch(rmsnorm_bwd_kernel<BF16, tpr.value, nv.value, false>);
  };
  constexpr int kMost = BF16 ? 4 : 2;          // pieces that a thread's registers hold
  auto with = [&](auto tpr) { go(tpr, std::integral_constant<int, kMost>()); };
  if (pieces <= 64) go(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  else if (pieces <= 128) go(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  else if (pieces <= 64 * kMost) with(std::integral_constant<int, 64>());
  else if (pieces <= 128 * kMost) with(std::integral_constant<int, 128>());
  else if (pieces <= 256 * kMost) with(std::integral_constant<int, 256>());
  else if (pieces <= 512 * kMost) with(std::integral_constant<int, 512>());
  else if (pieces <= 1024 * 2) go(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
  else go(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>());
  hipLaunchKernelGGL(rmsnorm_bwd_sum_kernel, dim3((unsigned)((c.d + 31) / 32)), dim3(256), 0, s, partial, dweight, groups,
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
