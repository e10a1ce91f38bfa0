// Root-mean-square norm with the residual's addition for gfx950, forward and backward.
//   forward   h = x + r,  rstd = (mean h^2 + eps)^-1/2,  y = h rstd w
//   backward  n = h rstd, g = w dy, dx = ds + rstd (g - n mean(g n)),  dw = sum over rows of dy n
// Bound by memory: a row is read once into registers (8 elements per thread and piece), its one or two sums
// are folded across the threads that share it, and it is written from the registers.
// Measured (bf16, with residual and stored sum: four arrays of T d elements): 16384 rows of 4096 94 us, 5.7 TB/s, as fast as a copy
// of that size; 777 of 1344 3.2 us and one of 4096 2.3, where a launch alone is 2.
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
  const int mine = threadIdx.x / TPR, row = blockIdx.x * kRows + mine;
  const long long base = (long long)min(row, T - 1) * pieces;          // rows past the end read the last one
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
    __shared__ float red[kRows][2 * kWaves];
    if (lane == 0) {
      red[mine][t >> 6] = ss;
      if constexpr (Q8) red[mine][kWaves + (t >> 6)] = top;
    }
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) ss += red[mine][i];
    if constexpr (Q8) {
#pragma unroll
      for (int i = 0; i < kWaves; ++i) top = fmaxf(top, red[mine][kWaves + i]);
    }
  }
  if (row >= T) return;
  const float rstd = rsqrtf(ss * inv_d + eps);
  float scale = 1.f, inv_scale = 1.f;
  if constexpr (Q8) {
    scale = e4m3_scale(top * rstd);          // top * rstd is the largest |y| as it is rounded below: rounding keeps the order
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
      if constexpr (Q8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = h[i][j] * w[i][j] * rstd * inv_scale;
        static_cast<uint2*>(y)[base + p] = to_e4m3x8(v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = h[i][j] * rstd * w[i][j];
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
  // One piece per thread as far as a workgroup reaches (us for 1, 777 and 8192 rows): 4096 columns by 512 threads 2.5, 6.3, 47.9,
  // by 256 with two pieces 2.9, 6.4, 52.4; 8192 by 1024 2.7, 10.4, 91, by 512 3.1, 10.1, 98; 1024 by 128 2.3, 3.1, 12.5, by 64 2.8, 3.4,
  // 12.0.
  // Not more threads than pieces: 1024 columns by 512 threads take 16.4 for 8192 rows.
  auto go = [&](auto kern, int tpr) {
    const int rows = tpr < 256 ? 256 / tpr : 1;
    hipLaunchKernelGGL(kern, dim3((unsigned)((c.T + rows - 1) / rows)), dim3(tpr < 256 ? 256 : tpr), 0, s, x, residual,
                       weight, sum_out, y, y_scale, rstd, c.T, pieces, 1.f / c.d, c.eps);
  };
  if (pieces <= 64) go(rmsnorm_kernel<BF16, 64, 1, Q8>, 64);
  else if (pieces <= 128) go(rmsnorm_kernel<BF16, 128, 1, Q8>, 128);
  else if (pieces <= 256) go(rmsnorm_kernel<BF16, 256, 1, Q8>, 256);
  else if (pieces <= 512) go(rmsnorm_kernel<BF16, 512, 1, Q8>, 512);
  else if (pieces <= 1024) go(rmsnorm_kernel<BF16, 1024, 1, Q8>, 1024);
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
// each workgroup, which a second kernel adds in their order: the sums do not depend on which workgroup ends first.
// Bound by memory (bf16 with ds: 8192 x 2048 31 us, 4.3 TB/s, 8192 x 8192 101 us, 5.3 TB/s) and, where rows are few, by two launches and
// the parts in between (fp32 777 x 1024 7.0 us: 4.0 and 2.3 by themselves).
constexpr int kBwdGroups = 512;          // workgroups at most: two per compute unit

template <bool BF16, int NV>
struct NormRow {
  Piece<BF16> dy[NV], h[NV], ds[NV > 2 ? 1 : NV];
  float rstd;
};

template <bool BF16, int TPR, int NV, bool DSUM>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) rmsnorm_bwd_kernel(const void* dy, const void* __restrict__ h,
                                                                            const float* __restrict__ weight,
                                                                            const float* __restrict__ rstd, const void* dsum,
                                                                            void* dx, float* __restrict__ partial, int T,
                                                                            int pieces, float inv_d) {
  constexpr int kRows = TPR < 256 ? 256 / TPR : 1, kWaves = TPR / 64;
  // Registers for the next row: with 1024 threads there are 128, which two pieces fill (8192 x 16384 204 us; 240 with the next row, spilt).
  constexpr bool kAhead = TPR < 1024 || NV == 1;
  // With four pieces not even the weights and the row as numbers fit: they are read and converted twice (8192 x 32768 484 us, 1072 kept).
  constexpr bool kLean = NV > 2;
  const int t = threadIdx.x % TPR, mine = threadIdx.x / TPR, lane = threadIdx.x & 63;
  __shared__ float red[2][kRows][kWaves];
  float w[kLean ? 1 : NV][8], dw[NV][8];
  auto load_weight = [&](int i, float (&to)[8], int from) {
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j] = 0.f;
    if (t + i * TPR < pieces) {
      Piece<false> b;
      b.load(weight, from + t + i * TPR);
      b.get(to);
    }
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.f;
    if constexpr (!kLean) load_weight(i, w[i], 0);
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
      if constexpr (DSUM && !kLean) x.ds[i].load(dsum, base + p);
    }
  };
  const int step = gridDim.x * kRows, row0 = blockIdx.x * kRows + mine;
  const int turns = (T - (int)blockIdx.x * kRows + step - 1) / step;          // the same for the whole workgroup
  NormRow<BF16, NV> cur, next;
  if constexpr (kAhead) load(cur, min(row0, T - 1));
  for (int k = 0; k < turns; ++k) {
    const int row = row0 + k * step;
    if constexpr (!kAhead) load(cur, min(row, T - 1));
    else if (k + 1 < turns) load(next, min(row + step, T - 1));
    const float r = row < T ? cur.rstd : 0.f;
    float g[kLean ? 1 : NV][8], n[kLean ? 1 : NV][8], dot = 0.f;
    int none = 0;
    auto terms = [&](int i, float (&gi)[8], float (&ni)[8]) {
      cur.dy[i].get(gi);
      cur.h[i].get(ni);
      if constexpr (kLean) load_weight(i, w[0], none);
#pragma unroll
      for (int j = 0; j < 8; ++j) ni[j] *= r;
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float (&gi)[8] = g[kLean ? 0 : i], (&ni)[8] = n[kLean ? 0 : i];
      if constexpr (kLean) asm volatile("" : "+v"(none));          // (keeps the loads of the weights here)
      terms(i, gi, ni);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (row < T) dw[i][j] = fmaf(gi[j], ni[j], dw[i][j]);
        gi[j] *= w[kLean ? 0 : i][j];
        dot = fmaf(gi[j], ni[j], dot);
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
          float (&gi)[8] = g[kLean ? 0 : i], (&ni)[8] = n[kLean ? 0 : i];
          if constexpr (kLean) {
            if constexpr (DSUM) cur.ds[0].load(dsum, base + t + i * TPR);
            asm volatile("" : "+v"(none));
            terms(i, gi, ni);
#pragma unroll
            for (int j = 0; j < 8; ++j) gi[j] *= w[0][j];
          }
          if constexpr (DSUM) cur.ds[kLean ? 0 : i].get(e);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            o[j] = r * (gi[j] - ni[j] * mean);
            if constexpr (DSUM) o[j] += e[j];
          }
          Piece<BF16> a;
          a.set(o);
          a.store(dx, base + t + i * TPR);
        }
      }
    }
    if constexpr (kAhead) cur = next;
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

// dw[j] = sum of n rows of the workspace (2.3 us for 256 rows of 1024): 32 columns per workgroup, four to a thread, 32 threads
// along the rows
__global__ void __launch_bounds__(256) rmsnorm_bwd_sum_kernel(const float* __restrict__ partial, float* dweight, int n,
                                                              int d) {
  __shared__ float4 red[32][8];
  const int c = threadIdx.x & 7, part = threadIdx.x >> 3, j = blockIdx.x * 32 + 4 * c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (j < d) {
    for (int i = part; i < n; i += 256) {          // eight requests at once; those past the end ask for the last row
      float4 v[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] = *reinterpret_cast<const float4*>(partial + (long long)min(i + 32 * x, n - 1) * d + j);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (i + 32 * x < n) { s.x += v[x].x; s.y += v[x].y; s.z += v[x].z; s.w += v[x].w; }
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
  // Threads per row by its length (us for 777 and 8192 rows, bf16): 1024 columns by 64 threads 6.0, 16.5, by 128 6.4, 17.4; 2048 by 128 8.2,
  // 30.1, by 256 9.1, 31.7; 2560 by 512 10.3, 36.9, by 256 11.0, 37.0; 4096 by 512 12.0, 55.8, by 256 12.6, 55.6; 8192 by 1024 16.1, 101,
  // by 512 16.6, 105.
  // Workgroups: one per compute unit, the parts of dw are fewer then, and two from three turns of each on, where their reads
  // overlap more (2048 columns: 2000 rows 12.4 with one, 13.3 with two; 4096 rows 18.2, 16.8).  Of 1024 threads always one (4096 x 8192
  // 55 against 62).
  const int pieces = c.d / 8;
  int groups = 0;
  auto go = [&](auto tpr, auto nv) {
    constexpr int kThreads = tpr.value < 256 ? 256 : tpr.value, kRows = kThreads / tpr.value;
    const int turns = (c.T + kRows - 1) / kRows;
    const int most = tpr.value < 1024 && turns >= 3 * kBwdGroups ? kBwdGroups : kBwdGroups / 2;
    const int each = (turns + most - 1) / most;
    groups = each ? (turns + each - 1) / each : 0;
    if (groups == 0) return;
    auto launch = [&](auto kern) {
      hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kThreads), 0, s, dy, h, weight, rstd, dsum, dx, partial, c.T, pieces,
                         1.f / c.d);
    };
    if (dsum) launch(rmsnorm_bwd_kernel<BF16, tpr.value, nv.value, true>);
    else launch(rmsnorm_bwd_kernel<BF16, tpr.value, nv.value, false>);
  };
  if (pieces <= 64) go(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  else if (pieces <= 128) go(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  else if (pieces <= 256) go(std::integral_constant<int, 128>(), std::integral_constant<int, 2>());
  else if (pieces <= 512) go(std::integral_constant<int, 512>(), std::integral_constant<int, 1>());
  else if (pieces <= 1024) go(std::integral_constant<int, 1024>(), std::integral_constant<int, 1>());
  else if (pieces <= 2048) go(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
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
