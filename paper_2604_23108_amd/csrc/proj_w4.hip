// Product of up to 32 rows with 4-bit weights and group scales, for gfx950 (the projections of a decode step).
//   y[t,n] = xs_t sum_g s_ng (sum_{k in g} c_nk x_tk - z_ng sum_{k in g} x_tk)
// Bound by memory: the codes are streamed once, 32 codes (16 bytes of a weight row) per lane and request.
//
// v_mfma_f32_16x16x32_bf16 with the rows of x as the first operand and 16 weight rows as the second, so that everything a
// lane accumulates belongs to one weight row, (lane & 15), and its scales multiply without another lane.
//   codes to operands   a code c placed under the exponent of 16 is the bf16 number 16 + c, exactly: one shift and one
//                       and-or per pair of codes.  The pairs that fall out are (0,4) (1,5) (2,6) (3,7) of eight; x lies in
//                       LDS in that order.  The offset leaves with the zero point: c - z = (16 + c) - (16 + z).
//   sums of x           a product with ones gives sum_{k in g} x_tk in the lanes that need it.
//   groups              one product reduces 8 codes of each of four lanes; with groups of 128 those are in one group as
//                       loaded, for 64 and 32 the lanes exchange words first (v_permlane32_swap, v_permlane16_swap).
#include "block.h"

namespace mohge {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

union ProjFrag {
  uint4 u;
  uint32_t w[4];
  bf16x8 v;
};

constexpr int kProjLds = 64 * 1024;          // bytes of staged rows of x

// 8 codes -> 16 + c as bf16, in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ void codes_to_bf16(const uint32_t c, ProjFrag& f) {
  f.w[0] = ((c << 3) & 0x00780078u) | 0x41804180u;
  f.w[1] = ((c >> 1) & 0x00780078u) | 0x41804180u;
  f.w[2] = ((c >> 5) & 0x00780078u) | 0x41804180u;
  f.w[3] = ((c >> 9) & 0x00780078u) | 0x41804180u;
}

// Words of the four lanes of a weight row (32 codes each, word w of lane q: codes 32 q + 8 w ..) -> words whose four lanes
// lie in one group
template <int GROUP>
__device__ __forceinline__ void regroup(uint32_t (&c)[4]) {
  if constexpr (GROUP <= 64) {
    const auto a = __builtin_amdgcn_permlane32_swap(c[0], c[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(c[1], c[3], false, false);
    c[0] = a[0]; c[2] = a[1]; c[1] = b[0]; c[3] = b[1];
  }
  if constexpr (GROUP <= 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(c[0], c[1], false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(c[2], c[3], false, false);
    c[0] = a[0]; c[1] = a[1]; c[2] = b[0]; c[3] = b[1];
  }
}

// First of the 8 reduction indices of word w in lane q, after regroup
template <int GROUP>
__device__ __forceinline__ int index_of(int w, int q) {
  if constexpr (GROUP == 128) return 32 * q + 8 * w;
  else if constexpr (GROUP == 64) return 64 * (w >> 1) + 32 * (q & 1) + 16 * (q >> 1) + 8 * (w & 1);
  else return 32 * w + 8 * q;
}

// Rows [T, n_in] of x, indices k0 .. k0 + n, to LDS as bf16 in the order 0 4 1 5 2 6 3 7 of every eight, zero past n_in
template <bool E4M3>
__device__ __forceinline__ void stage_rows(const void* x, int T, int n_in, int k0, int n, int pitch, unsigned char* lds) {
  const int per = n / 8;
  for (int i = threadIdx.x; i < T * per; i += 256) {
    const int t = i / per, p = i - t * per, k = k0 + 8 * p;
    uint32_t d[4] = {0u, 0u, 0u, 0u};
    if (k < n_in) {
      if constexpr (E4M3) {
        const uint2 c = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(x) + (long long)t * n_in + k);
        const uint32_t w[2] = {c.x, c.y};
#pragma unroll
        for (int j = 0; j < 2; ++j) {                       // exact: the upper halves of the fp32 patterns
          const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false);
          const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
          d[2 * j] = (__float_as_uint(a[0]) >> 16) | (__float_as_uint(a[1]) & 0xffff0000u);
          d[2 * j + 1] = (__float_as_uint(b[0]) >> 16) | (__float_as_uint(b[1]) & 0xffff0000u);
        }
      } else {
        const uint4 c = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + (long long)t * n_in + k);
        d[0] = c.x; d[1] = c.y; d[2] = c.z; d[3] = c.w;
      }
    }
    *reinterpret_cast<uint4*>(lds + t * pitch + 16 * p) =
        make_uint4(__builtin_amdgcn_perm(d[2], d[0], 0x05040100u), __builtin_amdgcn_perm(d[2], d[0], 0x07060302u),
                   __builtin_amdgcn_perm(d[3], d[1], 0x05040100u), __builtin_amdgcn_perm(d[3], d[1], 0x07060302u));
  }
}

struct ProjArgs {
  const void* x;
  const float* x_scale;
  const unsigned char* codes;
  const uint16_t* scales;
  const unsigned char* zeros;
  void* y;
  int T, n_in, n_out, chunk;          // chunk: indices of x staged at a time
};

// NT blocks of 16 rows of x.  KW of the workgroup's four waves share 16 weight rows, a unit (128 indices) each in turn.
template <int GROUP, int NT, int KW, bool E4M3, bool F32>
__global__ void __launch_bounds__(256) proj_w4_kernel(const ProjArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int kPerUnit = 128 / GROUP, kWords = 4 / kPerUnit;       // groups in a unit, words of a group
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, q = lane >> 4, kw = w % KW;
  const int n0 = (blockIdx.x * (4 / KW) + w / KW) * 16;
  const int row = min(n0 + m, a.n_out - 1), groups = a.n_in / GROUP;
  const unsigned char* cp = a.codes + (long long)row * (a.n_in / 2) + 16 * q;
  const uint16_t* sp = a.scales + (long long)row * groups;
  const unsigned char* zp = a.zeros ? a.zeros + (long long)row * groups : nullptr;
  const int pitch = a.chunk * 2 + 16;
  const unsigned char* xrow[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) xrow[t] = lds + min(16 * t + m, a.T - 1) * pitch;
  ProjFrag ones;
#pragma unroll
  for (int i = 0; i < 4; ++i) ones.w[i] = 0x3f803f80u;
  f32x4 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int k0 = 0; k0 < a.n_in; k0 += a.chunk) {
    const int n = min(a.chunk, (a.n_in - k0 + 127) / 128 * 128);
    if (k0 > 0) __syncthreads();
    stage_rows<E4M3>(a.x, a.T, a.n_in, k0, n, pitch, lds);
    __syncthreads();
    for (int u = 128 * kw; u < n; u += 128 * KW) {
      const int k = k0 + u;
      uint32_t c[4] = {0u, 0u, 0u, 0u};
      if (k + 32 * q < a.n_in) {
        const uint4 v = *reinterpret_cast<const uint4*>(cp + k / 2);
        c[0] = v.x; c[1] = v.y; c[2] = v.z; c[3] = v.w;
      }
      regroup<GROUP>(c);
#pragma unroll
      for (int g = 0; g < kPerUnit; ++g) {
        const int at = k / GROUP + g;
        const bool in = at < groups;                         // (the last unit may hold half of its groups)
        const float s = in ? bf16_to_f32(sp[at]) : 0.f;
        const float z = zp ? 16.f + (float)(in ? zp[at] : 0) : 24.f;
        f32x4 part[NT], sx[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) part[t] = sx[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
          ProjFrag wf;
          codes_to_bf16(c[g * kWords + j], wf);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            ProjFrag xf;
            xf.u = *reinterpret_cast<const uint4*>(xrow[t] + 2 * (u + index_of<GROUP>(g * kWords + j, q)));
            part[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf.v, wf.v, part[t], 0, 0, 0);
            sx[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf.v, ones.v, sx[t], 0, 0, 0);
          }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(s, fmaf(-z, sx[t][i], part[t][i]), acc[t][i]);
      }
    }
  }
  if constexpr (KW > 1) {                       // the waves of a row, added in their order
    __syncthreads();
    f32x4* red = reinterpret_cast<f32x4*>(lds);
#pragma unroll
    for (int t = 0; t < NT; ++t)
      if (kw > 0) red[(w * NT + t) * 64 + lane] = acc[t];
    __syncthreads();
    if (kw > 0) return;
#pragma unroll
    for (int x = 1; x < KW; ++x)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t] += red[((w + x) * NT + t) * 64 + lane];
  }
  if (n0 + m >= a.n_out) return;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * t + 4 * q + i;
      if (r < a.T) {
        float v = acc[t][i];
        if constexpr (E4M3) v *= a.x_scale[r];
        const long long at = (long long)r * a.n_out + n0 + m;
        if constexpr (F32) static_cast<float*>(a.y)[at] = v;
        else static_cast<uint16_t*>(a.y)[at] = (uint16_t)pack_bf16x2(v, 0.f);
      }
    }
}

template <int GROUP, int NT, int KW>
static void go_proj(const ProjArgs& a, bool e4m3, bool f32, hipStream_t s) {
  const unsigned blocks = (unsigned)((a.n_out + 64 / KW - 1) / (64 / KW));
  int bytes = a.T * (a.chunk * 2 + 16);
  if (KW > 1 && bytes < 4 * NT * 64 * 16) bytes = 4 * NT * 64 * 16;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), bytes, s, a); };
  if (e4m3) { if (f32) go(proj_w4_kernel<GROUP, NT, KW, true, true>); else go(proj_w4_kernel<GROUP, NT, KW, true, false>); }
  else { if (f32) go(proj_w4_kernel<GROUP, NT, KW, false, true>); else go(proj_w4_kernel<GROUP, NT, KW, false, false>); }
}

template <int GROUP>
static void go_proj(const ProjArgs& a, bool e4m3, bool f32, hipStream_t s) {
  const bool many = a.n_out >= 64 * 512;          // two workgroups per compute unit without a split of the reduction
  if (a.T <= 16) { if (many) go_proj<GROUP, 1, 1>(a, e4m3, f32, s); else go_proj<GROUP, 1, 4>(a, e4m3, f32, s); }
  else { if (many) go_proj<GROUP, 2, 1>(a, e4m3, f32, s); else go_proj<GROUP, 2, 4>(a, e4m3, f32, s); }
}

hipError_t launch_proj_w4(const mohge_proj_config& c, const void* x, const float* x_scale, const void* codes,
                          const void* scales, const void* zeros, void* y, hipStream_t s) {
  ProjArgs a;
  a.x = x; a.x_scale = x_scale; a.codes = static_cast<const unsigned char*>(codes);
  a.scales = static_cast<const uint16_t*>(scales); a.zeros = static_cast<const unsigned char*>(zeros); a.y = y;
  a.T = c.T; a.n_in = c.n_in; a.n_out = c.n_out;
  const int all = (c.n_in + 127) / 128 * 128, fit = (kProjLds / c.T - 16) / 2 / 128 * 128;
  a.chunk = all < fit ? all : fit;
  const bool e4m3 = c.x_dtype == MOHGE_E4M3, f32 = c.y_dtype == MOHGE_F32;
  if (c.group == 128) go_proj<128>(a, e4m3, f32, s);
  else if (c.group == 64) go_proj<64>(a, e4m3, f32, s);
  else go_proj<32>(a, e4m3, f32, s);
  return hipGetLastError();
}

}  // namespace mohge
