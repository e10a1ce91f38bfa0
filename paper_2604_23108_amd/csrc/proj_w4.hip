// Product of up to 32 rows with 4-bit weights and group scales, for gfx950 (the projections of a decode step).
//   y[t,n] = xs_t sum_g s_ng (sum_{k in g} c_nk x_tk - z_ng sum_{k in g} x_tk)
// Bound by memory: the codes are streamed once, 32 codes (16 bytes of a weight row) per lane and request.
//
// v_mfma_f32_16x16x32_bf16 with the rows of x as the first operand and 16 weight rows as the second, so that everything a
// lane accumulates belongs to one weight row, (lane & 15), and its scales multiply without another lane.
//   codes to operands   a code c placed under the exponent of 16 is the bf16 number 16 + c, exactly: one shift and one
//                       and-or per pair of codes.  The pairs that fall out are (0,4) (1,5) (2,6) (3,7) of eight; x lies in
//                       LDS in that order.  The offset leaves with the zero point: c - z = (16 + c) - (16 + z).
//                       (E4M3 rows of x become bf16 as well.  As E4M3 numbers, which the codes' bytes are by themselves in units of
//                       2^-9, the products need half the instructions, but v_mfma_f32_16x16x32_fp8_fp8 drops bits when it adds
//                       them: results 5e-5 off, where this form's are 2e-7.)
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

// 8 codes -> 16 + c as bf16, in the order 0 4 1 5 2 6 3 7.  (The mask and the exponent come in registers: an instruction holds one
// constant, and with two the and-or becomes an and and an or, which made the conversion half of all instructions again.)
__device__ __forceinline__ void codes_to_bf16(const uint32_t c, const uint32_t mask, const uint32_t sixteen, ProjFrag& f) {
  f.w[0] = ((c << 3) & mask) | sixteen;
  f.w[1] = ((c >> 1) & mask) | sixteen;
  f.w[2] = ((c >> 5) & mask) | sixteen;
  f.w[3] = ((c >> 9) & mask) | sixteen;
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

struct ProjArgs {
  const void* x;
  const float* x_scale;
  const unsigned char* codes;
  const uint16_t* scales;
  const unsigned char* zeros;
  void* y;
  int T, n_in, n_out, f32;
  int units;          // units staged at a time, a power of two; a unit is 128 indices (64 bytes) of a weight row
  int shift;          // log2 of the pieces of 8 indices in a staged row, units * 16
};

// 8 elements of x: requested, and later put to LDS as bf16 in the order 0 4 1 5 2 6 3 7
template <bool E4M3>
struct Eight {
  uint32_t d[E4M3 ? 2 : 4];
  __device__ __forceinline__ void load(const void* x, long long at, bool in) {
#pragma unroll
    for (int i = 0; i < (E4M3 ? 2 : 4); ++i) d[i] = 0u;
    if (!in) return;
    if constexpr (E4M3) {
      const uint2 c = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(x) + at);
      d[0] = c.x; d[1] = c.y;
    } else {
      const uint4 c = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + at);
      d[0] = c.x; d[1] = c.y; d[2] = c.z; d[3] = c.w;
    }
  }
  __device__ __forceinline__ void store(unsigned char* to) const {
    uint32_t w[4];
    if constexpr (E4M3) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {                       // exact: the upper halves of the fp32 patterns
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[j], false);
        const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[j], true);
        w[2 * j] = __builtin_amdgcn_perm(__float_as_uint(a[1]), __float_as_uint(a[0]), 0x07060302u);
        w[2 * j + 1] = __builtin_amdgcn_perm(__float_as_uint(b[1]), __float_as_uint(b[0]), 0x07060302u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = d[j];
    }
    *reinterpret_cast<uint4*>(to) =
        make_uint4(__builtin_amdgcn_perm(w[2], w[0], 0x05040100u), __builtin_amdgcn_perm(w[2], w[0], 0x07060302u),
                   __builtin_amdgcn_perm(w[3], w[1], 0x05040100u), __builtin_amdgcn_perm(w[3], w[1], 0x07060302u));
  }
};

// RT blocks of 16 weight rows: the codes of U units, requested together, with their scales and zero points
template <int GROUP, int RT, int U>
struct Batch {
  static constexpr int kPer = 128 / GROUP;             // groups in a unit
  uint4 w[RT][U];
  uint32_t s[RT][U * kPer / 2];                         // bf16 pairs
  uint32_t z[RT][(U * kPer + 3) / 4];                   // up to four bytes each

  // units u0 .. u0 + U - 1, those before `end`
  __device__ __forceinline__ void load(const ProjArgs& a, const int (&row)[RT], int u0, int end, int q) {
    const int groups = a.n_in / GROUP, g0 = u0 * kPer;
    if (u0 + U <= end && (u0 + U) * 128 <= a.n_in) {
#pragma unroll
      for (int f = 0; f < RT; ++f) {
        const unsigned char* cp = a.codes + (long long)row[f] * (a.n_in / 2) + u0 * 64 + 16 * q;
#pragma unroll
        for (int u = 0; u < U; ++u) w[f][u] = *reinterpret_cast<const uint4*>(cp + 64 * u);
        __builtin_memcpy(s[f], a.scales + (long long)row[f] * groups + g0, sizeof(s[f]));       // (rows need not be aligned)
        if (a.zeros) __builtin_memcpy(z[f], a.zeros + (long long)row[f] * groups + g0, U * kPer);
      }
    } else {
#pragma unroll
      for (int f = 0; f < RT; ++f) {
        const unsigned char* cp = a.codes + (long long)row[f] * (a.n_in / 2) + u0 * 64 + 16 * q;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          w[f][u] = make_uint4(0u, 0u, 0u, 0u);
          if (u0 + u < end && (u0 + u) * 128 + 32 * q < a.n_in) w[f][u] = *reinterpret_cast<const uint4*>(cp + 64 * u);
        }
#pragma unroll
        for (int g = 0; g < U * kPer; ++g) {
          const bool in = g0 + g < end * kPer && g0 + g < groups;
          const uint32_t sv = in ? a.scales[(long long)row[f] * groups + g0 + g] : 0u;
          const uint32_t zv = in && a.zeros ? a.zeros[(long long)row[f] * groups + g0 + g] : 0u;
          s[f][g / 2] = g & 1 ? s[f][g / 2] | sv << 16 : sv;
          z[f][g / 4] = g & 3 ? z[f][g / 4] | zv << (8 * (g & 3)) : zv;
        }
      }
    }
  }
};

// acc += unit u of the batch; x: LDS address of the unit in row 16 t + m of x
template <int GROUP, int RT, int NT, int U>
__device__ __forceinline__ void multiply(const Batch<GROUP, RT, U>& b, const int u, const bool zeros,
                                         const unsigned char* const (&x)[NT], const int q, f32x4 (&acc)[RT][NT]) {
  constexpr int kPer = 128 / GROUP, kWords = 4 / kPer;
  ProjFrag ones;
#pragma unroll
  for (int i = 0; i < 4; ++i) ones.w[i] = 0x3f803f80u;
  uint32_t mask = 0x00780078u, sixteen = 0x41804180u;
  asm("" : "+s"(mask));
  asm("" : "+v"(sixteen));
  uint32_t c[RT][4];
#pragma unroll
  for (int f = 0; f < RT; ++f) {
    c[f][0] = b.w[f][u].x; c[f][1] = b.w[f][u].y; c[f][2] = b.w[f][u].z; c[f][3] = b.w[f][u].w;
    regroup<GROUP>(c[f]);
  }
#pragma unroll
  for (int g = 0; g < kPer; ++g) {
    f32x4 part[RT][NT], sx[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      sx[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < RT; ++f) part[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      ProjFrag xf[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        xf[t].u = *reinterpret_cast<const uint4*>(x[t] + 2 * index_of<GROUP>(g * kWords + j, q));
        sx[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[t].v, ones.v, sx[t], 0, 0, 0);
      }
#pragma unroll
      for (int f = 0; f < RT; ++f) {
        ProjFrag wf;
        codes_to_bf16(c[f][g * kWords + j], mask, sixteen, wf);
#pragma unroll
        for (int t = 0; t < NT; ++t) part[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[t].v, wf.v, part[f][t], 0, 0, 0);
      }
    }
#pragma unroll
    for (int f = 0; f < RT; ++f) {
      const int at = u * kPer + g;
      const float s = __uint_as_float(at & 1 ? b.s[f][at / 2] & 0xffff0000u : b.s[f][at / 2] << 16);
      const float z = zeros ? 16.f + (float)((b.z[f][at / 4] >> (8 * (at & 3))) & 255u) : 24.f;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[f][t][i] = fmaf(s, fmaf(-z, sx[t][i], part[f][t][i]), acc[f][t][i]);
    }
  }
}

template <bool E4M3, int RT, int NT>
__device__ __forceinline__ void store_rows(const ProjArgs& a, const int n0, const int m, const int q, const f32x4 (&acc)[RT][NT]) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * t + 4 * q + i;
      if (r < a.T) {
        float xs = 1.f;
        if constexpr (E4M3) xs = a.x_scale[r];
#pragma unroll
        for (int f = 0; f < RT; ++f) {
          const int n = n0 + 16 * f + m;
          if (n < a.n_out) {
            const long long at = (long long)r * a.n_out + n;
            if (a.f32) static_cast<float*>(a.y)[at] = acc[f][t][i] * xs;
            else static_cast<uint16_t*>(a.y)[at] = (uint16_t)pack_bf16x2(acc[f][t][i] * xs, 0.f);
          }
        }
      }
    }
}

// Few weight rows: a workgroup has 16 RT of them, its KW waves a part of the reduction each.  A wave stages its own part of
// x without a barrier, and has NB batches of two units on the way while it multiplies.
template <int GROUP, int NT, int RT, int KW, int NB, bool E4M3>
__global__ void __launch_bounds__(64 * KW) proj_w4_split_kernel(const ProjArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int U = 2;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int n0 = blockIdx.x * 16 * RT;
  int row[RT];
#pragma unroll
  for (int f = 0; f < RT; ++f) row[f] = min(n0 + 16 * f + m, a.n_out - 1);
  const int nu = (a.n_in + 127) / 128, ub = nu * w / KW, ue = nu * (w + 1) / KW;
  const int pitch = a.units * 256 + 16, all = a.T << a.shift;
  unsigned char* const mine = lds + w * a.T * pitch;
  const unsigned char* xrow[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) xrow[t] = mine + min(16 * t + m, a.T - 1) * pitch;
  // x of the units from uc on: kPieces per lane requested, and later put to LDS
  constexpr int kPieces = 4 * NT;
  Eight<E4M3> e[kPieces];
  auto request = [&](int uc, int i0) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = i0 + 64 * j, t = i >> a.shift, k = uc * 128 + 8 * (i - (t << a.shift));
      if (i0 - lane + 64 * j < all)                 // (wave-uniform: no address for nothing)
        e[j].load(a.x, (long long)t * a.n_in + k, i < all && k < a.n_in);
    }
  };
  auto put = [&](int i0) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = i0 + 64 * j, t = i >> a.shift;
      if (i < all) e[j].store(mine + t * pitch + 16 * (i - (t << a.shift)));
    }
  };
  // what is waited for first is requested first
  request(ub, lane);
  Batch<GROUP, RT, U> b[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) b[i].load(a, row, ub + U * i, ue, q);
  f32x4 acc[RT][NT];
#pragma unroll
  for (int f = 0; f < RT; ++f)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  // (units: a multiple of NB * U, or all of the wave's)
  for (int uc = ub; uc < ue; uc += a.units) {
    if (uc > ub) request(uc, lane);
    put(lane);
    for (int i0 = lane + 64 * kPieces; i0 - lane < all; i0 += 64 * kPieces) {
      request(uc, i0);
      put(i0);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int last = min(uc + a.units, ue);
    for (int u0 = uc; u0 < last; u0 += U * NB) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        if (u0 + U * i < last) {                       // wave-uniform; past an odd end codes, scales and zero points are 0
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const unsigned char* x[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) x[t] = xrow[t] + (u0 - uc + U * i + u) * 256;
            multiply<GROUP, RT, NT, U>(b[i], u, a.zeros != nullptr, x, q, acc);
          }
          if (u0 + U * (NB + i) < ue) b[i].load(a, row, u0 + U * (NB + i), ue, q);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  // the waves' sums, added in their order
  __syncthreads();
  f32x4* red = reinterpret_cast<f32x4*>(lds);
  if (w > 0) {
#pragma unroll
    for (int f = 0; f < RT; ++f)
#pragma unroll
      for (int t = 0; t < NT; ++t) red[(((w - 1) * RT + f) * NT + t) * 64 + lane] = acc[f][t];
  }
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int x = 0; x < KW - 1; ++x)
#pragma unroll
    for (int f = 0; f < RT; ++f)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[f][t] += red[((x * RT + f) * NT + t) * 64 + lane];
  store_rows<E4M3, RT, NT>(a, n0, m, q, acc);
}

constexpr int proj_batch(int group) { return group == 32 ? 2 : 4; }      // (the scales of finer groups need the registers)

// Many weight rows: every wave has 16 RT of its own and the whole reduction; the workgroup's waves share the staged rows of x, one part
// in LDS while the next is on the way.
template <int GROUP, int NT, int RT, bool E4M3>
__global__ void __launch_bounds__(256, 2) proj_w4_kernel(const ProjArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int kPieces = 8;                            // per thread and part: T * units * 16 <= 8 * 256
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int n0 = (blockIdx.x * 4 + w) * 16 * RT;
  int row[RT];
#pragma unroll
  for (int f = 0; f < RT; ++f) row[f] = min(n0 + 16 * f + m, a.n_out - 1);
  const int nu = (a.n_in + 127) / 128;
  constexpr int U = proj_batch(GROUP);
  Batch<GROUP, RT, U> cur, next;
  cur.load(a, row, 0, nu, q);
  const int pitch = a.units * 256 + 16, all = a.T << a.shift;
  Eight<E4M3> e[kPieces];
  auto request = [&](int u0) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = threadIdx.x + 256 * j, t = i >> a.shift, k = u0 * 128 + 8 * (i - (t << a.shift));
      e[j].load(a.x, (long long)t * a.n_in + k, i < all && k < a.n_in);
    }
  };
  auto put = [&](unsigned char* to) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = threadIdx.x + 256 * j, t = i >> a.shift;
      if (i < all) e[j].store(to + t * pitch + 16 * (i - (t << a.shift)));
    }
  };
  request(0);
  put(lds);
  f32x4 acc[RT][NT];
#pragma unroll
  for (int f = 0; f < RT; ++f)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  __syncthreads();
  int turn = 0;
  for (int uc = 0; uc < nu; uc += a.units, turn ^= 1) {
    const int cu = min(a.units, nu - uc);
    const bool more = uc + a.units < nu;
    if (more) request(uc + a.units);
    const unsigned char* xrow[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) xrow[t] = lds + (turn * a.T + min(16 * t + m, a.T - 1)) * pitch;
    for (int u0 = uc; u0 < uc + cu; u0 += U) {
      next.load(a, row, u0 + U, nu, q);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u0 + u < uc + cu) {                       // wave-uniform
          const unsigned char* x[NT];
#pragma unroll
          for (int t = 0; t < NT; ++t) x[t] = xrow[t] + (u0 - uc + u) * 256;
          multiply<GROUP, RT, NT, U>(cur, u, a.zeros != nullptr, x, q, acc);
        }
      }
      cur = next;
    }
    if (more) put(lds + (turn ^ 1) * a.T * pitch);
    __syncthreads();
  }
  store_rows<E4M3, RT, NT>(a, n0, m, q, acc);
}

// Largest power of two of units, at least `batch`, whose T rows fit `bytes`; no more than it takes for `units`
static void stage_units(ProjArgs& a, int batch, int bytes, int units) {
  a.units = batch;
  while (a.units < units && a.T * (2 * a.units * 256 + 16) <= bytes) a.units *= 2;
  a.shift = log2_of(a.units * 16);
}

template <int GROUP, int NT, int RT, bool E4M3>
static hipError_t go_many(ProjArgs& a, hipStream_t s) {
  static std::atomic<unsigned long long> allowed;
  constexpr int kBytes = 8 * 256 * 16 + 32 * 16;          // staged rows, one part
  stage_units(a, proj_batch(GROUP), kBytes, (a.n_in + 127) / 128);
  auto kern = proj_w4_kernel<GROUP, NT, RT, E4M3>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(kern), 2 * kBytes, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)((a.n_out + 64 * RT - 1) / (64 * RT))), dim3(256), 2 * a.T * (a.units * 256 + 16), s, a);
  return hipGetLastError();
}

template <int GROUP, int NT, int RT, int KW, int NB, bool E4M3>
static hipError_t go_split(ProjArgs& a, hipStream_t s) {
  static std::atomic<unsigned long long> allowed;
  // staged rows of a workgroup: two of them per compute unit, or, where that is less than two batches per wave, one
  constexpr int kTwo = 72 * 1024, kOne = 144 * 1024;
  const int least = a.T * (2 * 256 * NB + 16) * KW;
  stage_units(a, 2 * NB, (least <= kTwo ? kTwo : kOne) / KW, ((a.n_in + 127) / 128 + KW - 1) / KW);
  int bytes = KW * a.T * (a.units * 256 + 16);
  if (bytes < (KW - 1) * RT * NT * 64 * 16) bytes = (KW - 1) * RT * NT * 64 * 16;
  auto kern = proj_w4_split_kernel<GROUP, NT, RT, KW, NB, E4M3>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(kern), 160 * 1024, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)((a.n_out + 16 * RT - 1) / (16 * RT))), dim3(64 * KW), bytes, s, a);
  return hipGetLastError();
}

template <int GROUP, int NT, bool E4M3>
static hipError_t go_proj(ProjArgs& a, hipStream_t s) {
  if (a.n_out >= 128 * 256) return go_many<GROUP, NT, 2, E4M3>(a, s);          // a workgroup or more of 128 rows per compute unit
  return go_split<GROUP, NT, 1, 4, 2, E4M3>(a, s);
}

template <int GROUP>
static hipError_t go_proj(ProjArgs& a, bool e4m3, hipStream_t s) {
  if (a.T <= 16) return e4m3 ? go_proj<GROUP, 1, true>(a, s) : go_proj<GROUP, 1, false>(a, s);
  return e4m3 ? go_proj<GROUP, 2, true>(a, s) : go_proj<GROUP, 2, false>(a, s);
}

hipError_t launch_proj_w4(const mohge_proj_config& c, const void* x, const float* x_scale, const void* codes,
                          const void* scales, const void* zeros, void* y, hipStream_t s) {
  ProjArgs a;
  a.x = x; a.x_scale = x_scale; a.codes = static_cast<const unsigned char*>(codes);
  a.scales = static_cast<const uint16_t*>(scales); a.zeros = static_cast<const unsigned char*>(zeros); a.y = y;
  a.T = c.T; a.n_in = c.n_in; a.n_out = c.n_out; a.f32 = c.y_dtype == MOHGE_F32;
  const bool e4m3 = c.x_dtype == MOHGE_E4M3;
  return c.group == 128 ? go_proj<128>(a, e4m3, s) : c.group == 64 ? go_proj<64>(a, e4m3, s) : go_proj<32>(a, e4m3, s);
}

}  // namespace mohge
