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
//                       (It makes a group's sums several times the result, at no bias: for x and weights of one sign, the worst case, with
//                       groups of 128 the errors are at most 6e-7 of the sum of |w x|, their mean below 2e-8 of it.)
//   sums of x           a product with ones gives sum_{k in g} x_tk in the lanes that need it.
//   groups              one product reduces 8 codes of each of four lanes; with groups of 128 those are in one group as
//                       loaded, for 64 and 32 the lanes exchange words first (v_permlane32_swap, v_permlane16_swap).
#include <type_traits>

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

constexpr int proj_batch(int group, int nt) { return (group == 32 ? 2 : 4) / nt; }      // (what the registers hold)

struct ProjArgs {
  const void* x;
  const float* x_scale;
  const unsigned char* codes;
  const uint16_t* scales;
  const unsigned char* zeros;
  void* y;
  int T, n_in, n_out, f32;
};

// A unit is 128 indices (64 bytes) of a weight row; U units are requested, staged and multiplied together.

// U units of the rows of x on their way to LDS: pieces of 8 elements, requested by N threads, P each, and later put there as bf16 in
// the order 0 4 1 5 2 6 3 7.  What depends on the thread alone is worked out once.
template <bool E4M3, int U, int N, int P>
struct Staged {
  static constexpr int kPitch = U * 256 + 16, kUnit = E4M3 ? 128 : 256;          // bytes of a unit of a row in LDS with 16 to spare, in x
  typedef typename std::conditional<E4M3, uint2, uint4>::type Piece8;
  Piece8 d[P];
  uint32_t from[P];          // byte in x of the piece of unit 0
  int to[P];                 // byte in LDS, or -1
  __device__ __forceinline__ void init(const ProjArgs& a, const int thread) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int i = thread + N * j, t = i / (U * 16), p = i % (U * 16);
      to[j] = t < a.T ? t * kPitch + 16 * p : -1;
      from[j] = (uint32_t)(min(t, a.T - 1) * a.n_in + 8 * p) * (E4M3 ? 1u : 2u);
    }
  }
  // units from u0 on, all within the rows
  __device__ __forceinline__ void request(const ProjArgs& a, const int u0) {
    const unsigned char* base = static_cast<const unsigned char*>(a.x) + u0 * kUnit;
#pragma unroll
    for (int j = 0; j < P; ++j) d[j] = *reinterpret_cast<const Piece8*>(base + from[j]);
  }
  // the same where the rows end within the units: zero past them
  __device__ __forceinline__ void request_last(const ProjArgs& a, const int u0) {
    const unsigned char* base = static_cast<const unsigned char*>(a.x) + u0 * kUnit;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      d[j] = Piece8();
      const int p = ((to[j] >= 0 ? to[j] : 0) % kPitch) / 16;
      if (to[j] >= 0 && u0 * 128 + 8 * p < a.n_in) d[j] = *reinterpret_cast<const Piece8*>(base + from[j]);
    }
  }
  __device__ __forceinline__ void put(unsigned char* lds) const {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      uint4 o;
      if constexpr (E4M3) {                                // exact: the upper halves of the fp32 patterns
        const auto u0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[j].x, false), u1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[j].x, true);
        const auto v0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[j].y, false), v1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[j].y, true);
        o = make_uint4(__builtin_amdgcn_perm(__float_as_uint(v0[0]), __float_as_uint(u0[0]), 0x07060302u),
                       __builtin_amdgcn_perm(__float_as_uint(v0[1]), __float_as_uint(u0[1]), 0x07060302u),
                       __builtin_amdgcn_perm(__float_as_uint(v1[0]), __float_as_uint(u1[0]), 0x07060302u),
                       __builtin_amdgcn_perm(__float_as_uint(v1[1]), __float_as_uint(u1[1]), 0x07060302u));
      } else {
        o = make_uint4(__builtin_amdgcn_perm(d[j].z, d[j].x, 0x05040100u), __builtin_amdgcn_perm(d[j].z, d[j].x, 0x07060302u),
                       __builtin_amdgcn_perm(d[j].w, d[j].y, 0x05040100u), __builtin_amdgcn_perm(d[j].w, d[j].y, 0x07060302u));
      }
      if (to[j] >= 0) *reinterpret_cast<uint4*>(lds + to[j]) = o;
    }
  }
};

// RT blocks of 16 weight rows: the codes of U units with their scales and zero points
template <int GROUP, int RT, int U, bool Z>
struct Batch {
  static constexpr int kPer = 128 / GROUP;             // groups in a unit
  uint4 w[RT][U];
  uint32_t s[RT][(U * kPer + 1) / 2];                   // bf16 pairs
  uint32_t z[RT][(U * kPer + 3) / 4];                   // up to four bytes each

  // units u0 .. u0 + U - 1, all within the row.  (No condition anywhere: the same number of loads every time, so that the waits
  // for the batch before can be counted instead of waiting for everything.)
  __device__ __forceinline__ void load(const ProjArgs& a, const int (&row)[RT], int u0, int q) {
    const int groups = a.n_in / GROUP, g0 = u0 * kPer;
#pragma unroll
    for (int f = 0; f < RT; ++f) {
      const unsigned char* cp = a.codes + (long long)row[f] * (a.n_in / 2) + u0 * 64 + 16 * q;
#pragma unroll
      for (int u = 0; u < U; ++u) w[f][u] = *reinterpret_cast<const uint4*>(cp + 64 * u);
      __builtin_memcpy(s[f], a.scales + (long long)row[f] * groups + g0, 2 * U * kPer);          // (rows need not be aligned)
      if constexpr (Z) __builtin_memcpy(z[f], a.zeros + (long long)row[f] * groups + g0, U * kPer);
    }
  }
  // the last units, those before `end`: codes, scales and zero points of the others are 0
  __device__ __forceinline__ void load_last(const ProjArgs& a, const int (&row)[RT], int u0, int end, int q) {
    const int groups = a.n_in / GROUP;
#pragma unroll
    for (int f = 0; f < RT; ++f) {
      const unsigned char* cp = a.codes + (long long)row[f] * (a.n_in / 2);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (u0 + u) * 64 + 16 * q;
        w[f][u] = make_uint4(0u, 0u, 0u, 0u);
        if (u0 + u < end && k < a.n_in / 2) w[f][u] = *reinterpret_cast<const uint4*>(cp + k);
      }
#pragma unroll
      for (int i = 0; i < (U * kPer + 1) / 2; ++i) s[f][i] = 0u;
#pragma unroll
      for (int i = 0; i < (U * kPer + 3) / 4; ++i) z[f][i] = 0u;
#pragma unroll
      for (int i = 0; i < U * kPer; ++i) {
        const int g = u0 * kPer + i;
        if (g < end * kPer && g < groups) {
          s[f][i / 2] |= (uint32_t)a.scales[(long long)row[f] * groups + g] << (16 * (i & 1));
          if constexpr (Z) z[f][i / 4] |= (uint32_t)a.zeros[(long long)row[f] * groups + g] << (8 * (i & 3));
        }
      }
    }
  }
};

// acc += unit u of the batch; x: LDS address of the unit in row 16 t + m of x
template <int GROUP, int RT, int NT, int U, bool Z>
__device__ __forceinline__ void multiply(const Batch<GROUP, RT, U, Z>& b, const int u, const unsigned char* const (&x)[NT], const int q,
                                         f32x4 (&acc)[RT][NT]) {
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
      float z = 24.f;
      if constexpr (Z) z = 16.f + (float)((b.z[f][at / 4] >> (8 * (at & 3))) & 255u);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[f][t][i] = fmaf(s, fmaf(-z, sx[t][i], part[f][t][i]), acc[f][t][i]);
    }
  }
}

// A sum straight from its definition
template <int GROUP, bool Z, bool E4M3>
__device__ __forceinline__ float direct_sum(const ProjArgs& a, const int r, const int n) {
  const int groups = a.n_in / GROUP;
  float sum = 0.f;
#pragma unroll 1
  for (int g = 0; g < groups; ++g) {
    const long long at = (long long)n * groups + g;
    const uint32_t* codes = reinterpret_cast<const uint32_t*>(a.codes) + at * (GROUP / 8);
    float z = 8.f, part = 0.f;
    if constexpr (Z) z = (float)a.zeros[at];
#pragma unroll 1
    for (int i = 0; i < GROUP / 8; ++i) {
      const long long piece = ((long long)r * a.n_in + g * GROUP) / 8 + i;
      float x[8];
      if constexpr (E4M3) {
        const uint2 d = static_cast<const uint2*>(a.x)[piece];
        const auto u0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)d.x, false), u1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)d.x, true);
        const auto v0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)d.y, false), v1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)d.y, true);
        x[0] = u0[0]; x[1] = u0[1]; x[2] = u1[0]; x[3] = u1[1]; x[4] = v0[0]; x[5] = v0[1]; x[6] = v1[0]; x[7] = v1[1];
      } else {
        Piece<true> p;
        p.load(a.x, piece);
        p.get(x);
      }
      const uint32_t c = codes[i];
#pragma unroll
      for (int j = 0; j < 8; ++j) part = fmaf((float)((c >> (4 * j)) & 15u) - z, x[j], part);
    }
    sum = fmaf(__uint_as_float((uint32_t)a.scales[at] << 16), part, sum);
    if (sum != sum) break;                        // NaN stays
  }
  return sum;
}

// Sums that are not finite are worked out again: the offset of 16 in front of the codes turns an infinite x into NaN, and overflows for
// numbers that the definition's products still hold.  (Calls without such sums take as long
// as without this; 32 rows, 65001 x 4096 45 us, with an infinite number in one row 0.3 ms.)
template <int GROUP, bool Z, bool E4M3, int RT, int NT>
__device__ __forceinline__ void store_rows(const ProjArgs& a, const int n0, const int m, const int q, const f32x4 (&acc)[RT][NT]) {
  unsigned again = 0;
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
            if (!(fabsf(acc[f][t][i]) < INFINITY)) again |= 1u << ((t * 4 + i) * RT + f);
          }
        }
      }
    }
  while (again) {
    const int e = __builtin_ctz(again), r = 16 * (e / (4 * RT)) + 4 * q + e / RT % 4, n = n0 + 16 * (e % RT) + m;
    again &= again - 1;
    float sum = direct_sum<GROUP, Z, E4M3>(a, r, n);
    if constexpr (E4M3) sum *= a.x_scale[r];
    const long long at = (long long)r * a.n_out + n;
    if (a.f32) static_cast<float*>(a.y)[at] = sum;
    else static_cast<uint16_t*>(a.y)[at] = (uint16_t)pack_bf16x2(sum, 0.f);
  }
}

// Few weight rows: a workgroup has 16 of them, its KW waves a part of the reduction each.  A wave stages its own part of x, U
// units at a time and without a barrier.
// P pieces of x per lane.
template <int GROUP, int NT, int KW, int U, int P, bool Z, bool E4M3>
__global__ void __launch_bounds__(64 * KW) proj_w4_split_kernel(const ProjArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int kPitch = U * 256 + 16;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const int row[1] = {min(n0 + m, a.n_out - 1)};
  const int nu = (a.n_in + 127) / 128, ub = nu * w / KW, ue = nu * (w + 1) / KW;
  unsigned char* const mine = lds + w * a.T * kPitch;
  const unsigned char* xrow[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) xrow[t] = mine + min(16 * t + m, a.T - 1) * kPitch;
  Staged<E4M3, U, 64, P> x;
  x.init(a, lane);
  auto put = [&]() {
    x.put(mine);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  f32x4 acc[1][NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[0][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  Batch<GROUP, 1, U, Z> cur, next;
  auto compute = [&]() {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned char* at[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) at[t] = xrow[t] + u * 256;
      multiply<GROUP, 1, NT, U, Z>(cur, u, at, q, acc);
    }
  };
  // whole batches, then one that is cut short
  const int whole = min(ue, a.n_in / 128), n = whole > ub ? (whole - ub) / U : 0;
  int u0 = ub;
  auto turn = [&]() {
    compute();
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    put();
    cur = next;
    u0 += U;
  };
  if (ub < ue) {                                 // what is waited for first is requested first
    if (n > 0) {
      x.request(a, ub);
      cur.load(a, row, ub, q);
    } else {
      x.request_last(a, ub);
      cur.load_last(a, row, ub, ue, q);
    }
    put();
    for (int i = 1; i < n; ++i) {
      x.request(a, u0 + U);
      next.load(a, row, u0 + U, q);
      turn();
    }
    if (n > 0 && u0 + U < ue) {
      x.request_last(a, u0 + U);
      next.load_last(a, row, u0 + U, ue, q);
      turn();
    }
    compute();
  }
  // the waves' sums, added in their order
  __syncthreads();
  f32x4* red = reinterpret_cast<f32x4*>(lds);
  if (w > 0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) red[((w - 1) * NT + t) * 64 + lane] = acc[0][t];
  }
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int x = 0; x < KW - 1; ++x)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[0][t] += red[(x * NT + t) * 64 + lane];
  store_rows<GROUP, Z, E4M3, 1, NT>(a, n0, m, q, acc);
}

// Many weight rows: every wave has 16 RT of its own and the whole reduction; the workgroup's waves share the staged rows of x, U units
// in LDS while the next are on the way.  P pieces of x per thread.
template <int GROUP, int NT, int RT, int P, bool Z, bool E4M3>
__global__ void __launch_bounds__(256, 2) proj_w4_kernel(const ProjArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int U = proj_batch(GROUP, NT), kPitch = U * 256 + 16;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int n0 = (blockIdx.x * 4 + w) * 16 * RT;
  int row[RT];
#pragma unroll
  for (int f = 0; f < RT; ++f) row[f] = min(n0 + 16 * f + m, a.n_out - 1);
  const int nu = (a.n_in + 127) / 128;
  Staged<E4M3, U, 256, P> x;
  x.init(a, threadIdx.x);
  f32x4 acc[RT][NT];
#pragma unroll
  for (int f = 0; f < RT; ++f)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  Batch<GROUP, RT, U, Z> cur, next;
  auto compute = [&](const unsigned char* from) {
    const unsigned char* xrow[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) xrow[t] = from + min(16 * t + m, a.T - 1) * kPitch;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned char* at[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) at[t] = xrow[t] + u * 256;
      multiply<GROUP, RT, NT, U, Z>(cur, u, at, q, acc);
    }
  };
  // whole batches, then one that is cut short
  const int n = a.n_in / (128 * U);
  unsigned char *from = lds, *to = lds + a.T * kPitch;
  int u0 = 0;
  auto turn = [&]() {
    compute(from);
    x.put(to);
    __syncthreads();                      // everybody has read `from`, which is written next
    cur = next;
    unsigned char* const was = from;
    from = to;
    to = was;
    u0 += U;
  };
  if (n > 0) {
    x.request(a, 0);
    cur.load(a, row, 0, q);
  } else {
    x.request_last(a, 0);
    cur.load_last(a, row, 0, nu, q);
  }
  x.put(lds);
  __syncthreads();
  for (int i = 1; i < n; ++i) {
    x.request(a, u0 + U);
    next.load(a, row, u0 + U, q);
    turn();
  }
  if (n > 0 && u0 + U < nu) {
    x.request_last(a, u0 + U);
    next.load_last(a, row, u0 + U, nu, q);
    turn();
  }
  compute(from);
  store_rows<GROUP, Z, E4M3, RT, NT>(a, n0, m, q, acc);
}

template <int GROUP, int NT, int RT, int P, bool Z, bool E4M3>
static hipError_t go_many(const ProjArgs& a, hipStream_t s) {
  static std::atomic<unsigned long long> allowed;
  constexpr int kPitch = proj_batch(GROUP, NT) * 256 + 16;
  auto kern = proj_w4_kernel<GROUP, NT, RT, P, Z, E4M3>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(kern), 2 * 32 * kPitch, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)((a.n_out + 64 * RT - 1) / (64 * RT))), dim3(256), 2 * a.T * kPitch, s, a);
  return hipGetLastError();
}

template <int GROUP, int NT, int KW, int U, int P, bool Z, bool E4M3>
static hipError_t go_split(const ProjArgs& a, hipStream_t s) {
  static std::atomic<unsigned long long> allowed;
  constexpr int kPitch = U * 256 + 16;
  int bytes = KW * a.T * kPitch;
  if (bytes < (KW - 1) * NT * 64 * 16) bytes = (KW - 1) * NT * 64 * 16;
  auto kern = proj_w4_split_kernel<GROUP, NT, KW, U, P, Z, E4M3>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(kern), KW * 16 * NT * kPitch, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)((a.n_out + 15) / 16)), dim3(64 * KW), bytes, s, a);
  return hipGetLastError();
}

// The form by size, each against the next best where the line is drawn (us; groups of 128, bf16 x; 32 rows: groups of 64 with zero points):
//   shared staging      up to 4 rows of x never (65001 x 4096, one row: 26.8 split, 27.6); above, from 80 weight rows per compute unit on:
//                       16 rows, 24576 x 4096 16.7 against 18.0, 12288 x 4096 15.6 against 10.9; 32 rows 27.6 against 33.8, 26.2 against 19.4.
//                       Two blocks of 16 weight rows per wave where one would not fit the machine at once: 32 rows, 65001 x 4096 47.8 against
//                       67.1, 49152 x 4096 45.6 against 42.3.
//   eight waves along   where there are units enough and few weight rows or long ones: 4096 x 4096 5.1 against 5.7 (16 rows), 8.7 against 10.0
//   the reduction       (32); 12288 x 1024 4.4 against 3.5 (one row).
//   units per batch     as many as the registers for x leave: one row, 24576 x 4096 11.6 with four, 13.2 with two.
template <int GROUP, bool Z, bool E4M3>
static hipError_t go_proj(const ProjArgs& a, hipStream_t s) {
  const int nu = (a.n_in + 127) / 128;
  if (a.T > 4 && a.n_out >= 80 * 256) {
    constexpr int P = proj_batch(GROUP, 1), P2 = proj_batch(GROUP, 2) * 2;          // pieces of x per thread for 16 and for 32 rows
    if (a.n_out <= 3 * 64 * 256) return a.T <= 16 ? go_many<GROUP, 1, 1, P, Z, E4M3>(a, s) : go_many<GROUP, 2, 1, P2, Z, E4M3>(a, s);
    return a.T <= 16 ? go_many<GROUP, 1, 2, P, Z, E4M3>(a, s) : go_many<GROUP, 2, 2, P2, Z, E4M3>(a, s);
  }
  if (nu >= 64 || (nu >= 32 && a.n_out <= 16 * 256)) {
    if (a.T <= 4) return go_split<GROUP, 1, 8, 4, 4, Z, E4M3>(a, s);
    if (a.T <= 8) return go_split<GROUP, 1, 8, 2, 4, Z, E4M3>(a, s);
    return a.T <= 16 ? go_split<GROUP, 1, 8, 2, 8, Z, E4M3>(a, s) : go_split<GROUP, 2, 8, 1, 8, Z, E4M3>(a, s);
  }
  if (a.T <= 4 && nu >= 16) return go_split<GROUP, 1, 4, 4, 4, Z, E4M3>(a, s);
  if (a.T <= 8) return go_split<GROUP, 1, 4, 2, 4, Z, E4M3>(a, s);
  return a.T <= 16 ? go_split<GROUP, 1, 4, 2, 8, Z, E4M3>(a, s) : go_split<GROUP, 2, 4, 1, 8, Z, E4M3>(a, s);
}

template <int GROUP>
static hipError_t go_proj(const ProjArgs& a, bool e4m3, hipStream_t s) {
  if (a.zeros) return e4m3 ? go_proj<GROUP, true, true>(a, s) : go_proj<GROUP, true, false>(a, s);
  return e4m3 ? go_proj<GROUP, false, true>(a, s) : go_proj<GROUP, false, false>(a, s);
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
