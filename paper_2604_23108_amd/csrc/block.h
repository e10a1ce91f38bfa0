// Internal declarations of the operators around the layer (mohge_block.h), shared by their host entry points
// and kernel files.
#pragma once
#include "common.h"
#include "mohge_block.h"

namespace mohge {

hipError_t launch_rmsnorm(const mohge_norm_config& c, const void* x, const void* residual, const float* weight,
                          void* sum_out, void* y, float* y_scale, float* rstd, hipStream_t s);
size_t norm_workspace_bytes(const mohge_norm_config& c);
hipError_t launch_rmsnorm_bwd(const mohge_norm_config& c, const void* dy, const void* h, const float* weight,
                              const float* rstd, const void* dsum, void* dx, float* dweight, void* ws, hipStream_t s);

hipError_t launch_cache_append(const mohge_cache_config& c, int n_tokens, const void* k, long long k_stride,
                               const void* v, long long v_stride, const int32_t* tok_offsets,
                               const int32_t* block_table, const int32_t* seq_lens, void* k_pages, void* v_pages,
                               float* k_scale, float* v_scale, hipStream_t s);
size_t cache_workspace_bytes(const mohge_cache_config& c);
hipError_t launch_cache_attention(const mohge_cache_config& c, const void* q, long long q_stride,
                                  const int32_t* block_table, const int32_t* seq_lens, const void* k_pages,
                                  const void* v_pages, const float* k_scale, const float* v_scale, float scale,
                                  void* out, float* lse, void* ws, hipStream_t s);

hipError_t launch_proj_w4(const mohge_proj_config& c, const void* x, const float* x_scale, const void* codes,
                          const void* scales, const void* zeros, void* y, hipStream_t s);

// log2 of a power of two
inline int log2_of(int v) {
  int n = 0;
  while ((1 << n) < v) ++n;
  return n;
}

// Scale of a row of E4M3 codes whose largest magnitude is amax; its reciprocal, by which the row is multiplied, is finite.  (For bf16 rows
// the codes are those of the quotients x / scale as well, for each of the 128 x 128 pairs of mantissas; exact steps to the quotient cost
// 0.7 us of 13 where 9003 tokens are appended, and change nothing.)
__device__ __forceinline__ float e4m3_scale(float amax) {
  return amax == 0.f ? 1.f : fmaxf(amax * (1.f / 448.f), 1.17549435e-38f);
}

// 8 floats -> 8 E4M3 codes, rounded to nearest even
__device__ __forceinline__ uint2 to_e4m3x8(const float (&v)[8]) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
  return make_uint2((unsigned)lo, (unsigned)hi);
}

// 8 consecutive elements: bf16 (one 16-byte access) or fp32 (two)
template <bool BF16>
struct Piece {
  uint4 u[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* base, long long piece) {
    const uint4* p = static_cast<const uint4*>(base) + piece * (BF16 ? 1 : 2);
    u[0] = p[0];
    if constexpr (!BF16) u[1] = p[1];
  }
  __device__ __forceinline__ void store(void* base, long long piece) const {
    uint4* p = static_cast<uint4*>(base) + piece * (BF16 ? 1 : 2);
    p[0] = u[0];
    if constexpr (!BF16) p[1] = u[1];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    if constexpr (BF16) {
      const uint32_t w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    } else {
      v[0] = __uint_as_float(u[0].x); v[1] = __uint_as_float(u[0].y);
      v[2] = __uint_as_float(u[0].z); v[3] = __uint_as_float(u[0].w);
      v[4] = __uint_as_float(u[1].x); v[5] = __uint_as_float(u[1].y);
      v[6] = __uint_as_float(u[1].z); v[7] = __uint_as_float(u[1].w);
    }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    if constexpr (BF16) {
      u[0] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                        pack_bf16x2(v[6], v[7]));
    } else {
      u[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      u[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    }
  }
};

}  // namespace mohge
