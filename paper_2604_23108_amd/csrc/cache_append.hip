// New keys and values into the pages of a cache, for gfx950: token i of the n new ones of a sequence of (now) len positions goes to
// position len - n + i, with an E4M3 cache as codes of x / scale, scale = max |x| (1 / 448) over the token's row of one head.
// Bound by memory: every thread takes 8 elements of one (token, head) row of the keys and of the values, requests them, and looks up
// where they go meanwhile (a chain of loads: the token's sequence, its length, its page); with an E4M3 cache the threads of a row
// fold its largest magnitude before they convert.  9003 tokens of 8 heads of 128 to 8 bits 13.5 us, 4.2 TB/s; 5023 of 4 heads of
// 256 as they are 8.5 us, 4.8 TB/s; one token for each of 32 sequences 2.1 us, a launch.
#include "block.h"

namespace mohge {

// 8 elements of a row to the pages: as they are, or as codes with a scale for the per_row threads (8, 16 or 32) of the row
template <bool BF16, bool E4M3>
__device__ __forceinline__ void store_piece(const Piece<BF16>& a, void* pages, float* scales, long long at, int per_row, int piece) {
  if constexpr (E4M3) {
    float x[8], top = 0.f;
    a.get(x);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[j]));
    for (int off = per_row >> 1; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const float scale = e4m3_scale(top), inv = 1.f / scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= inv;
    static_cast<uint2*>(pages)[at * per_row + piece] = to_e4m3x8(x);
    if (piece == 0) scales[at] = scale;
  } else {
    a.store(pages, at * per_row + piece);
  }
}

// Where token t goes: the row of the page array of its first head, negative if nowhere
__device__ __forceinline__ long long token_place(const mohge_cache_config& c, const int t, const int32_t* __restrict__ tok_offsets,
                                                 const int32_t* __restrict__ block_table, const int32_t* __restrict__ seq_lens,
                                                 const int page_shift) {
  // the sequence: the last one whose first row is not behind this one
  int b = t, after = 1;
  if (tok_offsets) {
    int lo = 0, hi = c.n_seqs;                      // tok_offsets[lo] <= t < tok_offsets[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tok_offsets[mid] <= t) lo = mid;
      else hi = mid;
    }
    b = lo;
    after = tok_offsets[b + 1] - t;
  }
  const int pos = seq_lens[b] - after;
  const int col = pos >> page_shift;
  if (after < 1 || pos < 0 || col >= c.max_pages) return -1;
  const int page = block_table[(long long)b * c.max_pages + col];
  if ((unsigned)page >= (unsigned)c.n_pages) return -1;
  return (((long long)page * c.n_kv_heads) << page_shift) + (pos & (c.page_size - 1));
}

template <bool BF16, bool E4M3>
__global__ void __launch_bounds__(256) cache_append_kernel(
    const mohge_cache_config c, const int n_tokens, const void* __restrict__ k, const long long k_stride,
    const void* __restrict__ v, const long long v_stride, const int32_t* __restrict__ tok_offsets,
    const int32_t* __restrict__ block_table, const int32_t* __restrict__ seq_lens, void* k_pages, void* v_pages,
    float* k_scale, float* v_scale, const int page_shift) {
  const int per_row = c.head_size / 8, per_token = c.n_kv_heads * per_row;
  const unsigned idx = blockIdx.x * 256u + threadIdx.x;          // (fewer than 2^31 pieces)
  const int t = (int)(idx / (unsigned)per_token), rest = (int)(idx % (unsigned)per_token);
  if (t >= n_tokens) return;                       // whole rows: per_row divides the wave
  const int head = rest / per_row, piece = rest % per_row;
  Piece<BF16> ka, va;
  ka.load(k, t * k_stride / 8 + rest);
  va.load(v, t * v_stride / 8 + rest);
  // a wave with one token looks it up with scalar loads (9003 tokens to 8 bits 15.9 us without, 13.5 with)
  const int t0 = __builtin_amdgcn_readfirstlane(t);
  long long at = __ballot(t != t0) == 0 ? token_place(c, t0, tok_offsets, block_table, seq_lens, page_shift)
                                        : token_place(c, t, tok_offsets, block_table, seq_lens, page_shift);
  if (at < 0) return;
  at += (long long)head << page_shift;
  store_piece<BF16, E4M3>(ka, k_pages, k_scale, at, per_row, piece);
  store_piece<BF16, E4M3>(va, v_pages, v_scale, at, per_row, piece);
}

hipError_t launch_cache_append(const mohge_cache_config& c, int n_tokens, const void* k, long long k_stride,
                               const void* v, long long v_stride, const int32_t* tok_offsets,
                               const int32_t* block_table, const int32_t* seq_lens, void* k_pages, void* v_pages,
                               float* k_scale, float* v_scale, hipStream_t s) {
  const long long threads = (long long)n_tokens * c.n_kv_heads * (c.head_size / 8);
  const dim3 grid((unsigned)((threads + 255) / 256));
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, c, n_tokens, k, k_stride, v, v_stride, tok_offsets, block_table,
                       seq_lens, k_pages, v_pages, k_scale, v_scale, log2_of(c.page_size));
  };
  if (c.dtype == MOHGE_F32) go(cache_append_kernel<false, false>);
  else if (c.cache_dtype == MOHGE_E4M3) go(cache_append_kernel<true, true>);
  else go(cache_append_kernel<true, false>);
  return hipGetLastError();
}

}  // namespace mohge
