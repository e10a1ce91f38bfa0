// Attention of one new token per sequence over a paged cache, for gfx950.
//   s_j = scale q.k_j over the n positions of the sequence, out = sum_j softmax(s)_j v_j, lse = log sum_j exp s_j
// Bound by memory: every key and value is read once, by the wave that multiplies it, straight into the operand
// registers of the matrix cores; nothing passes through LDS but the join of a workgroup's waves.
//
// A wave takes 32 positions at a time (two halves of 16, each inside one page), for up to 16 query heads of one kv
// head.  Lane (m, q) = (lane & 15, lane >> 4):
//   scores    S^T = K Q^T: the keys are the first operand, lane (m, q) holds pieces of key m; the result leaves
//             the lane with the scores of positions 4q..4q+3 of query head m, in either half;
//   softmax   running maximum and sum per query head; everything a lane has belongs to head m, so the rescaling of
//             its sums needs no other lane, and the maximum two exchanges;
//   values    O^T = V^T P^T: the weights are already where the second operand wants them (positions 4q..4q+3, head m);
//             lane (m, q) loads rows 4q..4q+3 of V, elements m D/16 .. (m+1) D/16 - 1, in one access per row, and turns
//             two rows into pairs by v_perm.  Result j of the lane is element (D/16) (4q + i) + j of head m's output.
// The weights are split into two bf16 parts (the rest after the first is below 2^-17 of it), which costs one more
// product and keeps them as good as fp32: one bf16 rounding of them would be as large as the output's own.
// fp32 caches go through the fp32 matrix cores (16x16x4) with the same assignment, four positions at a time.
#include "block.h"

namespace mohge {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

enum { kCacheF32 = 0, kCacheBf16 = 1, kCacheE4m3 = 2 };

constexpr int kAttWaves = 4;
constexpr float kLog2e = 1.44269504088896340736f;

struct AttArgs {
  const void* q;
  long long q_stride;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const void* k_pages;
  const void* v_pages;
  const float* k_scale;
  const float* v_scale;
  void* out;
  float* lse;
  float* part_o;              // [pieces][rows][D]
  float2* part_ml;            // [pieces][rows]: maximum (of s log2 e) and sum
  float scale2;               // scale * log2 e
  int n_seqs, n_heads, n_kv, group, page_shift, n_pages, max_pages, splits, chunk;
};

__device__ __forceinline__ uint32_t cvt_bf16x2(uint32_t codes, bool hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 r = hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, true)
                      : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, false);
  return __builtin_bit_cast(uint32_t, r);
}

union AttFrag {
  uint4 u;
  uint32_t w[4];
  bf16x8 v;
};

// N bytes (4, 8 or multiples of 16) at p into words
template <int N>
__device__ __forceinline__ void load_bytes(uint32_t* w, const unsigned char* p) {
  if constexpr (N == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (N == 8) {
    const uint2 t = *reinterpret_cast<const uint2*>(p);
    w[0] = t.x; w[1] = t.y;
  } else {
#pragma unroll
    for (int i = 0; i < N / 16; ++i) {
      const uint4 t = *reinterpret_cast<const uint4*>(p + 16 * i);
      w[4 * i] = t.x; w[4 * i + 1] = t.y; w[4 * i + 2] = t.z; w[4 * i + 3] = t.w;
    }
  }
}

template <int CACHE, int D>
struct AttTile {
  static constexpr int kBytes = CACHE == kCacheF32 ? 4 : CACHE == kCacheBf16 ? 2 : 1;
  static constexpr int kRow = D * kBytes;
  static constexpr int kKeyLoads = kRow / 64;             // 16 bytes per lane each, 64 bytes of a key's row
  static constexpr int kValBytes = kRow / 16;             // bytes of a value row per lane
  static constexpr int kQWords = CACHE == kCacheF32 ? D / 4 : D / 8;       // words of the query operand per lane

  uint32_t k[2][kKeyLoads * 4];
  uint32_t v[2][4][kValBytes / 4];
  float ks[2][4], vs[2][4];

  // half hf of the tile lies in the page row `at` (rows of the page array)
  __device__ __forceinline__ void load(int hf, const AttArgs& a, long long at, int lane) {
    const int m = lane & 15, q = lane >> 4;
    const unsigned char* kp = static_cast<const unsigned char*>(a.k_pages) + (at + m) * kRow + 16 * q;
#pragma unroll
    for (int i = 0; i < kKeyLoads; ++i) load_bytes<16>(&k[hf][4 * i], kp + 64 * i);
    const unsigned char* vp = static_cast<const unsigned char*>(a.v_pages) + (at + 4 * q) * kRow + m * kValBytes;
#pragma unroll
    for (int i = 0; i < 4; ++i) load_bytes<kValBytes>(v[hf][i], vp + i * kRow);
    if constexpr (CACHE == kCacheE4m3) {
      load_bytes<16>(reinterpret_cast<uint32_t*>(ks[hf]), reinterpret_cast<const unsigned char*>(a.k_scale + at + 4 * q));
      load_bytes<16>(reinterpret_cast<uint32_t*>(vs[hf]), reinterpret_cast<const unsigned char*>(a.v_scale + at + 4 * q));
    }
  }

  // scores of positions 4q..4q+3 of half hf
  __device__ __forceinline__ f32x4 scores(int hf, const uint32_t (&qw)[kQWords]) const {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kKeyLoads; ++i) {
      if constexpr (CACHE == kCacheF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[hf][4 * i + e]), __uint_as_float(qw[4 * i + e]), s, 0, 0, 0);
      } else if constexpr (CACHE == kCacheBf16) {
        AttFrag kf, qf;
#pragma unroll
        for (int e = 0; e < 4; ++e) { kf.w[e] = k[hf][4 * i + e]; qf.w[e] = qw[4 * i + e]; }
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf.v, qf.v, s, 0, 0, 0);
      } else {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          AttFrag kf, qf;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            kf.w[e] = cvt_bf16x2(k[hf][4 * i + 2 * p + (e >> 1)], e & 1);
            qf.w[e] = qw[8 * i + 4 * p + e];
          }
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf.v, qf.v, s, 0, 0, 0);
        }
      }
    }
    if constexpr (CACHE == kCacheE4m3) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] *= ks[hf][i];
    }
    return s;
  }

  // rows of V past the sequence's end hold anything: their weight is 0, and 0 times NaN is not
  __device__ __forceinline__ void clear_values(int hf, int i) {
#pragma unroll
    for (int w = 0; w < kValBytes / 4; ++w) v[hf][i][w] = 0u;
    if constexpr (CACHE == kCacheE4m3) vs[hf][i] = 0.f;
  }

  // o += V^T p for both halves
  __device__ __forceinline__ void values(f32x4 (&o)[D / 16], const float (&p)[2][4]) const {
    if constexpr (CACHE == kCacheF32) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
            o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[hf][i][j]), p[hf][i], o[j], 0, 0, 0);
    } else {
      AttFrag hi, lo;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          float a = p[hf][i], b = p[hf][i + 1];
          if constexpr (CACHE == kCacheE4m3) { a *= vs[hf][i]; b *= vs[hf][i + 1]; }
          const uint32_t w = pack_bf16x2(a, b);
          hi.w[2 * hf + i / 2] = w;
          lo.w[2 * hf + i / 2] = pack_bf16x2(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
        }
#pragma unroll
      for (int jj = 0; jj < D / 32; ++jj) {                  // elements 2jj and 2jj + 1
        AttFrag f0, f1;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint32_t r[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (CACHE == kCacheBf16) r[i] = v[hf][i][jj];
            else r[i] = cvt_bf16x2(v[hf][i][jj >> 1], jj & 1);
          }
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            f0.w[2 * hf + i / 2] = __builtin_amdgcn_perm(r[i + 1], r[i], 0x05040100u);
            f1.w[2 * hf + i / 2] = __builtin_amdgcn_perm(r[i + 1], r[i], 0x07060302u);
          }
        }
        o[2 * jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0.v, hi.v, o[2 * jj], 0, 0, 0);
        o[2 * jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0.v, lo.v, o[2 * jj], 0, 0, 0);
        o[2 * jj + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1.v, hi.v, o[2 * jj + 1], 0, 0, 0);
        o[2 * jj + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1.v, lo.v, o[2 * jj + 1], 0, 0, 0);
      }
    }
  }
};

// The query operand of head m (zero for heads past the group)
template <int CACHE, int D, int W>
__device__ __forceinline__ void load_query(uint32_t (&qw)[W], const AttArgs& a, long long at, bool there, int q) {
#pragma unroll
  for (int i = 0; i < W; ++i) qw[i] = 0u;
  if (!there) return;
  if constexpr (CACHE == kCacheF32) {
    const float* p = static_cast<const float*>(a.q) + at + 4 * q;          // elements 16 i + 4 q ..
#pragma unroll
    for (int i = 0; i < W / 4; ++i) load_bytes<16>(&qw[4 * i], reinterpret_cast<const unsigned char*>(p + 16 * i));
  } else if constexpr (CACHE == kCacheBf16) {
    const uint16_t* p = static_cast<const uint16_t*>(a.q) + at + 8 * q;    // elements 32 i + 8 q ..
#pragma unroll
    for (int i = 0; i < W / 4; ++i) load_bytes<16>(&qw[4 * i], reinterpret_cast<const unsigned char*>(p + 32 * i));
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(a.q) + at + 16 * q;   // elements 64 i + 16 q ..
#pragma unroll
    for (int i = 0; i < W / 8; ++i) load_bytes<32>(&qw[8 * i], reinterpret_cast<const unsigned char*>(p + 64 * i));
  }
}

template <int CACHE>
__device__ __forceinline__ void store_out(void* out, long long at, const float* v) {       // 4 elements
  if constexpr (CACHE == kCacheF32)
    *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(v[0], v[1], v[2], v[3]);
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// grid: sequences x kv heads x blocks of 16 query heads x splits
template <int CACHE, int D>
__global__ void __launch_bounds__(64 * kAttWaves) cache_attention_kernel(const AttArgs a) {
  typedef AttTile<CACHE, D> Tile;
  __shared__ float red_o[kAttWaves - 1][D / 4][64];
  __shared__ float red_ml[kAttWaves - 1][2][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int blocks = (a.group + 15) / 16;
  const int split = blockIdx.x % a.splits, row = blockIdx.x / a.splits;
  const int b = row / (a.n_kv * blocks), kv = row / blocks % a.n_kv, g0 = row % blocks * 16;
  const bool there = g0 + m < a.group;
  const int head = kv * a.group + g0 + m;
  const int S = 1 << a.page_shift;
  const int n = a.seq_lens[b];
  const int len = min(n, a.max_pages << a.page_shift);
  int bad = n > len;
  const int begin = split * a.chunk, end = len - begin < a.chunk ? len : begin + a.chunk;
  if (split > 0 && begin >= len) return;            // (the join takes the pieces that the length has)
  const int32_t* table = a.block_table + (long long)b * a.max_pages;

  uint32_t qw[Tile::kQWords];
  load_query<CACHE, D>(qw, a, b * a.q_stride + (long long)head * D, there, q);
  f32x4 o[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, sum = 0.f;

  for (int t0 = begin + 32 * w; t0 < end; t0 += 32 * kAttWaves) {
    Tile tile;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int h0 = t0 + 16 * hf < end ? t0 + 16 * hf : t0;        // a half past the end: read again, and masked
      int page = table[h0 >> a.page_shift];
      if ((unsigned)page >= (unsigned)a.n_pages) { page = 0; bad = 1; }
      tile.load(hf, a, (((long long)page * a.n_kv + kv) << a.page_shift) + (h0 & (S - 1)), lane);
    }
    float s[2][4];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const f32x4 z = tile.scores(hf, qw);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[hf][i] = z[i] * a.scale2;
    }
    if (t0 + 32 > end) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + 16 * hf + 4 * q + i >= end) {
            s[hf][i] = -INFINITY;
            tile.clear_values(hf, i);
          }
    }
    float next = top;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int i = 0; i < 4; ++i) next = fmaxf(next, s[hf][i]);
    next = fmaxf(next, __shfl_xor(next, 16, 64));
    next = fmaxf(next, __shfl_xor(next, 32, 64));
    const float ref = next == -INFINITY ? 0.f : next;
    const float shrink = __builtin_amdgcn_exp2f(top - ref);
    top = next;
    float p[2][4];
    sum *= shrink;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[hf][i] = __builtin_amdgcn_exp2f(s[hf][i] - ref);
        sum += p[hf][i];
      }
#pragma unroll
    for (int j = 0; j < D / 16; ++j) o[j] *= shrink;
    tile.values(o, p);
  }
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);

  // join of the waves, in their order
  if (bad) sum = NAN;
  if (w > 0) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) red_o[w - 1][4 * j + i][lane] = o[j][i];
    red_ml[w - 1][0][lane] = top;
    red_ml[w - 1][1][lane] = sum;
  }
  __syncthreads();
  if (w > 0) return;
  float all = top;
#pragma unroll
  for (int x = 0; x < kAttWaves - 1; ++x) all = fmaxf(all, red_ml[x][0][lane]);
  const float ref = all == -INFINITY ? 0.f : all;
  float f = __builtin_amdgcn_exp2f(top - ref);
  sum *= f;
#pragma unroll
  for (int j = 0; j < D / 16; ++j) o[j] *= f;
#pragma unroll
  for (int x = 0; x < kAttWaves - 1; ++x) {
    f = __builtin_amdgcn_exp2f(red_ml[x][0][lane] - ref);
    sum = fmaf(f, red_ml[x][1][lane], sum);
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j][i] = fmaf(f, red_o[x][4 * j + i][lane], o[j][i]);
  }
  if (!there) return;
  // element (D/16) (4q + i) + j: D/16 in a row for every i
  if (len <= a.chunk) {
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : NAN;
    const long long at = ((long long)b * a.n_heads + head) * D + (D / 4) * q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; j += 4) {
        const float r[4] = {o[j][i] * inv, o[j + 1][i] * inv, o[j + 2][i] * inv, o[j + 3][i] * inv};
        store_out<CACHE>(a.out, at + (D / 16) * i + j, r);
      }
    if (a.lse && q == 0) a.lse[(long long)b * a.n_heads + head] = (ref + log2f(sum)) * (1.f / kLog2e);
  } else {
    const long long piece = ((long long)b * a.n_heads + head) * a.splits + split;
    float* to = a.part_o + piece * D + (D / 4) * q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; j += 4)
        *reinterpret_cast<float4*>(to + (D / 16) * i + j) = make_float4(o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]);
    if (q == 0) a.part_ml[piece] = make_float2(all, sum);
  }
}

// The pieces of one (sequence, head), joined in their order: D/4 threads with 4 elements each
template <int CACHE, int D>
__global__ void __launch_bounds__(64) cache_attention_join_kernel(const AttArgs a) {
  const int row = blockIdx.x, b = row / a.n_heads;
  const int len = min(a.seq_lens[b], a.max_pages << a.page_shift);
  if (len <= a.chunk) return;
  const int pieces = (len + a.chunk - 1) / a.chunk;
  const float2* ml = a.part_ml + (long long)row * a.splits;
  const float* po = a.part_o + (long long)row * a.splits * D;
  float all = -INFINITY;
  for (int p = 0; p < pieces; ++p) all = fmaxf(all, ml[p].x);
  const float ref = all == -INFINITY ? 0.f : all;
  float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  const int e = threadIdx.x * 4;
  if (e >= D) return;
  for (int p = 0; p < pieces; ++p) {
    const float f = __builtin_amdgcn_exp2f(ml[p].x - ref);
    const float4 v = *reinterpret_cast<const float4*>(po + (long long)p * D + e);
    sum = fmaf(f, ml[p].y, sum);
    o[0] = fmaf(f, v.x, o[0]); o[1] = fmaf(f, v.y, o[1]); o[2] = fmaf(f, v.z, o[2]); o[3] = fmaf(f, v.w, o[3]);
  }
  const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : NAN;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] *= inv;
  store_out<CACHE>(a.out, (long long)row * D + e, o);
  if (a.lse && threadIdx.x == 0) a.lse[row] = (ref + log2f(sum)) * (1.f / kLog2e);
}

// Pieces of `chunk` positions per sequence
static void cache_splits(const mohge_cache_config& c, int& splits, int& chunk) {
  const int step = 32 * kAttWaves;
  const int longest = c.max_pages * c.page_size;
  const long long rows = (long long)(c.n_seqs > 0 ? c.n_seqs : 1) * c.n_kv_heads * ((c.n_heads / c.n_kv_heads + 15) / 16);
  long long want = (1024 + rows - 1) / rows;
  const long long most = (longest + step - 1) / step;
  if (want > most) want = most;
  if (want < 1) want = 1;
  chunk = (int)((longest + want - 1) / want);
  chunk = (chunk + step - 1) / step * step;
  splits = (longest + chunk - 1) / chunk;
}

size_t cache_workspace_bytes(const mohge_cache_config& c) {
  int splits, chunk;
  cache_splits(c, splits, chunk);
  const size_t pieces = (size_t)c.n_seqs * c.n_heads * splits;
  return splits > 1 ? pieces * (c.head_size * sizeof(float) + sizeof(float2)) : 0;
}

template <int CACHE, int D>
static void go_attention(const AttArgs& a, hipStream_t s) {
  const int blocks = (a.group + 15) / 16;
  hipLaunchKernelGGL((cache_attention_kernel<CACHE, D>), dim3((unsigned)(a.n_seqs * a.n_kv * blocks * a.splits)), dim3(64 * kAttWaves), 0,
                     s, a);
  if (a.splits > 1)
    hipLaunchKernelGGL((cache_attention_join_kernel<CACHE, D>), dim3(a.n_seqs * a.n_heads), dim3(64), 0, s, a);
}

template <int CACHE>
static void go_attention(const AttArgs& a, int D, hipStream_t s) {
  if (D == 64) go_attention<CACHE, 64>(a, s);
  else if (D == 128) go_attention<CACHE, 128>(a, s);
  else go_attention<CACHE, 256>(a, s);
}

hipError_t launch_cache_attention(const mohge_cache_config& c, const void* q, long long q_stride,
                                  const int32_t* block_table, const int32_t* seq_lens, const void* k_pages,
                                  const void* v_pages, const float* k_scale, const float* v_scale, float scale,
                                  void* out, float* lse, void* ws, hipStream_t s) {
  AttArgs a;
  a.q = q; a.q_stride = q_stride; a.block_table = block_table; a.seq_lens = seq_lens;
  a.k_pages = k_pages; a.v_pages = v_pages; a.k_scale = k_scale; a.v_scale = v_scale;
  a.out = out; a.lse = lse; a.scale2 = scale * kLog2e;
  a.n_seqs = c.n_seqs; a.n_heads = c.n_heads; a.n_kv = c.n_kv_heads; a.group = c.n_heads / c.n_kv_heads;
  a.page_shift = log2_of(c.page_size); a.n_pages = c.n_pages; a.max_pages = c.max_pages;
  cache_splits(c, a.splits, a.chunk);
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + (size_t)c.n_seqs * c.n_heads * a.splits * c.head_size);
  if (c.cache_dtype == MOHGE_F32) go_attention<kCacheF32>(a, c.head_size, s);
  else if (c.cache_dtype == MOHGE_BF16) go_attention<kCacheBf16>(a, c.head_size, s);
  else go_attention<kCacheE4m3>(a, c.head_size, s);
  return hipGetLastError();
}

}  // namespace mohge
