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
// product: one bf16 rounding of them would be as large as the output's own.  (32 ragged sequences up to 8191: 280 of 131072 bf16 outputs are not
// the rounded exact value, 62 to 94 where everything is fp32.)
// fp32 caches go through the fp32 matrix cores (16x16x4) with the same assignment, four positions at a time.
//
// Work split: the positions of every (sequence, kv head, block of 16 query heads) are cut into units of four tiles, one for each wave (128
// positions, or 64 where a tile is one half), and the units of all of them, in one row, into equal stretches, one for each workgroup that
// the machine holds at once: whatever the lengths, every workgroup has about the same number of units.  The stretches follow from
// the lengths, which every workgroup reads for itself.  A row that lies in several stretches leaves parts (sums, maximum and total)
// in the workspace, and the workgroup that finishes last joins them in their order: how many parts there are depends on the
// lengths alone, so equal calls have equal results.
//
// Measured (us; TB/s of keys and values; bf16, 32 query heads over 8 kv heads of 128, pages of 16): 32 sequences of 4096 97..100, 5.4;
// 32 of 0..8191 112, 4.8; two of some 115000, 8 bits, 104, 4.7; one of 1531 (16 over 4 heads of 64) 7.6.  The loads alone, without any
// arithmetic on what they bring, take as long (99.7, 116 for 117, 7.5): the kernel is bound by its reads, and short calls by a launch and a
// chain of five dependent accesses (length, page, tile, part and counter, parts).
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
  unsigned long long* done;   // [rows]: parts of a row that are complete, in units of part_unit; 0 between calls
  float2* part_o;             // [2 per workgroup][D / 8][4][heads of a row]: pairs of a lane's elements, lane after lane
  float2* part_ml;            // [2 per workgroup][heads of a row]: maximum (of s log2 e) and sum
  float scale2;               // scale * log2 e
  int n_seqs, n_heads, n_kv, group, page_shift, n_pages, max_pages;
};

__device__ __forceinline__ uint32_t cvt_bf16x2(uint32_t codes, bool hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 r = hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, true)
                      : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, false);
  return __builtin_bit_cast(uint32_t, r);
}

typedef short bf16x4 __attribute__((ext_vector_type(4)));

union AttFrag {
  uint4 u;
  uint32_t w[4];
  bf16x8 v;
  bf16x4 half;
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

// Halves of 16 positions in a tile.  One where two would leave the registers to a single wave per SIMD (us with two and with one, 32
// query heads over 8 kv heads): E4M3 of 256, 128 sequences of up to 300 positions 47.5 and 35.1, 32 of up to 4096 76 and 67, 32 of
// 4096 105 and 106; fp32 of 128, the same 60 and 47, 113 and 109, 190 and 194.  A bf16 cache of 256 stays with two: 58 and 54, 114 and 122.
constexpr int att_halves(int cache, int d) {
  return cache == kCacheF32 ? (d == 64 ? 2 : 1) : cache == kCacheE4m3 && d == 256 ? 1 : 2;
}

template <int CACHE, int D>
struct AttTile {
  static constexpr int H = att_halves(CACHE, D);
  static constexpr int kBytes = CACHE == kCacheF32 ? 4 : CACHE == kCacheBf16 ? 2 : 1;
  static constexpr int kRow = D * kBytes;
  static constexpr int kKeyLoads = kRow / 64;             // 16 bytes per lane each, 64 bytes of a key's row
  static constexpr int kValBytes = kRow / 16;             // bytes of a value row per lane
  static constexpr int kQWords = CACHE == kCacheF32 ? D / 4 : D / 8;       // words of the query operand per lane

  uint32_t k[H][kKeyLoads * 4];
  uint32_t v[H][4][kValBytes / 4];
  float ks[H][4], vs[H][4];

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

  // V^T p over the positions of the halves (4 or 8 per lane)
  static __device__ __forceinline__ f32x4 product(const AttFrag& v, const AttFrag& p, const f32x4 o) {
    if constexpr (H == 2) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, p.v, o, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v.half, p.half, o, 0, 0, 0);
  }

  // o += V^T p for all halves
  __device__ __forceinline__ void values(f32x4 (&o)[D / 16], const float (&p)[H][4]) const {
    if constexpr (CACHE == kCacheF32) {
#pragma unroll
      for (int hf = 0; hf < H; ++hf)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
            o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[hf][i][j]), p[hf][i], o[j], 0, 0, 0);
    } else {
      AttFrag hi, lo;
#pragma unroll
      for (int hf = 0; hf < H; ++hf)
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
        for (int hf = 0; hf < H; ++hf) {
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
        o[2 * jj] = product(f0, hi, o[2 * jj]);
        o[2 * jj] = product(f0, lo, o[2 * jj]);
        o[2 * jj + 1] = product(f1, hi, o[2 * jj + 1]);
        o[2 * jj + 1] = product(f1, lo, o[2 * jj + 1]);
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

// a / b for a < 2^31, 0 < b
__device__ __forceinline__ int udiv(int a, int b) { return (int)((unsigned)a / (unsigned)b); }

// Units of a sequence: at least one, which writes the result of an empty one
template <int UNIT>
__device__ __forceinline__ int units_of(const AttArgs& a, int b) {
  const int len = min(max(a.seq_lens[b], 0), a.max_pages << a.page_shift);
  return len > 0 ? (len + UNIT - 1) / UNIT : 1;
}

// Stores that go through the XCD's cache, so that a workgroup on any XCD reads them once they are complete
__device__ __forceinline__ void store_through(float2* p, const float2 v) {
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
// ... and loads that see them.  (An acquiring fence instead makes every wave that joins invalidate its XCD's cache.)
__device__ __forceinline__ float2 load_through(const float2* p) {
  return __builtin_bit_cast(float2, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED,
                                                      __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ void store_through(float* p, const float v) {
  __hip_atomic_store(reinterpret_cast<unsigned*>(p), __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Stretches of `per` units begin at multiples of it, except in rows that are short or hardly longer than a stretch: those are not cut, a
// stretch begins at their nearer end.  (A part has to be written, counted and read again: 464 rows of 8 units in stretches of 5 take
// 20.8 us cut and 17.6 whole.  Short are 3 units, or 4 of an 8-bit cache: 128 rows of 4 units 13.3 us cut and 18.3 whole, 8 of 3 units
// 8.4 and 7.5; 32 of 4 units in 8 bits 9.0 and 8.4.)
struct Stretches {
  int per, few;
  __device__ __forceinline__ bool keep_whole(int units) const {
    return units <= few || (units >= per && units <= per + max(1, per / 2));
  }
  // unit v, which is unit `start` of a row of `units`
  __device__ __forceinline__ int begin(int v, int start, int units) const {
    return !keep_whole(units) ? v : 2 * start <= units ? v - start : v + units - start;
  }
  // the stretches that hold the first and the last unit of a row that is cut, which begins at unit r0
  __device__ __forceinline__ int first_of(int r0) const { return udiv(r0, per); }
  __device__ __forceinline__ int last_of(int r0, int units) const { return udiv(r0 + units - 1, per); }
};

// What a part adds to its row's counter: an odd number, whose first 2^24 multiples all lie 2^34 and more away from 0 (mod 2^64), another one for
// another number of parts.  So only a counter that was 0 comes to parts * part_unit(parts), at the last part; from another start (small
// numbers that the memory held, what calls that overlapped left) it does not, in this call or a later one.  Counted by ones, a counter of
// 1 would have parts joined that are not written yet, and be 1 again afterwards.  (2^64 over the golden ratio, and 2^64 (sqrt 2 - 1).)
__device__ __forceinline__ unsigned long long part_unit(int parts) {
  return 0x9e3779b97f4a7c15ull + (unsigned long long)parts * 0x6a09e667f3bcc908ull;
}

// A row of which this workgroup has a part
struct Part {
  int b, row, first, parts;          // sequence, row of it, first workgroup, workgroups
};

template <int CACHE, int D, int OCC>
__global__ void __launch_bounds__(64 * kAttWaves, OCC) cache_attention_kernel(const AttArgs a) {
  typedef AttTile<CACHE, D> Tile;
  constexpr int H = Tile::H, kTile = 16 * H, kUnit = kTile * kAttWaves;
  constexpr int kOutBytes = CACHE == kCacheF32 ? 4 : 2;
  __shared__ float red_o[kAttWaves - 1][D / 4][64];
  __shared__ float red_ml[kAttWaves - 1][2][64];
  __shared__ int last[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, q = lane >> 4;
  const int blocks = (a.group + 15) / 16, rows = a.n_kv * blocks, gmax = min(a.group, 16);
  const int S = 1 << a.page_shift;

  // units of all sequences, and this workgroup's stretch [u, u_end)
  int mine = lane < a.n_seqs ? units_of<kUnit>(a, lane) : 0;          // of sequences base .. base + 63
  int upto = wave_incl_scan(mine), base = 0;
  int total = __builtin_amdgcn_readlane(upto, 63);
  for (int b0 = 64; b0 < a.n_seqs; b0 += 64)
    total += __builtin_amdgcn_readlane(wave_incl_scan(b0 + lane < a.n_seqs ? units_of<kUnit>(a, b0 + lane) : 0), 63);
  total *= rows;
  // (two units at least where rows have 1024 positions in the mean: with one, more parts are joined than it helps)
  Stretches cut;
  cut.few = CACHE == kCacheE4m3 ? 4 : 3;
  cut.per = max(udiv(total + (int)gridDim.x - 1, gridDim.x), total >= 1024ll / kUnit * a.n_seqs * rows ? 2 : 1);
  int before = 0;                                 // units (of one row) in front of sequence `base`
  // the sequence b of unit v (at least as far as the last one asked for), its row, the unit's place in the row
  int b, units, first, row, start;
  auto locate = [&](int v) {
    unsigned long long hit;
    while (!(hit = __ballot((long long)(before + upto) * rows > v))) {
      before += __builtin_amdgcn_readlane(upto, 63);
      base += 64;
      mine = base + lane < a.n_seqs ? units_of<kUnit>(a, base + lane) : 0;
      upto = wave_incl_scan(mine);
    }
    const int at = (int)__builtin_ctzll(hit);
    b = base + at;
    units = __builtin_amdgcn_readlane(mine, at);
    first = (before + __builtin_amdgcn_readlane(upto, at) - units) * rows;          // unit 0 of the sequence's row 0
    row = udiv(v - first, units);
    start = v - first - row * units;
  };
  auto begin_of = [&](int i) {
    if ((long long)i * cut.per >= total) return total;
    locate(i * cut.per);
    return cut.begin(i * cut.per, start, units);
  };
  int u = begin_of(blockIdx.x);
  const int base0 = base, before0 = before, mine0 = mine, upto0 = upto;
  const int u_end = begin_of(blockIdx.x + 1);
  if (u >= u_end) return;
  base = base0; before = before0; mine = mine0; upto = upto0;
  Part part[2];                                   // (the first row and the last one)
  int n_parts = 0;
  const int pitch = 4 * gmax, mine_at = q * gmax + m;
  f32x4 o[D / 16];
  float top, sum;
  // the waves' sums, joined by the first in their order
  auto join_waves = [&]() {
    if (w > 0) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) red_o[w - 1][4 * j + i][lane] = o[j][i];
      red_ml[w - 1][0][lane] = top;
      red_ml[w - 1][1][lane] = sum;
    }
    __syncthreads();
    if (w == 0) {
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
      top = all;
    }
  };
  // lane (m, q) has the elements (D/16) (4q + i) + j of head m: D/16 in a row for every i
  auto finish = [&](long long hd) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;             // (no weight at all: 0; NaN stays)
    const long long to = hd * D + (D / 4) * q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; j += 4) {
        const float r[4] = {o[j][i] * inv, o[j + 1][i] * inv, o[j + 2][i] * inv, o[j + 3][i] * inv};
        store_out<CACHE>(a.out, to + (D / 16) * i + j, r);
      }
    if (a.lse && q == 0) a.lse[hd] = ((top == -INFINITY ? 0.f : top) + log2f(sum)) * (1.f / kLog2e);
  };
  auto clear = [&]() {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    top = -INFINITY;
    sum = 0.f;
  };

  while (u < u_end) {
    locate(u);
    const int n_units = min(units - start, u_end - u);
    const int kv = udiv(row, blocks), g0 = (row - kv * blocks) * 16;
    const bool there = g0 + m < a.group;
    const int head = kv * a.group + g0 + m;
    const int n = a.seq_lens[b];
    const int len = min(max(n, 0), a.max_pages << a.page_shift);
    int bad = n > len;

    const int32_t* table = a.block_table + (long long)b * a.max_pages;
    uint32_t qw[Tile::kQWords];
    load_query<CACHE, D>(qw, a, b * a.q_stride + (long long)head * D, there, q);
    clear();

    // this wave's tiles: kUnit apart from p0 on, those in front of p_end
    const int p0 = start * kUnit + w * kTile, p_end = min(len, (start + n_units) * kUnit);
    const int tiles = p_end > p0 ? (p_end - p0 + kUnit - 1) / kUnit : 0;
    constexpr int kAhead = 64 / H;                 // tiles whose pages a wave looks up together, one half per lane
    int pages = 0;
    auto look_up = [&](int t0) {
      const int pos = p0 + (t0 + lane / H) * kUnit + 16 * (lane % H);
      const bool in = pos < p_end && t0 + lane / H < tiles;
      pages = in ? table[pos >> a.page_shift] : 0;
      if (__ballot((unsigned)pages >= (unsigned)a.n_pages)) bad = 1;
      if ((unsigned)pages >= (unsigned)a.n_pages) pages = 0;
    };
    auto load = [&](Tile& tile, int t) {
#pragma unroll
      for (int hf = 0; hf < H; ++hf) {
        const int pos = p0 + t * kUnit + 16 * hf;
        const int half = pos < p_end ? hf : 0;                    // a half past the end: read the first again, and mask it
        const long long page = __builtin_amdgcn_readlane(pages, (t % kAhead) * H + half);
        tile.load(hf, a, ((page * a.n_kv + kv) << a.page_shift) + ((pos - 16 * (hf - half)) & (S - 1)), lane);
      }
    };
    auto compute = [&](Tile& tile, int t) {
      const int pos = p0 + t * kUnit;
      float s[H][4];
#pragma unroll
      for (int hf = 0; hf < H; ++hf) {
        const f32x4 z = tile.scores(hf, qw);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[hf][i] = z[i] * a.scale2;
      }
      if (pos + kTile > p_end) {
#pragma unroll
        for (int hf = 0; hf < H; ++hf)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (pos + 16 * hf + 4 * q + i >= p_end) {
              s[hf][i] = -INFINITY;
              tile.clear_values(hf, i);
            }
      }
      float next = top;
#pragma unroll
      for (int hf = 0; hf < H; ++hf)
#pragma unroll
        for (int i = 0; i < 4; ++i) next = fmaxf(next, s[hf][i]);
      next = fmaxf(next, __shfl_xor(next, 16, 64));
      next = fmaxf(next, __shfl_xor(next, 32, 64));
      const float ref = next == -INFINITY ? 0.f : next;
      const float shrink = __builtin_amdgcn_exp2f(top - ref);
      top = next;
      sum *= shrink;
      float p[H][4];
#pragma unroll
      for (int hf = 0; hf < H; ++hf)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[hf][i] = __builtin_amdgcn_exp2f(s[hf][i] - ref);
          sum += p[hf][i];
        }
#pragma unroll
      for (int j = 0; j < D / 16; ++j) o[j] *= shrink;
      tile.values(o, p);
    };
    if (tiles > 0) {
      // one tile on the way while the one before is multiplied
      Tile cur, next;
      look_up(0);
      load(cur, 0);
      int t = 0;
      for (; t + 1 < tiles; ++t) {
        if ((t + 1) % kAhead == 0) look_up(t + 1);
        load(next, t + 1);
        compute(cur, t);
        cur = next;
      }
      compute(cur, t);
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (bad) sum = NAN;

    join_waves();
    if (n_units == units) {
      if (w == 0 && there) finish((long long)b * a.n_heads + head);
    } else {
      // A part: pairs of elements, lane after lane (elements of one head after the other would be written 8 bytes here and there:
      // 40 us for 29 sequences of 1000 positions and 256 heads where this took 31)
      const int r0 = first + row * units;
      const Part mine_of = {b, row, cut.first_of(r0), cut.last_of(r0, units) - cut.first_of(r0) + 1};
      part[n_parts > 0] = mine_of;
      ++n_parts;
      if (w == 0 && there) {
        const int slot = 2 * blockIdx.x + (start == 0);
        float2* to = a.part_o + (long long)slot * (D / 8) * pitch + mine_at;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int i = 0; i < 4; i += 2) store_through(to + (2 * j + i / 2) * pitch, make_float2(o[j][i], o[j][i + 1]));
        if (q == 0) store_through(a.part_ml + (long long)slot * gmax + m, make_float2(top, sum));
        // until the parts are joined the result is NaN: if the counters were not 0 at the start, nothing can pass for one
        if (start == 0) {
          const float nan = __uint_as_float(0x7fc07fc0u);          // also as two bf16 numbers
          unsigned char* out = static_cast<unsigned char*>(a.out) + (((long long)b * a.n_heads + head) * D + (D / 4) * q) * kOutBytes;
#pragma unroll
          for (int i = 0; i < D / 4 * kOutBytes; i += 8) store_through(reinterpret_cast<float2*>(out + i), make_float2(nan, nan));
          if (a.lse && q == 0) store_through(a.lse + (long long)b * a.n_heads + head, nan);
        }
      }
    }
    __syncthreads();                        // red_o and red_ml have been read
    u += n_units;
  }
  if (n_parts == 0) return;

  // A row's parts are complete where the last one is counted; that workgroup joins them.  (Counted at the end, when the first part's
  // stores have long arrived.)
  if (w == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (lane < n_parts) {
      const Part p = lane == 0 ? part[0] : part[1];
      unsigned long long* const done = a.done + (long long)p.b * rows + p.row;
      const unsigned long long unit = part_unit(p.parts), all = (unsigned long long)p.parts * unit;
      const bool complete = __hip_atomic_fetch_add(done, unit, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + unit == all;
      if (complete) __hip_atomic_fetch_add(done, 0ull - all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last[lane] = complete;
    }
  }
  __syncthreads();
  for (int k = 0; k < n_parts; ++k) {
    if (!last[k]) continue;
    const Part pt = k == 0 ? part[0] : part[1];
    const int kv = udiv(pt.row, blocks), g0 = (pt.row - kv * blocks) * 16;
    const bool there = g0 + m < a.group;
    // In the order of their workgroups, a fourth for each wave: the first is its workgroup's second slot, the others their first.
    clear();
    const int p_begin = pt.parts * w / kAttWaves, p_last = pt.parts * (w + 1) / kAttWaves;
    auto add = [&](const float2 ml, const float2 (&v)[D / 8]) {
      const float next = fmaxf(top, ml.x), ref = next == -INFINITY ? 0.f : next;
      const float f = __builtin_amdgcn_exp2f(top - ref), g = __builtin_amdgcn_exp2f(ml.x - ref);
      top = next;
      sum = sum * f + ml.y * g;
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          o[j][i] = o[j][i] * f + v[2 * j + i / 2].x * g;
          o[j][i + 1] = o[j][i + 1] * f + v[2 * j + i / 2].y * g;
        }
    };
    if (gmax > 8 || pt.parts <= 3 * kAttWaves) {
#pragma unroll 2
      for (int p = p_begin; p < p_last; ++p) {
        const long long slot = 2 * (pt.first + p) + (p == 0);
        float2 ml = make_float2(-INFINITY, 0.f), v[D / 8];
#pragma unroll
        for (int x = 0; x < D / 8; ++x) v[x] = make_float2(0.f, 0.f);
        if (there) {
          ml = load_through(a.part_ml + slot * gmax + m);
          const float2* from = a.part_o + slot * (D / 8) * pitch + mine_at;
#pragma unroll
          for (int x = 0; x < D / 8; ++x) v[x] = load_through(from + x * pitch);
        }
        add(ml, v);
      }
    } else {
      // Many parts of up to 8 heads: the lanes that the heads leave over take parts as well, lane m has head m mod 2^lg and every (16 >> lg)th
      // part of the wave (32 heads over 8: one sequence of 16000 positions, 63 parts a row, 28 us, 37 with the heads' lanes alone; one
      // of 4000, 16 parts, 11.8 and 12.7; with fewer the exchange at the end takes longer than it saves).  A lane whose part or head is
      // another lane's loads that and counts it with a weight of 0, or nowhere.
      const int lg = gmax > 4 ? 3 : gmax > 2 ? 2 : gmax - 1;
      const int hm = min(m & ((1 << lg) - 1), gmax - 1);
#pragma unroll 2
      for (int p0 = p_begin; p0 < p_last; p0 += 16 >> lg) {
        const int p = min(p0 + (m >> lg), p_last - 1);
        const long long slot = 2 * (pt.first + p) + (p == 0);
        float2 ml = load_through(a.part_ml + slot * gmax + hm), v[D / 8];
        const float2* from = a.part_o + slot * (D / 8) * pitch + q * gmax + hm;
#pragma unroll
        for (int x = 0; x < D / 8; ++x) v[x] = load_through(from + x * pitch);
        if (p0 + (m >> lg) >= p_last) ml = make_float2(-INFINITY, 0.f);
        add(ml, v);
      }
      for (int off = 1 << lg; off < 16; off <<= 1) {
        const float2 ml = make_float2(__shfl_xor(top, off, 64), __shfl_xor(sum, off, 64));
        float2 v[D / 8];
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int i = 0; i < 4; i += 2) v[2 * j + i / 2] = make_float2(__shfl_xor(o[j][i], off, 64), __shfl_xor(o[j][i + 1], off, 64));
        add(ml, v);
      }
    }
    join_waves();
    if (w == 0 && there) finish((long long)pt.b * a.n_heads + kv * a.group + g0 + m);
    __syncthreads();
  }
}

// Waves per SIMD that the registers of a form allow (two tiles and the sums of one)
constexpr int att_waves(int cache, int d) {
  return d == 256 ? (cache == kCacheE4m3 ? 2 : 1) : d == 64 && cache != kCacheF32 ? 3 : 2;
}

static int att_rows(const mohge_cache_config& c) { return c.n_kv_heads * ((c.n_heads / c.n_kv_heads + 15) / 16); }

// Workgroups: as many as are resident at once, no more than there can be units
static int att_groups(const mohge_cache_config& c) {
  const int cache = c.cache_dtype == MOHGE_F32 ? kCacheF32 : c.cache_dtype == MOHGE_BF16 ? kCacheBf16 : kCacheE4m3;
  const int unit = 16 * att_halves(cache, c.head_size) * kAttWaves;
  const long long units = (long long)c.n_seqs * att_rows(c) * (((long long)c.max_pages * c.page_size + unit - 1) / unit);
  const long long most = 256 * att_waves(cache, c.head_size);
  return (int)(units < most ? units : most);
}

static size_t att_done_bytes(const mohge_cache_config& c) { return ((size_t)c.n_seqs * att_rows(c) * sizeof(unsigned long long) + 255) / 256 * 256; }

size_t cache_workspace_bytes(const mohge_cache_config& c) {
  const int group = c.n_heads / c.n_kv_heads, gmax = group < 16 ? group : 16;
  return att_done_bytes(c) + (size_t)att_groups(c) * 2 * gmax * (c.head_size * sizeof(float) + sizeof(float2));
}

template <int CACHE>
static void go_attention(const AttArgs& a, int D, int groups, hipStream_t s) {
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(64 * kAttWaves), 0, s, a); };
  if (D == 64) go(cache_attention_kernel<CACHE, 64, att_waves(CACHE, 64)>);
  else if (D == 128) go(cache_attention_kernel<CACHE, 128, att_waves(CACHE, 128)>);
  else go(cache_attention_kernel<CACHE, 256, att_waves(CACHE, 256)>);
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
  const int groups = att_groups(c), gmax = a.group < 16 ? a.group : 16;
  a.done = static_cast<unsigned long long*>(ws);
  a.part_o = reinterpret_cast<float2*>(static_cast<unsigned char*>(ws) + att_done_bytes(c));
  a.part_ml = a.part_o + (size_t)groups * gmax * c.head_size;
  if (c.cache_dtype == MOHGE_F32) go_attention<kCacheF32>(a, c.head_size, groups, s);
  else if (c.cache_dtype == MOHGE_BF16) go_attention<kCacheBf16>(a, c.head_size, groups, s);
  else go_attention<kCacheE4m3>(a, c.head_size, groups, s);
  return hipGetLastError();
}

}  // namespace mohge
