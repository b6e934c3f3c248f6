// What the kernels of the attention over the 4-bit cache share.
#pragma once

#include <type_traits>

#include "macko_kv.h"

namespace macko {

typedef int V8i __attribute__((ext_vector_type(8)));
typedef int V4i __attribute__((ext_vector_type(4)));
typedef float V4f __attribute__((ext_vector_type(4)));
typedef __bf16 B2 __attribute__((ext_vector_type(2)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef _Float16 H2 __attribute__((ext_vector_type(2)));
typedef _Float16 H8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4, kTile = 32, kMostSplits = 256;
constexpr int kMostTokens = 1 << 30;                  // of a sequence: sums of a length and a launch's steps stay in 31 bits
constexpr uint32_t kNoNumber = 253; // a group of values with this byte or a higher one may read as infinite in bf16 and in 32 bits, with 255 it is NaN
constexpr float kLift = 8.f;       // how far, in powers of two, a score may pass the running maximum before that moves

struct Grid {
  int32_t row_blocks, splits;      // of a sequence's rows and of its tokens, at most
  int32_t rows, unit;              // rows of a block; tokens that a workgroup goes on by
  int32_t ordered;                 // long sequences first
  uint32_t shared_inverse;         // 2^32 / a.shared, rounded up; 0 for 1
  int64_t chunk;                   // tokens of a split, at least; a multiple of unit
  float* parts;                    // [tokens * heads][splits][D], then [tokens * heads][splits][2]: maximum and sum, then used_splits
};

// How many splits the tokens of a row are in, written with the first of them: [tokens * heads].
template <class A, class G>
__device__ inline int32_t* used_splits(const A& a, const G& g) {
  return reinterpret_cast<int32_t*>(g.parts + a.tokens * a.heads * g.splits * (a.pool.dim + 2));
}

struct Launch {
  KvAttention a;
  Grid g;
};
typedef const __attribute__((address_space(4))) Launch* LaunchPtr;

// Read through the scalar cache: nothing writes them while a kernel runs.
__device__ inline int32_t constant(const int32_t* p) { return *(const __attribute__((address_space(4))) int32_t*)p; }

struct Sequence {
  int length, first, queries, rows;
};
__device__ inline Sequence sequence_of(const KvAttention& a, int b) {
  Sequence s;
  s.length = min(max(0, constant(a.lengths + b)), kMostTokens);
  s.first = a.start ? min(max(constant(a.start + b), 0), (int)a.tokens) : b;
  s.queries = a.start ? min(max(constant(a.start + b + 1), s.first), (int)a.tokens) - s.first : 1;
  s.rows = s.queries * a.shared;
  return s;
}

// Rows of a block: row r belongs to query r / shared.  Behind the first one's the quotient is small, and exact as a product (shared is at most 2^15).
struct Rows {
  int first, query;                // the block's first row, and its query
  __device__ int query_of(const KvAttention& a, const Grid& g, int row) const {
    const uint32_t more = (uint32_t)(row - query * a.shared);
    return query + (int)(g.shared_inverse ? __umulhi(more, g.shared_inverse) : more);
  }
};
__device__ inline Rows rows_of(const KvAttention& a, int first_row) { return Rows{first_row, first_row == 0 ? 0 : first_row / a.shared}; }

// The tokens that the rows of a block see, and how they are split.
struct Span {
  int first, lo, hi, chunk, used;  // [first, hi); lo: first, down to a multiple of 16
  int all_lo, all_hi;              // every row of the block sees [all_lo, all_hi)
};
__device__ inline Span span_of(const KvAttention& a, const Grid& g, const Sequence& s, const Rows& rows) {
  Span p;
  const int qa = rows.query, qb = rows.query_of(a, g, min(rows.first + g.rows - 1, s.rows - 1)), offset = s.length - s.queries;
  p.hi = min(max(offset + qb + 1, 0), s.length);
  p.all_hi = min(max(offset + qa + 1, 0), s.length);
  const int lo = a.window ? max(offset + qa - a.window + 1, 0) : 0;
  p.all_lo = a.window ? max(offset + qb - a.window + 1, 0) : 0;
  p.first = min(lo, p.hi);
  p.lo = p.first & ~15;
  p.chunk = kMostTokens;
  p.used = 1;
  if (g.splits > 1) {
    const int range = max(p.hi - p.lo, 0);
    p.chunk = (int)g.chunk;
    if ((int64_t)p.chunk * g.splits < range) p.chunk = (int)(((unsigned)range + g.splits * g.unit - 1) / (unsigned)(g.splits * g.unit)) * g.unit;      // longer than was said
    p.used = max(1, (int)(((unsigned)range + p.chunk - 1) / (unsigned)p.chunk));
  }
  return p;
}

__device__ inline int later(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The sequence that is n-th by length, longest first (at most 64 of them): workgroups start in this order, and the last ones to end are short (64
// sequences of 1024 to 4096 tokens: 143 us, 148 as they come).
__device__ inline int nth_longest(const KvAttention& a, int n, int lane) {
  const int key = lane < a.batch ? min(max(a.lengths[lane], 0), (1 << 25) - 1) * 64 + 63 - lane : -1;
  int longer = 0;
#pragma unroll
  for (int m = 0; m < 64; ++m) longer += __builtin_amdgcn_readlane(key, m) > key;
  return __builtin_ctzll(__ballot(longer == n && lane < a.batch));
}

// Four values as 8-bit numbers, and 16 times what they leave over in their place.
__device__ inline int part_of(float* x) {
  int word = 0;
  word = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], word, false);
  word = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], word, true);
  x[0] = (x[0] - __builtin_amdgcn_cvt_f32_fp8(word, 0)) * 16.f;
  x[1] = (x[1] - __builtin_amdgcn_cvt_f32_fp8(word, 1)) * 16.f;
  x[2] = (x[2] - __builtin_amdgcn_cvt_f32_fp8(word, 2)) * 16.f;
  x[3] = (x[3] - __builtin_amdgcn_cvt_f32_fp8(word, 3)) * 16.f;
  return word;
}

// Lane (n, j) = lane % 16, lane / 16 of the queries' operand for one tile of rows: row n, 8-bit parts, each 16 times what the one before left over, and a
// byte of scale for each part.  `src`: the row's channels, read where `there`.
template <int NG, bool BF>
__device__ inline void load_queries(const uint16_t* src, bool there, float sign, int n, int j, V8i (&q)[(NG + 3) / 4][BF ? 2 : 3], int (&q_byte)[(NG + 3) / 4]) {
  constexpr int D = 32 * NG, NK = (NG + 3) / 4, NP = BF ? 2 : 3;
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) {
    float x[2][16];
    uint32_t top[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {                     // a lane's channels of the operand: 16 in each half of 128
      const int channel = kk * 128 + u * 64 + j * 16;
      Packed8 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
      if (there && channel < D) {
        lo = *reinterpret_cast<const Packed8Any*>(src + channel);
        hi = *reinterpret_cast<const Packed8Any*>(src + channel + 8);
      }
      unpack8<BF>(lo, x[u]);
      unpack8<BF>(hi, x[u] + 8);
      uint32_t most = 0;                              // magnitudes are ordered as their bits are, infinities and NaN above all
#pragma unroll
      for (int i = 0; i < 16; ++i) most = max(most, __builtin_bit_cast(uint32_t, x[u][i]) & 0x7FFFFFFFu);
      most = max(most, (uint32_t)__shfl_xor((int)most, 16));      // two lanes share a group
      top[u] = max(most >> 23, 20u) - 7u;             // largest magnitude to [128, 256)
      const float up = __builtin_bit_cast(float, (254u - top[u]) << 23) * sign;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[u][i] *= up;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
#pragma unroll
        for (int w = 0; w < 4; ++w) q[kk][p][u * 4 + w] = part_of(x[u] + 4 * w);
      }
    }
    // lane j gives the scale of group j: groups 0 and 1 are those of lanes 0 and 2 (first half), 2 and 3 of the second
    const int from = n + 32 * (j & 1), t0 = __shfl((int)top[0], from), t1 = __shfl((int)top[1], from);
    const int t = j < 2 ? t0 : t1;
    q_byte[kk] = t | (t - 4) << 8 | (t - 8) << 16;
  }
}

// Two values of one token, channels 32g + m and 32g + 16 + m, in 16 bits each: fp16 (HALF) or bf16.
template <bool HALF, int BYTE>
__device__ inline uint32_t decode_pair(uint32_t word, uint32_t bytes) {
  // the conversion looks at the exponent field of its scale alone
  const uint32_t unit = BYTE == 0 ? bytes << 23 : BYTE == 1 ? bytes << 15 : BYTE == 2 ? bytes << 7 : bytes >> 1;
  if (HALF) return __builtin_bit_cast(uint32_t, (H2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, __builtin_bit_cast(float, unit), BYTE));
  return __builtin_bit_cast(uint32_t, (B2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, __builtin_bit_cast(float, unit), BYTE));
}
template <bool HALF>
__device__ inline uint32_t decode_at(uint32_t word, uint32_t bytes, int at) {
  switch (at) {
    case 0: return decode_pair<HALF, 0>(word, bytes);
    case 1: return decode_pair<HALF, 1>(word, bytes);
    case 2: return decode_pair<HALF, 2>(word, bytes);
    default: return decode_pair<HALF, 3>(word, bytes);
  }
}
template <bool HALF>
__device__ inline V4f multiply(V4i a, V4i b, V4f c) {
  if (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, a), __builtin_bit_cast(H8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
}
// Weights as a first part and what it leaves over.
template <bool HALF>
__device__ inline void parts_of(const float* w, V4i& hi, V4i& lo) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float w0 = w[2 * i], w1 = w[2 * i + 1];
    if (HALF) {
      // what is left over comes from the pair as it is packed: one instruction a weight that takes half of a register as it is and rounds what it gives
      float less = -1.f;
      asm("" : "+s"(less));                              // (a plain difference is made of three)
      const int pair = later(__builtin_bit_cast(int, H2{(_Float16)w0, (_Float16)w1}));
      const H2 h = __builtin_bit_cast(H2, pair);
      hi[i] = pair;
      lo[i] = __builtin_bit_cast(int, H2{(_Float16)__builtin_fmaf((float)h[0], less, w0), (_Float16)__builtin_fmaf((float)h[1], less, w1)});
    } else {
      // cut off, not rounded: that takes no instruction but the one that joins two of them
      const uint32_t b0 = __builtin_bit_cast(uint32_t, w0), b1 = __builtin_bit_cast(uint32_t, w1);
      const B2 l = {(__bf16)(w0 - __builtin_bit_cast(float, b0 & 0xFFFF0000u)), (__bf16)(w1 - __builtin_bit_cast(float, b1 & 0xFFFF0000u))};
      hi[i] = (int)__builtin_amdgcn_perm(b1, b0, 0x07060302u);
      lo[i] = __builtin_bit_cast(int, l);
    }
  }
}

// (macko_kv_prompt.hip) many rows
int launch_prompt(const KvAttention& a, const Grid& g, hipStream_t stream);
int prompt_row_tiles(int dim);       // of a wavefront there

}  // namespace macko
