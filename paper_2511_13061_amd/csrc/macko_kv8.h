// Layout of the 8-bit key/value cache, shared by the kernels that fill it and those that read it.
//
// Blocks of 16 tokens of one key/value head lie one after the other: [page][head][block of the page].  A block of D channels is 32 D bytes,
//   key codes    [16][D]      a lane of the matrix instruction takes 16 channels of "its" token as they lie
//   value codes  [4][D][4]    [token / 4][channel][token % 4]: a lane finds 4 tokens of "its" channels together, 4 channels in 16 bytes
// and has two bytes of scale in an array of their own, keys' and values': a code stands for its number times 2^(b - 127), 1 <= b <= 246.
// A byte of scale belongs to 16 tokens: a block is written by one group of lanes, which sees all of a call's tokens for it.
#pragma once

#include "macko_kv.h"

namespace macko {

constexpr int kBlockTokens = 16, kBlockBits = 4;
constexpr uint32_t kMostScale = 246;     // 448 * 2^119 is a number in bf16 and in 32 bits, 256 * 2^120 is not
constexpr float kMostCode = 448.f;

struct Kv8Pool {
  uint8_t* codes;
  uint8_t* scales;
  int64_t pages;
  int32_t heads;             // key/value heads
  int32_t dim;
  int32_t page_bits;         // log2(page_size)
};

// The block of the pool that holds token `at` of a page.
__host__ __device__ inline int64_t kv8_block(const Kv8Pool& p, int64_t page, int head, int at) {
  return ((page * p.heads + head) << (p.page_bits - kBlockBits)) + (at >> kBlockBits);
}

// The byte of a block whose largest finite magnitude has these bits: 448 is 1.75 * 2^8, and a mantissa above 1.75 carries.
__device__ inline uint32_t scale_byte(uint32_t bits) {
  const uint32_t e = (bits + 0x1FFFFFu) >> 23;
  return e > 8u ? min(e - 8u, kMostScale) : 1u;
}
__device__ inline float power_of(uint32_t byte) { return __builtin_bit_cast(float, byte ? byte << 23 : 0x00400000u); }      // 2^-127 too

// Four codes of a word as 32-bit numbers, and back (to nearest, ties to even, 448 at most).
typedef float F2 __attribute__((ext_vector_type(2)));
__device__ inline void numbers_of(uint32_t word, float* x) {
  const F2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true);
  x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
}
__device__ inline uint32_t codes_of(const float* x) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -kMostCode, kMostCode);
  int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true);
}

// A 4 x 4 matrix of bytes, a row in each word, turned over.
__device__ inline void turn_words(const uint32_t (&r)[4], uint32_t (&c)[4]) {
  const uint32_t ab_lo = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), ab_hi = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);      // a0 b0 a1 b1, a2 b2 a3 b3
  const uint32_t cd_lo = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), cd_hi = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
  c[0] = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x05040100u);
  c[1] = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x07060302u);
  c[2] = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x05040100u);
  c[3] = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x07060302u);
}

}  // namespace macko
