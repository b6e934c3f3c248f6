// What the kernels of the attention over the 8-bit cache share.  Sequences, rows, spans of tokens, parts and their join are those of the 4-bit cache's attention.
#pragma once

#include "macko_kv8.h"
#include "macko_kv_attention.h"

namespace macko {

struct Kv8Attention {
  KvAttention a;             // pool.data: the codes
  const uint8_t* scales;
};

struct Launch8 {
  KvAttention a;
  Grid g;
  const uint8_t* scales;
};

int64_t kv8_attention_workspace(const KvAttention& a);       // floats
int launch_kv8_attention(const Kv8Attention& a, float* workspace, hipStream_t stream);
// (macko_kv8_prompt.hip) many rows, in blocks of g.rows
int launch_kv8_rows(const Launch8& l, hipStream_t stream);

// The sequence whose rows hold `row`: the last one that starts there or before (`batch`: behind them all, -1: in front).  64 starts at a time.
__device__ inline int sequence_at(const int32_t* start, int batch, int row, int lane) {
  int lo = 0, count = batch + 1;                          // the last of [lo, lo + count) that is at most `row`
  while (count > 1) {
    const int step = (count + 63) / 64, at = min(lane * step, count - 1);
    const uint64_t before = __ballot(start[lo + at] <= row && lane * step < count);
    if (before == 0) return -1;
    const int steps = __popcll(before) - 1;
    lo += steps * step;
    count = min(step, count - steps * step);
  }
  return lo;
}

template <int W>
__device__ inline void load_words(uint32_t* to, const uint8_t* from) {
  typedef uint32_t Words __attribute__((ext_vector_type(W)));
  const Words w = *reinterpret_cast<const Words*>(from);
#pragma unroll
  for (int i = 0; i < W; ++i) to[i] = w[i];
}

// The same in all lanes: in a scalar register.
__device__ inline float scalar(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }

// Two neighbouring codes of a word as a pair of 16 bits, times a power of two of which the conversion looks at the exponent alone.
template <bool BF>
__device__ inline int pair_of(uint32_t word, float unit, bool high) {
  if (BF) return __builtin_bit_cast(int, (B2)(high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, unit, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, unit, false)));
  return __builtin_bit_cast(int, (H2)(high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, unit, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, unit, false)));
}
// Eight codes as the matrix instruction's operand.
template <bool BF>
__device__ inline V4i operand_of(uint32_t lo, uint32_t hi, float unit) {
  return V4i{pair_of<BF>(lo, unit, false), pair_of<BF>(lo, unit, true), pair_of<BF>(hi, unit, false), pair_of<BF>(hi, unit, true)};
}
// A byte of ones for every byte of a word of codes that is not a number.
__device__ inline uint32_t not_numbers(uint32_t word) {
  const uint32_t x = (word & 0x7F7F7F7Fu) + 0x01010101u;      // carries stay in their bytes: 0x7F + 1
  return (x & 0x80808080u) >> 7;
}

}  // namespace macko
