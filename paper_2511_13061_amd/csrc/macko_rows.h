// Attention of many rows, over keys and values in 16 bits as they lie packed or (PAGED) over the pages of the 8-bit cache: there the matrix cores and the
// vector units are what bounds a step, not memory.
//
// Rows are the queries of one key/value head, token by token and in it head by head.  The four (or eight) wavefronts of a workgroup have 32 rows of their own each and go
// along the tokens together, 64 at a time (32 with wide heads), which all of them bring into LDS in 16 bits while those before are multiplied:
//   scores   S^T = K Q^T by mfma 32x32x16 in the queries' type: products of 16 bits, sums of 32.  Column r of S^T is row r: a lane holds 16 of a row's scores on 32
//            tokens.  A cached block's power of two goes onto its keys (bf16, where it changes nothing but the exponent) or its scores (fp16).
//   weights  2^(score * unit + base), base so that the running maximum is at kTop; it moves only when a weight passes that by kLift, and only then do lanes talk.
//            A row's sum is that of the weights as they go into the products, so that what their rounding does to a row that one token dominates cancels out;
//            sums that a call returns are taken before the rounding.
//   values   O^T += V^T P^T by mfma 32x32x16.  The lanes of S^T that hold a token's weights are those that P^T needs: nothing moves between lanes.
// A wavefront's matrix and vector instructions are in turns in one order: the scores of the next 64 tokens between the weights of these, the maxima of those
// between the values of these.  (One step after the other took 185 us where this took 160: 4096 tokens, 128 channels, 32 heads on 8, fp16; 365 and 327 over the 8-bit cache.)
// Matrix cores (43 % busy) and vector units (42 %), which a wavefront's turns overlap in part alone, bound it, at the clock of the moment (2.2 GHz, and down to 1.7 on a warm card): packed,
// one sequence of 8192 tokens, 32 heads on 8, bf16: 32 channels 244 us (564 TFLOP/s), 64 333 (825), 96 450 (917), 128 543 (1012), 160 750 (916), 192 815 (1013), 224 1550 (620), 256 1556 (707):
// two wavefronts of more than 192 channels do not fit a SIMD's registers; fp16 4 to 9 % longer.  (Another card: 128 channels 620 us.)  1024 queries on each of 2 x 8192 tokens of the 8-bit
// cache, 128 channels: bf16 275 us (940), fp16 285.
// Weights are one part of 16 bits: of bf16 (8 bits, as the results have) for packed bf16, of fp16 else (11 bits from 2^-24 of a row's maximum on), which holds cached values too,
// with the powers of two of their blocks from 2^-15 to 2^6 of a first one's.
// A value that is not finite would reach every row of its step, with weight 0 where it is not seen: a block of rows with results that are not numbers is gone
// through again, carefully: such values are left out of the products and added row by row.  With fp16 weights it is gone through again too where what
// those below fp16's normal numbers have lost may come to half a unit in the last place of a row's largest result, and where cached values do not fit;
// there weights and packed fp16 values are two bf16 parts each.  If every block is: 8192 packed tokens of 128 channels, fp16, 586 us and 1686 with it; 1024 queries on 8192 cached
// tokens 169 and 378 (bf16 164 and 372).
#pragma once

#include "macko_kv8_attention.h"

namespace macko {

typedef float V16f __attribute__((ext_vector_type(16)));
typedef uint32_t U2 __attribute__((ext_vector_type(2)));
typedef short S4 __attribute__((ext_vector_type(4)));

struct LaunchRows {
  KvAttention a;
  Grid g;
  const uint8_t* scales;                                  // PAGED
  const uint16_t *k, *v;                                  // else
  int64_t k_token, k_head, v_token, v_head;
};

// Tokens of a step: what the registers hold of one and the next.
constexpr int row_step(int ng, bool paged, int waves) { return ng > 4 || (ng > 2 && !paged && waves == 4) ? 32 : 64; }

template <bool HALF>
__device__ inline V16f multiply32(V4i a, V4i b, V16f c) {
  if (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(H8, a), __builtin_bit_cast(H8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
}

// Where the 16 bytes `chunk` of a token's channels lie in its row of LDS, so that what is read or written at once lies in different banks (256 bytes of them): 16 bytes of
// each of 16 tokens (keys read), 64 of each of 4 (values read, both written).  Rows that are not a multiple of 256 bytes begin in different banks by themselves.
template <int NG>
__device__ inline int key_chunk(int token, int chunk) {
  return chunk ^ (NG % 4 == 0 ? (token & 3) << 2 | (token >> 2 & 3) : NG % 2 == 0 ? (token & 2) << 1 | (token >> 2 & 3) : token >> 2 & 3);
}
template <int NG>
__device__ inline int value_chunk(int token, int chunk) {
  return chunk ^ (NG % 4 == 0 ? (token & 3) << 2 : NG % 2 == 0 ? (token & 2) << 1 : 0);
}

// 16 lanes read 4 rows of 16 values and get 16 columns of 4.
__device__ inline U2 read_turned(const uint8_t* at) {
  typedef __attribute__((address_space(3))) S4* Lds;
  return __builtin_bit_cast(U2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(__attribute__((address_space(3))) void*)at));
}

// NaN where one of them is.
__device__ inline float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// The two numbers that lane l and lane l ^ 32 have, in both.
struct Halves {
  float low, high;
};
__device__ inline Halves halves_of(float x) {
  const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t low = both[0], high = both[1];
  return Halves{__builtin_bit_cast(float, low), __builtin_bit_cast(float, high)};
}

// The sum of a pair's two numbers and x.
template <bool HALF>
__device__ inline float add_pair(int pair, float x) {
  if (HALF) return __builtin_amdgcn_fdot2(__builtin_bit_cast(H2, pair), H2{(_Float16)1.f, (_Float16)1.f}, x, false);
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(B2, pair), B2{(__bf16)1.f, (__bf16)1.f}, x, false);
}

// One block of rows: sequence b's from first_row on (PAGED: of `split`), or the call's.
template <int NG, bool BF, bool PAGED, int WAVES>
__device__ inline void rows_block(const LaunchRows& args, uint8_t* lds, const Sequence& seq, int b, int head, int split, int first_row) {
  const KvAttention& a = args.a;
  const Grid& g = args.g;
  constexpr int D = 32 * NG, CH = 4 * NG, STEP = row_step(NG, PAGED, WAVES), PARTS = STEP / 32, kRows = 32 * WAVES, kTile = STEP * D * 2;      // bytes of a step's keys, or values
  constexpr bool HALF = !BF || PAGED;                     // weights and values in fp16
  // lds: keys [2], values [2], and below
  uint8_t* const lds_values = lds + 2 * kTile;
  float* const lds_unit = reinterpret_cast<float*>(lds + 4 * kTile);        // [4][4]: of the blocks' keys, four steps' because they are read a step later than the keys
  uint32_t* const lds_odd = reinterpret_cast<uint32_t*>(lds_unit + 16);     // [2]: tokens of a step with values that are not finite
  uint32_t* const lds_word = lds_odd + 2;                                   // [WAVES]

  // worked out for each block of rows anew: kept from one to the next it would hold registers
  const int thread = later(threadIdx.x), wave = __builtin_amdgcn_readfirstlane(thread >> 6), lane = thread & 63, col = lane & 31, h = lane >> 5;
  const float unit = scalar(a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.4426950408889634f);
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : 0xFFFFFFFFu;

  // ---- the block: its rows, the tokens [begin, end) that they see, [all_lo, all_hi) that all of them see
  const int total_rows = PAGED ? seq.rows : (int)a.tokens * a.shared, first_token = PAGED ? seq.first : 0;
  const Rows rows = rows_of(a, first_row);
  const int row = first_row + wave * 32 + col;            // the lane's
  int begin, end, low = 0, all_lo, all_hi;
  int place;                                              // of the row's query: it sees the tokens t with 0 <= place - t < reach
  uint32_t reach;
  Span span{};
  bool bad = false;
  const int32_t* const table = PAGED ? a.tables + b * a.table_stride : nullptr;
  if constexpr (PAGED) {
    span = span_of(a, g, seq, rows);
    if (split >= span.used) return;
    begin = span.lo + split * span.chunk;
    end = span.hi - begin > span.chunk ? begin + span.chunk : span.hi;
    low = span.first;
    all_lo = span.all_lo, all_hi = span.all_hi;
    bad = end > begin && (a.table_width == 0 || a.pool.pages == 0);
    if (bad) end = begin;
    place = row < total_rows ? seq.length - seq.queries + rows.query_of(a, g, row) : -1;
    reach = a.window ? (uint32_t)a.window : 0x7FFFFFFFu;
  } else {
    int t0 = rows.query, t1 = rows.query_of(a, g, min(first_row + kRows, total_rows) - 1), low1 = 0;
    place = row < total_rows ? rows.query_of(a, g, row) : -1;
    reach = place + 1;
    if (a.start) {
      const int s0 = max(sequence_at(a.start, a.batch, t0, lane), 0);
      t0 = max(t0, a.start[0]);
      t1 = min(t1, min(a.start[a.batch], (int)a.tokens) - 1);
      if (t0 > t1) return;
      reach = 0;
      for (int s = s0; s < a.batch; ++s) {
        const int from = a.start[s], to = a.start[s + 1];
        if (from > t1) break;
        if (t0 >= from && t0 < to) low = from;
        if (t1 >= from && t1 < to) low1 = from;
        if (place >= from && place < to) reach = place - from + 1;
      }
    }
    if (a.window) {
      low = max(low, t0 - a.window + 1);
      low1 = max(low1, t1 - a.window + 1);
      reach = min(reach, (uint32_t)a.window);
    }
    low = max(low, 0);
    begin = low, end = t1 + 1, all_lo = low1, all_hi = t0 + 1;
  }
  const int last_block = (end - 1) >> 4;                  // PAGED

  // ---- queries as the operand: channels 16 s + 8 h + (0 .. 7) of the lane's row
  V4i q[2 * NG];
  {
    const bool there = row < total_rows;
    const int query = rows.query_of(a, g, there ? row : first_row), in_token = (there ? row : first_row) - query * a.shared;
    const uint16_t* const src = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(first_token + query) * a.q_token + (int64_t)(head * a.shared + in_token) * a.q_head + h * 8;
#pragma unroll
    for (int s = 0; s < 2 * NG; ++s) {
      Packed8 raw = {0, 0, 0, 0};
      if (there) raw = *reinterpret_cast<const Packed8Any*>(src + s * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) q[s][i] = (int)((raw[i] ^ flip) & keep);
    }
  }

  // ---- a step's tokens on their way.  Packed: THREADS threads have a token, 16 bytes at a time.  PAGED: a wavefront has a block of 16 tokens, its keys and its
  // values (BOTH) or one of them.
  constexpr int THREADS = 64 * WAVES / STEP, PER = (CH + THREADS - 1) / THREADS;
  constexpr bool BOTH = WAVES * 16 == STEP;
  Packed8 key_part[PAGED ? 1 : PER], value_part[PAGED ? 1 : PER];
  uint32_t key_code[PAGED ? 2 * NG : 1], value_code[PAGED && BOTH ? 2 * NG : 1], key_scale = 0, value_scale = 0;
  int pages = 0;                                          // PAGED: a lane has the page of one block of the next steps
  int64_t key_block = 0;                                  // PAGED, BOTH: where the values of the keys before lie
  uint32_t largest = PAGED ? 1 : 0;                       // packed, HALF: magnitudes of values, two at a time; PAGED: a block's byte, 0 where all values are zero
  int first_byte = 0;                                     // PAGED: what values are held relative to
  bool wide = false;                                      // PAGED: a block's byte lies too far from that one
  const int own = BOTH ? wave : wave >> 1;
  int who = thread;                                       // worked out again for the careful steps: what follows from it would hold registers until then
  const bool brings_keys = BOTH || (wave & 1) == 0, brings_values = BOTH || (wave & 1) == 1;
  constexpr int kAhead = 64 / (STEP / 16);                // steps whose pages the lanes have
  auto look_up = [&](int at) {
    if constexpr (PAGED) {
      const int index = min((at >> 4) + (later(threadIdx.x) & 63), last_block) >> (a.pool.page_bits - kBlockBits);
      const int page = table[min(index, a.table_width - 1)];
      const bool fine = index < a.table_width && page >= 0 && page < a.pool.pages;
      bad = bad || __any(!fine);
      pages = fine ? page : 0;
    }
  };
  auto block_of = [&](int at, int slot) {
    const int bits = a.pool.page_bits - kBlockBits, block = min((at >> 4) + own, last_block);
    return (((int64_t)__builtin_amdgcn_readlane(pages, slot * (STEP / 16) + own) * a.pool.heads + head) << bits) + (block & ((1 << bits) - 1));
  };
  auto load_codes = [&](uint32_t* to, const uint8_t* from, uint32_t lane_at, uint32_t stride, uint32_t rest_at) {
#pragma unroll
    for (int i = 0; i < NG / 2; ++i) load_words<4>(to + 4 * i, from + lane_at + i * stride);
    if (NG % 2) load_words<2>(to + 2 * NG - 2, from + rest_at + (NG / 2) * stride);
  };
  auto load_keys = [&](int at, int slot) {
    if constexpr (PAGED) {
      if (!brings_keys) return;
      const int n = who & 15, j = who >> 4 & 3;
      key_block = block_of(at, slot);
      key_scale = args.scales[key_block * 2];
      load_codes(key_code, a.pool.data + key_block * (32 * D), n * D + j * 16, 64, n * D + j * 8);
    } else {
      // what lies behind the end is never seen
      const uint16_t* const k = args.k + (int64_t)min(at + who / THREADS, end - 1) * args.k_token + (int64_t)head * args.k_head + who % THREADS * 8;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (CH % THREADS == 0 || who % THREADS + i * THREADS < CH) key_part[i] = *reinterpret_cast<const Packed8Any*>(k + i * THREADS * 8);
    }
  };
  auto load_values = [&](int at, int64_t block) {
    if constexpr (PAGED) {
      if (!brings_values) return;
      const int n = who & 15, j = who >> 4 & 3;
      value_scale = args.scales[block * 2 + 1];
      load_codes(BOTH ? value_code : key_code, a.pool.data + block * (32 * D) + 16 * D, j * 4 * D + n * 16, 256, j * 4 * D + n * 8);
    } else {
      const uint16_t* const v = args.v + (int64_t)min(at + who / THREADS, end - 1) * args.v_token + (int64_t)head * args.v_head + who % THREADS * 8;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (CH % THREADS == 0 || who % THREADS + i * THREADS < CH) value_part[i] = *reinterpret_cast<const Packed8Any*>(v + i * THREADS * 8);
    }
  };
  auto finite = [](uint32_t bits) { return BF ? (bits & 0x7F80u) != 0x7F80u : (bits & 0x7C00u) != 0x7C00u; };
  auto store_keys = [&](int number) {
    const int buffer = number & 1;
    uint8_t* const keys = lds + buffer * kTile;
    if constexpr (PAGED) {
      if (!brings_keys) return;
      const float key_unit = power_of(key_scale);
      const int n = who & 15, j = who >> 4 & 3, token = own * 16 + n;
      if (!BF && (who & 63) == 0) lds_unit[(number & 3) * 4 + own] = fminf(key_unit * unit, 0x1.fffffep127f);
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        // words 2i and 2i + 1: channels 64 (i / 2) + 16 j + 8 (i % 2) on, or the last 32 channels' 8 j
        const int chunk = i < NG / 2 * 2 ? (i / 2) * 8 + 2 * j + i % 2 : (NG / 2) * 8 + j;
        *reinterpret_cast<V4i*>(keys + (token * CH + key_chunk<NG>(token, chunk)) * 16) = operand_of<BF>(key_code[2 * i], key_code[2 * i + 1], BF ? key_unit : 1.f);
      }
    } else {
      const int token = who / THREADS;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int chunk = who % THREADS + THREADS * i;
        if (CH % THREADS == 0 || chunk < CH) *reinterpret_cast<Packed8*>(keys + (token * CH + key_chunk<NG>(token, chunk)) * 16) = key_part[i];
      }
    }
  };
  // PAGED: the bytes of a word of values, 4 tokens of a channel, that some row sees.
  auto seen_bytes = [&](int at) {
    uint32_t mask = 0xFFFFFFFFu;
    if (at < low || at + STEP > end) {                    // what no row sees may be anything
      mask = 0;
      const int first = at + (own * 4 + (later(threadIdx.x) >> 4 & 3)) * 4;      // kept from one use to the next it would hold a register; so in look_up
#pragma unroll
      for (int i = 0; i < 4; ++i) mask |= first + i >= low && first + i < end ? 255u << 8 * i : 0u;
    }
    return mask;
  };
  // PAGED: powers of two above the first blocks' with which fp16 holds a block's values.
  auto fits = [](int above) { return above <= 6 && above >= -15; };
  // PAGED: whether the block has values other than zero, whose factor alone counts: that of zeros, 2^-126, is far from all others.
  auto holds = [&](uint32_t mask) {
    const uint32_t* const code = BOTH ? value_code : key_code;
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < 2 * NG; ++w) any |= code[w];
    return __any((any & mask & 0x7F7F7F7Fu) != 0) != 0;
  };
  // CAREFUL: without what is not finite, whose tokens are marked; values of fp16 as two bf16 parts, the second in the other buffer.
  auto store_values = [&](int at, int buffer, auto careful) {
    constexpr bool CAREFUL = decltype(careful)::value;
    uint8_t* const values = lds_values + buffer * kTile;
    if constexpr (PAGED) {
      if (!brings_values) return;
      const int above = (int)value_scale - first_byte;
      const float value_unit = CAREFUL ? power_of(value_scale) : power_of((uint32_t)min(max(127 + above, 1), 254));
      if (!CAREFUL) {
        wide = wide || !fits(above);
        largest = max(largest, value_scale);
      }
      const int n = who & 15, j = who >> 4 & 3, quad = own * 4 + j;
      const uint32_t mask = seen_bytes(at);
      const uint32_t* const code = BOTH ? value_code : key_code;
#pragma unroll
      for (int w = 0; w < 2 * NG; w += 2) {               // two channels: 4 tokens each, 16 bytes together
        const int channel = w < NG / 2 * 4 ? (w / 4) * 64 + n * 4 + w % 4 : (NG / 2) * 64 + n * 2 + (w - NG / 2 * 4);
        uint32_t x[2] = {code[w] & mask, code[w + 1] & mask};
        if (CAREFUL) {
          const uint32_t odd0 = not_numbers(x[0]), odd1 = not_numbers(x[1]);
          x[0] &= ~(odd0 * 255u), x[1] &= ~(odd1 * 255u);
#pragma unroll 1
          for (int i = 0; i < 4; ++i)
            if ((odd0 | odd1) >> 8 * i & 1) atomicOr(lds_odd + (quad >> 3), 1u << ((quad * 4 + i) & 31));
        }
        *reinterpret_cast<V4i*>(values + (quad * D + channel) * 8) = operand_of<CAREFUL>(x[0], x[1], value_unit);
      }
    } else {
      const int token = who / THREADS;
      if (at + STEP > end && at + token >= end) {
#pragma unroll
        for (int i = 0; i < PER; ++i) value_part[i] = Packed8{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int chunk = who % THREADS + THREADS * i, at_value = (token * CH + value_chunk<NG>(token, chunk)) * 16;
        if (CH % THREADS != 0 && chunk >= CH) continue;
        if constexpr (!CAREFUL) {
          *reinterpret_cast<Packed8*>(values + at_value) = value_part[i];
          if (HALF) {
            typedef uint16_t Us2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int w = 0; w < 4; ++w)
              largest = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Us2, largest), __builtin_bit_cast(Us2, value_part[i][w] & 0x7FFF7FFFu)));
          }
        } else {
          Packed8 hi = value_part[i], lo = {0, 0, 0, 0};
          bool odd = false;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            if (!finite(hi[w])) hi[w] &= 0xFFFF0000u, odd = true;
            if (!finite(hi[w] >> 16)) hi[w] &= 0xFFFFu, odd = true;
          }
          if (odd) atomicOr(lds_odd + (token >> 5), 1u << (token & 31));
          if (!BF) {
            float x[8], y[8];
            unpack8<false>(hi, x);
            hi = pack8<true>(x);
            unpack8<true>(hi, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] -= y[e];
            lo = pack8<true>(x);
            *reinterpret_cast<Packed8*>(values + kTile + at_value) = lo;
          }
          *reinterpret_cast<Packed8*>(values + at_value) = hi;
        }
      }
    }
  };

  // ---- operands from LDS
  constexpr int kKeys = NG % 4 == 0 ? 8 : NG % 2 == 0 ? 4 : 2, kValues = NG % 4 == 0 ? 4 : NG % 2 == 0 ? 2 : 1;
  uint32_t key_of[kKeys], value_of[kValues];              // by the part of a chunk's number that is swizzled; the rest are constants
  auto find_operands = [&](int thread) {                  // for the careful steps again, as `who`
    const int lane = thread & 63, col = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) key_of[i] = (col * CH + key_chunk<NG>(col, 2 * i + h)) * 16;
    if constexpr (PAGED) {
      value_of[0] = (h * D + col) * 8;
    } else {
      const int w = lane & 15, token = 4 * h + (w >> 2), inner = (lane >> 4 & 1) * 2 + ((w & 3) >> 1);
#pragma unroll
      for (int i = 0; i < kValues; ++i) value_of[i] = (token * CH + value_chunk<NG>(token, 4 * i + inner)) * 16 + (w & 1) * 8;
    }
  };
  find_operands(thread);
  auto key_operand = [&](int buffer, int part, int s) {       // tokens 32 part + col
    return *reinterpret_cast<const V4i*>(lds + buffer * kTile + key_of[s % kKeys] + (part * 32 * CH + s / kKeys * kKeys * 2) * 16);
  };
  auto value_operand = [&](int buffer, int c, int e) {        // channel 32 c + col, tokens 16 e + 4 h, + 8
    U2 lo, hi;
    if constexpr (PAGED) {
      const uint8_t* const from = lds_values + buffer * kTile + value_of[0] + (e * 4 * D + c * 32) * 8;
      lo = *reinterpret_cast<const U2*>(from), hi = *reinterpret_cast<const U2*>(from + 2 * D * 8);
    } else {
      const uint8_t* const from = lds_values + buffer * kTile + value_of[c % kValues] + c / kValues * kValues * 64 + e * 16 * CH * 16;
      lo = read_turned(from), hi = read_turned(from + 8 * CH * 16);
    }
    return V4i{(int)lo[0], (int)lo[1], (int)hi[0], (int)hi[1]};
  };

  // ---- the row's state
  float base = 0.f, limit = -INFINITY;                    // what scores are lifted by, and how large they may then be; nothing seen yet: 0 and -infinity
  float sum = 0.f, rest = 0.f;                            // of the weights as they are multiplied, and what its roundings left out
  float lost = 0.f;                                       // what the weights lost as they were rounded: little, so that a token far ahead takes nothing from the sum of all others
  V16f out[NG];
  const int want_sums_now = __builtin_amdgcn_readfirstlane(a.sums != nullptr);
  constexpr bool kSumsApart = !PAGED && NG <= 2;          // loops of their own for calls with sums: else the weights are made twice there, for want of registers
  auto begin_rows = [&] {
    base = 0.f, limit = -INFINITY, sum = rest = lost = 0.f;
#pragma unroll
    for (int c = 0; c < NG; ++c) out[c] = V16f{};
  };
  // what scores of tokens 16 e on are multiplied with
  auto unit_of = [&](int number, int e) { return PAGED && !BF ? lds_unit[(number & 3) * 4 + e] : unit; };
  auto hide = [&](V16f& x, int at) {
    // the lane's tokens are at + 4 h + (0 .. 3), + 8 and so on: it sees those from `from` to before `to`, a bit each
    const int behind = max(place + 1 - at - 4 * (later(threadIdx.x) >> 5 & 1), 0), from = min(max(behind - (int)reach, 0), 32), to = min(behind, 32);
    const uint32_t seen = (uint32_t)(((uint64_t{1} << to) - 1) & ~((uint64_t{1} << from) - 1));
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t keep = (uint32_t)((int32_t)(seen << (31 - ((i & 3) + 8 * (i >> 2)))) >> 31);
      const float score = x[i];                           // a cast of an element's bits takes the first one's
      x[i] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, score) & keep) | (0xFF800000u & ~keep));
    }
  };
  auto largest_of = [&](const V16f& x, int half) {
    float most = larger(x[8 * half], x[8 * half + 1]);
#pragma unroll
    for (int i = 2; i < 8; i += 2) most = larger(larger(most, x[8 * half + i]), x[8 * half + i + 1]);
    return most;
  };
  // `most`: the largest lifted score of the step
  auto lift = [&](float most, float kTop, float kMost) {
    const Halves both = halves_of(most);
    float by = fmaxf(both.low, both.high);
    if (limit > -INFINITY) by = fmaxf(by, kTop);
    if (!(by > -INFINITY)) return;
    const float to = base - (by - kTop);
    by = limit > -INFINITY ? __builtin_amdgcn_exp2f(to - base) : 1.f;
    base = to;
    limit = kMost;
    sum *= by, rest *= by, lost *= by;
#pragma unroll
    for (int c = 0; c < NG; ++c) out[c] *= by;
  };
  auto add_sum = [&](float more) {
    const float lacking = more + rest, now = sum + lacking;
    rest = lacking - (now - sum);
    sum = now;
  };

  // A step's products with the scores of the one behind it: while the matrix cores are at those, the vector units weigh this one's.
  auto step = [&](int at, int number, int buffer, V16f (&x)[PARTS], V16f (&next)[PARTS], float (&top)[2 * PARTS], auto want_sums, auto bring_values) {
    constexpr float kTop = HALF ? 10.f : 0.f, kMost = kTop + (HALF ? 5.f : kLift);
    if (at < all_lo || at + STEP > all_hi) {
      asm volatile("");                                   // a branch, not selections that every step would make
#pragma unroll
      for (int part = 0; part < PARTS; ++part) hide(x[part], at + part * 32);
#pragma unroll
      for (int e = 0; e < 2 * PARTS; ++e) top[e] = largest_of(x[e / 2], e & 1);
    }
    float units[2 * PARTS], most = -INFINITY;
#pragma unroll
    for (int e = 0; e < 2 * PARTS; ++e) {
      units[e] = unit_of(number, e);
      most = fmaxf(most, __builtin_fmaf(top[e], units[e], base));
    }
    if (__any(most > limit)) lift(most, kTop, kMost);
    if constexpr (!kSumsApart) {
      if (want_sums_now) {
        float more = 0.f, same = base;
        asm volatile("" : "+v"(same));                    // weights of their own: those below would be made here, not beside the products
#pragma unroll
        for (int i = 0; i < 16 * PARTS; ++i) more += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i / 16][i % 16], units[i / 8], same));
        lost += more;                                     // less what went in, below
      }
    }
    constexpr int kKeyFlight = PAGED ? 2 : 3;             // steps of keys' operands on their way; what the registers hold
    V4i p[2 * PARTS], key[kKeyFlight][PARTS];
    float more = 0.f, exact = 0.f;
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      next[part] = V16f{};
#pragma unroll
      for (int s = 0; s < kKeyFlight - 1; ++s) key[s][part] = key_operand(buffer ^ 1, part, s);
    }
#pragma unroll
    for (int s = 0; s < 2 * NG; ++s) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        if (s + kKeyFlight - 1 < 2 * NG) key[(s + kKeyFlight - 1) % kKeyFlight][part] = key_operand(buffer ^ 1, part, s + kKeyFlight - 1);
        next[part] = multiply32<!BF>(key[s % kKeyFlight][part], q[s], next[part]);
      }
#pragma unroll
      for (int pair = s * 8 * PARTS / (2 * NG); pair < (s + 1) * 8 * PARTS / (2 * NG); ++pair) {
        const int i = 2 * pair;
        const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i / 16][i % 16], units[i / 8], base));
        const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i / 16][i % 16 + 1], units[i / 8], base));
        int both = (int)pack2<!HALF>(w0, w1);
        asm volatile("" : "+v"(both));                    // here, not where it is used
        p[i / 8][i % 8 / 2] = both;
        more = add_pair<HALF>(both, more);
        if constexpr (decltype(want_sums)::value) exact += w0 + w1;
      }
    }
    if constexpr (decltype(want_sums)::value) lost += exact - more;
    else if (!kSumsApart && want_sums_now) lost -= more;
    bring_values();
    constexpr int kFlight = 4, kAll = NG * 2 * PARTS;     // values' operands on their way
    V4i value[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight - 1; ++k) value[k] = value_operand(buffer, k / (2 * PARTS), k % (2 * PARTS));
#pragma unroll
    for (int k = 0; k < kAll; ++k) {
      __builtin_amdgcn_sched_barrier(0);
      const int ahead = k + kFlight - 1;
      if (ahead < kAll) value[ahead % kFlight] = value_operand(buffer, ahead / (2 * PARTS), ahead % (2 * PARTS));
      out[k / (2 * PARTS)] = multiply32<HALF>(value[k % kFlight], p[k % (2 * PARTS)], out[k / (2 * PARTS)]);
#pragma unroll
      for (int pair = k * 8 * PARTS / kAll; pair < (k + 1) * 8 * PARTS / kAll; ++pair) {
        const int i = 2 * pair;
        const float x0 = next[i / 16][i % 16], x1 = next[i / 16][i % 16 + 1];
        top[i / 8] = i % 8 == 0 ? larger(x0, x1) : larger(larger(top[i / 8], x0), x1);
      }
    }
    add_sum(more);
  };

  // A step by itself, carefully: weights (and packed fp16 values) in two bf16 parts, values that are not finite row by row.
  auto careful_step = [&](int at) {
    const bool masked = at < all_lo || at + STEP > all_hi;
#pragma unroll 1
    for (int part = 0; part < PARTS; ++part) {
      const int from = at + part * 32;
      V16f x = {};
#pragma unroll
      for (int s = 0; s < 2 * NG; ++s) {
        if (s % 2 == 0) __builtin_amdgcn_sched_barrier(0);          // two operands on their way, or the registers do not hold them
        x = multiply32<!BF>(key_operand(0, part, s), q[s], x);
      }
      if (masked) hide(x, from);
      const float unit0 = unit_of(0, 2 * part), unit1 = unit_of(0, 2 * part + 1);
      const float most = fmaxf(__builtin_fmaf(largest_of(x, 0), unit0, base), __builtin_fmaf(largest_of(x, 1), unit1, base));
      if (__any(most > limit)) lift(most, 0.f, kLift);
      float weight[16], more = 0.f, together = 0.f;
      V4i hi[2], lo[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        weight[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], i < 8 ? unit0 : unit1, base));
        together += weight[i];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        parts_of<false>(weight + 8 * e, hi[e], lo[e]);
#pragma unroll
        for (int i = 0; i < 4; ++i) more = add_pair<false>(lo[e][i], add_pair<false>(hi[e][i], more));
      }
      lost += together - more;
      add_sum(more);
#pragma unroll
      for (int c = 0; c < NG; ++c) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const V4i v = value_operand(0, c, 2 * part + e);
          out[c] = multiply32<false>(v, lo[e], out[c]);
          if (!BF && !PAGED) out[c] = multiply32<false>(value_operand(1, c, 2 * part + e), hi[e], out[c]);
          out[c] = multiply32<false>(v, hi[e], out[c]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      uint32_t odd = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_odd[part]);
      while (odd) {
        const int t = __builtin_ctz(odd), token = from + t, index = (t & 3) + 4 * (t >> 3);
        odd &= odd - 1;
        if (token >= end) continue;
        const uint8_t* codes = nullptr;
        if constexpr (PAGED) {
          // the first pass has looked all of these entries up: where one names no page, nobody gets here
          const int block = token >> 4, bits = a.pool.page_bits - kBlockBits;
          codes = a.pool.data + ((((int64_t)table[block >> bits] * a.pool.heads + head) << bits) + (block & ((1 << bits) - 1))) * (32 * D) + 16 * D + (token >> 2 & 3) * 4 * D + (token & 3);
        }
        float w = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) w = i == index ? weight[i] : w;
        w = __shfl(w, col + 32 * (t >> 2 & 1));
        if ((uint32_t)(place - token) >= reach) continue;
#pragma unroll
        for (int c = 0; c < NG; ++c) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);      // a few values at a time, or the registers do not hold what is on its way
            const int channel = c * 32 + (i & 3) + 8 * (i >> 2) + 4 * h;
            if constexpr (PAGED) {
              if ((codes[channel * 4] & 0x7F) == 0x7F) out[c][i] = NAN;
            } else {
              const uint32_t bits = args.v[(int64_t)token * args.v_token + (int64_t)head * args.v_head + channel];
              if (!finite(bits)) out[c][i] += w * to_float<BF>(bits);
            }
          }
        }
      }
    }
  };

  begin_rows();
  if (begin < end) {
    if (thread == 0) lds_odd[0] = 0;                      // a block of rows that is gone through again sets it
    typedef std::integral_constant<bool, true> Yes;
    typedef std::integral_constant<bool, false> No;
    look_up(begin);
    load_keys(begin, 0);
    load_values(begin, BOTH ? key_block : brings_values ? block_of(begin, 0) : 0);
    if constexpr (PAGED) {
      // the largest byte of the first step that has values other than zero
      int from = begin;
      for (int s = 0;;) {
        if (brings_values) {
          const bool held = holds(seen_bytes(from));
          if (lane == 0) lds_word[own] = held ? max(value_scale, 1u) : 0u;
        }
        __syncthreads();
        uint32_t byte = 0;
#pragma unroll
        for (int i = 0; i < STEP / 16; ++i) byte = max(byte, lds_word[i]);
        first_byte = __builtin_amdgcn_readfirstlane((int)byte);
        from += STEP;
        if (first_byte > 0 || from >= end) break;
        __syncthreads();                                  // all have read the words
        if (++s == kAhead) {
          look_up(from);
          s = 0;
        }
        load_values(from, brings_values ? block_of(from, s) : 0);
      }
      if (first_byte == 0) first_byte = 127;              // zeros alone
      if (from > begin + STEP) {
        look_up(begin);
        load_values(begin, brings_values ? block_of(begin, 0) : 0);
      }
    }
    int slot = 1;                                         // of the next keys' pages
    int64_t value_block = 0;
    store_keys(0);
    store_values(begin, 0, No{});
    if (begin + STEP < end) {
      load_keys(begin + STEP, slot);
      value_block = key_block;
      store_keys(1);
    }
    __syncthreads();
    V16f scores[2][PARTS];
    float top[2 * PARTS];                                 // the largest of 16 tokens' scores that the lane has
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      scores[0][part] = V16f{};
#pragma unroll
      for (int s = 0; s < 2 * NG; ++s) scores[0][part] = multiply32<!BF>(key_operand(0, part, s), q[s], scores[0][part]);
      top[2 * part] = largest_of(scores[0][part], 0), top[2 * part + 1] = largest_of(scores[0][part], 1);
    }
    __syncthreads();
    int number = 0;
    auto turn = [&](int at, int buffer, V16f (&x)[PARTS], V16f (&next)[PARTS], auto want_sums) {
      // keys of the step behind the next; what is looked up for them serves the values a step later
      const int64_t block = !BOTH && PAGED && brings_values && at + STEP < end ? block_of(at + STEP, slot) : value_block;
      ++slot;
      if (at + 2 * STEP < end) {
        if (slot == kAhead) {
          look_up(at + 2 * STEP);
          slot = 0;
        }
        load_keys(at + 2 * STEP, slot);
        value_block = key_block;
      }
      step(at, number, buffer, x, next, top, want_sums, [&] {
        if (at + STEP < end) load_values(at + STEP, block);
      });
      if (at + 2 * STEP < end) store_keys(number + 2);
      if (at + STEP < end) store_values(at + STEP, buffer ^ 1, No{});
      ++number;
      __syncthreads();
    };
    auto go = [&](auto want_sums) {
      for (int at = begin; at < end; at += 2 * STEP) {
        turn(at, 0, scores[0], scores[1], want_sums);
        if (at + STEP >= end) break;
        turn(at + STEP, 1, scores[1], scores[0], want_sums);
      }
    };
    if (kSumsApart && a.sums) go(std::integral_constant<bool, kSumsApart>{});
    else go(No{});
    if constexpr (PAGED) {
      // Bytes far from the others may be those of zeros: each wavefront goes through its blocks again (looking at the values in every step took 1 to 5 % of all calls).
      if (wide) {
        wide = false;
        largest = 0;
        who = later(threadIdx.x);
        for (int at = begin, s = 0; at < end && !wide; at += STEP, s = s + 1 == kAhead ? 0 : s + 1) {
          if (s == 0) look_up(at);
          load_values(at, block_of(at, s));
          if (!holds(seen_bytes(at))) continue;
          wide = !fits((int)value_scale - first_byte);
          largest = max(largest, max(value_scale, 1u));
        }
      }
    }
    float all = 0.f;
#pragma unroll
    for (int c = 0; c < NG; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) all += out[c][i];
    bool again = all != all || wide;
    if (HALF) {
      // A weight below fp16's normal numbers is off by 2^-25 at most, in units of which the row's largest is 2^10 at least.
      uint32_t most = largest;
      if (!PAGED) {
        most = max(most >> 16, most & 0xFFFFu);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, m));
      }
      if (lane == 0 && (!PAGED || brings_values)) lds_word[PAGED ? own : wave] = most;
      __syncthreads();
      most = 0;
#pragma unroll
      for (int i = 0; i < (PAGED ? STEP / 16 : WAVES); ++i) most = max(most, lds_word[i]);
      float far = PAGED && most == 0 ? 0.f : PAGED ? kMostCode * power_of((uint32_t)min(max(127 + (int)most - first_byte, 1), 254)) : most >= 0x7C00u ? INFINITY : to_float<false>(most);
      far *= (float)(end - begin) * (BF ? 0x1p-25f * 0x1p9f : 0x1p-25f * 0x1p12f);
      float large = 0.f;
#pragma unroll
      for (int c = 0; c < NG; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) large = fmaxf(large, fabsf(out[c][i]));
      const Halves both = halves_of(large);
      large = fmaxf(both.low, both.high);
      again = again || (limit > -INFINITY && large < far);
    }
    // With a page missing nobody goes again: the rows are NaN as it is.  All wavefronts have looked up the same entries, so that all stay.
    if (!bad && __any(again) && (later(threadIdx.x) & 63) == 0) atomicOr(lds_odd, 1u);
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane((int)lds_odd[0])) {
      __syncthreads();
      begin_rows();
      first_byte = 127;
      who = later(threadIdx.x);
      find_operands(who);
      for (int at = begin, s = 0; at < end; at += STEP, s = s + 1 == kAhead ? 0 : s + 1) {
        if (s == 0) look_up(at);
        load_keys(at, s);
        load_values(at, BOTH ? key_block : PAGED && brings_values ? block_of(at, s) : 0);
        const int clears = later(threadIdx.x);
        if (clears < 2) lds_odd[clears] = 0;
        __syncthreads();
        store_keys(0);
        store_values(at, 0, Yes{});
        __syncthreads();
        careful_step(at);
        __syncthreads();
      }
    }
  }

  const Halves sums = halves_of(sum + rest), losses = halves_of(lost);
  float total = sums.low + sums.high, whole = total + (losses.low + losses.high);      // of the weights before they are rounded
  const int thread_of = later(threadIdx.x), row_of = first_row + (thread_of >> 6) * 32 + (thread_of & 31), half = thread_of >> 5 & 1;
  if (PAGED ? row_of >= total_rows : reach == 0) return;
  if (bad) total = whole = NAN;
  const int query = rows.query_of(a, g, row_of), head_of = head * a.shared + row_of - query * a.shared;
  const int64_t token = first_token + query;
  const float most = limit > -INFINITY ? -base : -INFINITY;
  const int64_t part = (token * a.heads + head_of) * g.splits + split;
  const bool parted = PAGED && span.used > 1;
  // A part whose sum is asked for has that of the weights before they are rounded, and results to match: joined, each part counts by that sum, and rounding cancels out
  // within the part.
  const bool whole_part = parted && a.sums && total != 0.f;
  // the power of two by itself: with 1 / total it may be less than 32 bits hold, where results are not
  const float one = PAGED && begin < end ? power_of((uint32_t)first_byte) : 1.f, r = whole_part ? whole / total : parted ? 1.f : total == 0.f ? 0.f : 1.f / total;
  uint16_t* const dst = reinterpret_cast<uint16_t*>(a.out) + token * a.out_token + head_of * a.out_head + half * 4;
#pragma unroll
  for (int c = 0; c < NG; ++c) {
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      V4f o = {out[c][i] * r, out[c][i + 1] * r, out[c][i + 2] * r, out[c][i + 3] * r};
      if (PAGED) o *= one;
      const int channel = c * 32 + 2 * i;
      if (parted) {
        *reinterpret_cast<V4f*>(g.parts + part * D + half * 4 + channel) = o;
      } else {
        typedef uint32_t Pair __attribute__((ext_vector_type(2), aligned(2)));
        *reinterpret_cast<Pair*>(dst + channel) = Pair{pack2<BF>(o[0], o[1]), pack2<BF>(o[2], o[3])};
      }
    }
  }
  if (half > 0) return;
  if (parted) {
    float* const ms = g.parts + a.tokens * a.heads * g.splits * D + part * 2;
    ms[0] = most;
    ms[1] = whole_part ? whole : total;
    if (split == 0) used_splits(a, g)[token * a.heads + head_of] = span.used;
    return;
  }
  if (PAGED && g.splits > 1) used_splits(a, g)[token * a.heads + head_of] = 1;
  if (a.sums) a.sums[token * a.heads + head_of] = (most + __builtin_amdgcn_logf(whole)) * 0.6931471805599453f;
}

template <int NG, bool BF, bool PAGED, int WAVES>
__global__ __launch_bounds__(64 * WAVES, NG > 6 ? 1 : 2) void rows_kernel(const LaunchRows args) {
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int kRows = 32 * WAVES;
  const KvAttention& a = args.a;
  const Grid& g = args.g;
  if constexpr (PAGED) {
    const int split = g.splits == 1 ? 0 : g.row_blocks == 1 ? (int)blockIdx.z : (int)blockIdx.z / g.row_blocks, block = (int)blockIdx.z - split * g.row_blocks;
    int b = blockIdx.y;
    if (g.ordered) b = nth_longest(a, b, threadIdx.x & 63);
    const Sequence seq = sequence_of(a, b);
    // the last rows see most and start first
    for (int first_row = (g.row_blocks - 1 - block) * kRows; first_row < seq.rows; first_row += g.row_blocks * kRows) {
      rows_block<NG, BF, PAGED, WAVES>(args, lds, seq, b, blockIdx.x, split, first_row);
      __syncthreads();
    }
  } else {
    const int block = (int)(blockIdx.x / (uint32_t)a.pool.heads), head = (int)blockIdx.x - block * a.pool.heads;
    rows_block<NG, BF, PAGED, WAVES>(args, lds, Sequence{}, 0, head, 0, (g.row_blocks - 1 - block) * kRows);
  }
}

template <int NG, bool BF, bool PAGED, int WAVES>
int launch_rows(const LaunchRows& l, dim3 grid, hipStream_t stream) {
  constexpr int lds = 4 * row_step(NG, PAGED, WAVES) * 32 * NG * 2 + 4 * (16 + 2 + WAVES);
  if (lds > 64 * 1024) MACKO_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&rows_kernel<NG, BF, PAGED, WAVES>), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  hipLaunchKernelGGL((rows_kernel<NG, BF, PAGED, WAVES>), grid, dim3(64 * WAVES), lds, stream, l);
  MACKO_HIP_TRY(hipGetLastError());
  return MACKO_OK;
}

}  // namespace macko
