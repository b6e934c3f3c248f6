// The 8-bit key/value cache: new tokens into it (macko_kv8_append) and its values back (macko_kv8_read); the C entry points of these and of the attention
// over the cache.
//
// A block of 16 tokens of a head has m = its largest finite magnitude, the least byte b with m <= 448 * 2^(b-127), and codes round(x * 2^(127-b)).  A value takes 2 bytes in and 1
// out, or the other way round, and some ten operations: memory bounds reads (65536 tokens of 8 heads of 128 channels 74 us, 5.4 TB/s; 16384 18 us, 5.5) and queries, loads that wait
// for each other keys and values (16384 tokens 31 us, 3.2 TB/s; with 32 heads of queries 79 us, 4.7), a launch short calls (one token 5.9 us, 64 tokens of as many sequences 6.9).
#include <cmath>

#include "macko_kv8.h"
#include "macko_kv8_attention.h"

namespace macko {
namespace {

constexpr int kBlock = 256, kWave = 64;
constexpr int64_t kMostBlocks = (int64_t{1} << 24) - 1;  // a launch has fewer than 2^32 threads
typedef float V4 __attribute__((ext_vector_type(4)));
typedef uint32_t W2 __attribute__((ext_vector_type(2)));
typedef uint32_t W4 __attribute__((ext_vector_type(4)));

struct AppendArgs {
  const uint16_t *q, *k, *v;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head;
  uint16_t* out;
  int64_t out_token, out_head;
  const uint16_t *q_weight, *k_weight;
  const int32_t* positions;
  const float* table;
  int64_t table_rows;
  const int32_t *tables, *lengths, *start;
  int64_t table_stride;
  Kv8Pool pool;
  int64_t tokens;
  int32_t q_groups;          // append_kernel: workgroups that share a token's queries out
  int32_t table_width, batch, heads, dim, rot, interleaved;
  int32_t rows;              // that are looked for blocks together
  int32_t groups;            // wavefronts (append_kernel) or workgroups (blocks_kernel) that share the heads' keys out, and as many their values
  float eps;
};

// The sum, and the largest of whole numbers, over neighbouring lanes, in all of them.
template <int LANES>
__device__ inline float sum_over(float x) {
#pragma unroll
  for (int m = 1; m < LANES; m <<= 1) x += __shfl_xor(x, m);
  return x;
}
template <int LANES>
__device__ inline uint32_t most_over(uint32_t x) {
#pragma unroll
  for (int m = 1; m < LANES; m <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, m));
  return x;
}

// What turns the head of one token: a lane's cosines and sines (the sine's sign is that of the lane's half).
struct Turn {
  float c[8], s[8];
  int other;                 // the lane that holds the other channels of this one's pairs
  bool turned, placed;
};
// `row`: the cosines, then the sines, of the token's position.
__device__ inline Turn turn_by(const AppendArgs& a, const float* row, bool placed, int lane) {
  Turn t;
  const int half = a.rot >> 4;                            // lanes of half a turned part
  t.other = lane >= 2 * half ? lane : lane < half ? lane + half : lane - half;
  t.placed = placed;
  t.turned = placed && lane < 2 * half;
  if (t.turned) {
    row += a.interleaved ? lane * 4 : (lane < half ? lane : t.other) * 8;
    *reinterpret_cast<V4*>(t.c) = *reinterpret_cast<const V4*>(row);
    *reinterpret_cast<V4*>(t.s) = *reinterpret_cast<const V4*>(row + a.rot / 2);
    if (!a.interleaved) {
      *reinterpret_cast<V4*>(t.c + 4) = *reinterpret_cast<const V4*>(row + 4);
      *reinterpret_cast<V4*>(t.s + 4) = *reinterpret_cast<const V4*>(row + a.rot / 2 + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) t.s[i] = lane < half ? -t.s[i] : t.s[i];
    }
  }
  return t;
}
__device__ inline Turn turn_of(const AppendArgs& a, int64_t token, int lane) {
  const int64_t at = a.rot > 0 ? a.positions[token] : 0;
  return turn_by(a, a.table + at * a.rot, a.rot == 0 || (at >= 0 && at < a.table_rows), lane);
}

// 8 channels of a head, normalised and turned; NaN where the token's position lies outside the table.
template <bool BF, int LT>
__device__ inline void finish(const AppendArgs& a, Packed8 raw, const uint16_t* weight, const Turn& t, int lane, float* y) {
#pragma clang fp contract(off)     // products are rounded before they are added: keys near the edge of two codes take the same one everywhere
  unpack8<BF>(raw, y);
  if (weight) {
    float sum = 0.f, w[8] = {};
    if (lane * 8 < a.dim) unpack8<BF>(*reinterpret_cast<const Packed8Any*>(weight + lane * 8), w);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(y[e], y[e], sum);
    const float r = 1.f / sqrtf(sum_over<LT>(sum) / (float)a.dim + a.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = y[e] * r * w[e];
  }
  if (a.rot == 0) return;
  if (a.interleaved) {
    if (t.turned) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = y[2 * e], v = y[2 * e + 1];
        y[2 * e] = u * t.c[e] - v * t.s[e];
        y[2 * e + 1] = u * t.s[e] + v * t.c[e];
      }
    }
  } else {
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], t.other, LT);
    if (t.turned) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] * t.c[e] + z[e] * t.s[e];
    }
  }
  if (!t.placed) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = NAN;
  }
}

// The next block of 16 places of a sequence that a call's rows from w.row on begin: its new tokens are the places [first, last), the rows row0 + place.
struct Walk {
  int row, end, b;
};
struct NewTokens {
  int row0, first, last;
  int b, place;              // the sequence, the block's first token in it
};
// The page that a block lies in; < 0: none.
__device__ inline int page_of(const AppendArgs& a, const NewTokens& n) {
  const int index = n.place >> a.pool.page_bits, page = index < a.table_width ? constant(a.tables + n.b * a.table_stride + index) : -1;
  return page >= 0 && page < a.pool.pages ? page : -1;
}
__device__ inline Walk walk_of(const AppendArgs& a, int chunk, int lane64) {
  Walk w{chunk * a.rows, min((chunk + 1) * a.rows, (int)a.tokens), 0};
  w.b = a.start ? sequence_at(a.start, a.batch, w.row, lane64) : w.row;
  if (w.b < 0) w.b = 0, w.row = min(max(a.start[0], 0), w.end);
  return w;
}
__device__ inline bool next_block(const AppendArgs& a, Walk& w, NewTokens& n) {
  while (w.row < w.end && w.b < a.batch) {
    const int from = a.start ? min(max(constant(a.start + w.b), 0), (int)a.tokens) : w.row, to = a.start ? min(max(constant(a.start + w.b + 1), 0), (int)a.tokens) : w.row + 1;
    if (w.row >= to) {                                    // the sequence's rows are over, or it has none
      ++w.b;
      continue;
    }
    const int place = min(max(constant(a.lengths + w.b), 0), kMostTokens) - (to - w.row);
    if (place < 0) {                                      // more rows than tokens: these have no place
      w.row = min(to, w.row - place);
      continue;
    }
    n.first = place & 15, n.last = min(16, n.first + (to - w.row));
    n.row0 = w.row - n.first;
    const bool begins = n.first == 0 || w.row == from;
    const int b = w.b;
    w.row = n.row0 + n.last;
    if (!begins) continue;                                // the block begins in rows before these
    n.b = b, n.place = place & ~15;
    return true;
  }
  return false;
}

// Keys or values (VALUE) of one head for one block, by LT * TG lanes: lane (t, l) has 8 channels of TPL places, so that the values' words, 4 places of a channel, are made
// without another lane; all of a block's new tokens are there at once, and the largest magnitude takes one round of exchanges.  Only where the byte of scale
// grows are the block's earlier tokens read at all.
template <int LB>
struct Unit {
  static constexpr int LT = 1 << LB, TG = LT <= 16 ? 4 : 2, GROUP = LT * TG, TPL = 16 / TG, PAIRS = kWave / GROUP;
  Packed8 raw[TPL];
  int head;
  bool there;
};
template <int LB, bool VALUE>
__device__ inline void load_unit(const AppendArgs& a, Unit<LB>& u, const NewTokens& n, int lane64) {
  const int lane = lane64 & (Unit<LB>::LT - 1), first_place = (lane64 >> LB) % Unit<LB>::TG * Unit<LB>::TPL;
  const uint16_t* const src = VALUE ? a.v + u.head * a.v_head + lane * 8 : a.k + u.head * a.k_head + lane * 8;
  const int64_t stride = VALUE ? a.v_token : a.k_token;
#pragma unroll
  for (int r = 0; r < Unit<LB>::TPL; ++r) {
    const int p = first_place + r;
    u.raw[r] = Packed8{0, 0, 0, 0};
    if (u.there && lane * 8 < a.dim && p >= n.first && p < n.last) u.raw[r] = *reinterpret_cast<const Packed8Any*>(src + (int64_t)(n.row0 + p) * stride);
  }
}
__device__ inline bool is_finite(float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu) < 0x7F800000u; }
// turn_at(place): what turns the keys of that token.
template <bool BF, int LB, bool VALUE, class TurnAt>
__device__ inline void store_unit(const AppendArgs& a, const Unit<LB>& u, const NewTokens& n, int page, int lane64, TurnAt turn_at) {
  constexpr int LT = Unit<LB>::LT, TPL = Unit<LB>::TPL, GROUP = Unit<LB>::GROUP;
  const int lane = lane64 & (LT - 1), first_place = (lane64 >> LB) % Unit<LB>::TG * TPL;
  const bool mine = lane * 8 < a.dim;
  const int64_t block = kv8_block(a.pool, page, u.head, n.place & ((1 << a.pool.page_bits) - 1));
  uint8_t* const scale = a.pool.scales + block * 2 + VALUE;
  uint8_t* const codes = a.pool.codes + (block * 2 + VALUE) * (int64_t)(kBlockTokens * a.dim);
  const uint32_t had = n.first > 0 ? *scale : 0u;
  float y[TPL][8];
#pragma unroll
  for (int r = 0; r < TPL; ++r) {
    __builtin_amdgcn_sched_barrier(0);                    // one place's cosines and sines at a time, and so below: what more hold of registers costs wavefronts
    if constexpr (VALUE) unpack8<BF>(u.raw[r], y[r]);
    else finish<BF, LT>(a, u.raw[r], a.k_weight, turn_at(min(max(first_place + r, n.first), n.last - 1)), lane, y[r]);
  }
  if (n.first > 0 || n.last < 16) {
#pragma unroll
    for (int r = 0; r < TPL; ++r) {
      const bool fresh = first_place + r >= n.first && first_place + r < n.last;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[r][e] = fresh ? y[r][e] : 0.f;
    }
  }
  float most = 0.f;                                       // NaN where something is
#pragma unroll
  for (int r = 0; r < TPL; ++r)
#pragma unroll
    for (int e = 0; e < 8; ++e) most = __builtin_elementwise_maximum(most, fabsf(y[r][e]));
  const bool any_odd = __any(!(most < INFINITY));
  if (any_odd) {
    asm volatile("");                                     // a branch, not selections that every block would make; so below
    most = 0.f;
#pragma unroll
    for (int r = 0; r < TPL; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, is_finite(y[r][e]) ? fabsf(y[r][e]) : 0.f);
  }
  const uint32_t byte = max(scale_byte(most_over<GROUP>(__builtin_bit_cast(uint32_t, most))), had);
  const bool grown = n.first > 0 && byte > had;
  const float down = power_of(254u - min(byte, 254u));
  if (u.there && (lane64 & (GROUP - 1)) == 0 && (n.first == 0 || grown)) *scale = (uint8_t)byte;
  const int begin = grown ? 0 : n.first;                  // places that are written
  if (!u.there || !mine) return;
  uint32_t word[TPL][2];                                  // 8 codes of a place
#pragma unroll
  for (int r = 0; r < TPL; ++r) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float* const x = y[r] + 4 * h;
      int both = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * down, x[1] * down, 0, false);
      word[r][h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * down, x[3] * down, both, true);
    }
  }
  if (any_odd || __any(byte >= kMostScale)) {             // what is not finite, and what 448 does not reach
    asm volatile("");
#pragma unroll
    for (int r = 0; r < TPL; ++r) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[4];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = is_finite(y[r][4 * h + e]) ? y[r][4 * h + e] * down : 0.f;
        word[r][h] = codes_of(x);
#pragma unroll
        for (int e = 0; e < 4; ++e) word[r][h] |= is_finite(y[r][4 * h + e]) ? 0u : 0x7Fu << 8 * e;
      }
    }
  }
  if (grown) {                                            // the tokens in front again
    const float again = power_of(127u - min(byte - had, 127u));
#pragma unroll
    for (int r = 0; r < TPL; ++r) {
      const int p = first_place + r;
      __builtin_amdgcn_sched_barrier(0);
      if (p >= n.first) continue;
      uint32_t old[2] = {0, 0};
      if (VALUE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) old[e >> 2] |= (uint32_t)codes[((p >> 2) * a.dim + lane * 8 + e) * 4 + (p & 3)] << 8 * (e & 3);
      } else {
        const W2 w = *reinterpret_cast<const W2*>(codes + p * a.dim + lane * 8);
        old[0] = w[0], old[1] = w[1];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float z[4];
        numbers_of(old[h], z);
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = (old[h] >> 8 * e & 0x7Fu) == 0x7Fu ? 0.f : z[e] * again;
        uint32_t w = codes_of(z);
#pragma unroll
        for (int e = 0; e < 4; ++e) w |= (old[h] >> 8 * e & 0x7Fu) == 0x7Fu ? 0x7Fu << 8 * e : 0u;
        word[r][h] = w;
      }
    }
  }
  if constexpr (!VALUE) {
#pragma unroll
    for (int r = 0; r < TPL; ++r) {
      const int p = first_place + r;
      if (p >= begin && p < n.last) *reinterpret_cast<W2*>(codes + p * a.dim + lane * 8) = W2{word[r][0], word[r][1]};
    }
  } else {
#pragma unroll
    for (int q = 0; q < TPL / 4; ++q) {
      const int p = first_place + 4 * q;
      uint8_t* const quad = codes + ((p >> 2) * a.dim + lane * 8) * 4;
      uint32_t out[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t rows4[4] = {word[4 * q][h], word[4 * q + 1][h], word[4 * q + 2][h], word[4 * q + 3][h]};
        uint32_t cols[4];
        turn_words(rows4, cols);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[4 * h + e] = cols[e];
      }
      if (p >= begin && p + 4 <= n.last) {
        *reinterpret_cast<W4*>(quad) = W4{out[0], out[1], out[2], out[3]};
        *reinterpret_cast<W4*>(quad + 16) = W4{out[4], out[5], out[6], out[7]};
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (p + i < begin || p + i >= n.last) continue;
#pragma unroll
          for (int e = 0; e < 8; ++e) quad[e * 4 + i] = (uint8_t)(out[e] >> 8 * i);
        }
      }
    }
  }
}

// Few tokens: a workgroup either turns queries of a token (groups of LT lanes take a head) or stores the block that begins in a row: each wavefront the keys or
// the values of one head or, where a block takes fewer lanes, of several.  One launch; its time is a launch's and four loads' that wait for each other (lengths, table, rows, byte).
template <bool BF, int LB>
__global__ __launch_bounds__(kBlock) void append_kernel(const AppendArgs a) {
  constexpr int LT = 1 << LB, GROUP = Unit<LB>::GROUP, PAIRS = Unit<LB>::PAIRS;
  const int lane64 = threadIdx.x & 63, lane = lane64 & (LT - 1);
  if ((int)blockIdx.x < a.q_groups) {
    const int head = (int)blockIdx.x * (kBlock / LT) + (threadIdx.x >> LB);
    const bool there = head < a.heads && lane * 8 < a.dim;
    for (int64_t token = blockIdx.y; token < a.tokens; token += gridDim.y) {
      Packed8 raw = {0, 0, 0, 0};
      if (there) raw = *reinterpret_cast<const Packed8Any*>(a.q + token * a.q_token + head * a.q_head + lane * 8);
      float y[8];
      finish<BF, LT>(a, raw, a.q_weight, turn_of(a, token, lane), lane, y);
      if (there) *reinterpret_cast<Packed8Any*>(a.out + token * a.out_token + head * a.out_head + lane * 8) = pack8<BF>(y);
    }
    return;
  }
  const int rest = ((int)blockIdx.x - a.q_groups) * (kBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // keys' heads, then values'
  if (rest >= 2 * a.groups) return;
  const int head = (rest >= a.groups ? rest - a.groups : rest) * PAIRS + lane64 / GROUP;
  Unit<LB> u;
  u.there = head < a.pool.heads;
  u.head = u.there ? head : 0;
  auto store = [&](auto value) {
    constexpr bool VALUE = decltype(value)::value;
    for (int chunk = blockIdx.y; chunk < (int)a.tokens; chunk += gridDim.y) {
      Walk w = walk_of(a, chunk, lane64);
      NewTokens n;
      while (next_block(a, w, n)) {
        load_unit<LB, VALUE>(a, u, n, lane64);            // under way before the page is known
        const int page = page_of(a, n);
        if (page >= 0) store_unit<BF, LB, VALUE>(a, u, n, page, lane64, [&](int place) { return turn_of(a, n.row0 + place, lane); });
      }
    }
  };
  if (rest >= a.groups) store(std::integral_constant<bool, true>{});
  else store(std::integral_constant<bool, false>{});
}

// Many tokens, keys and values alone: a workgroup takes the blocks that begin in 16 rows, for the keys or the values of 4 times as many heads as a wavefront has
// at once.  What turns the keys is brought into LDS once for all of them.  Its loads wait for each other, so that wavefronts count: with three workgroups to a compute unit
// 37 us for 16384 tokens of 8 heads of 128 channels, with four, for which no more than 128 registers are there, 31.  More heads to a workgroup, the next ones' rows on their way, gave
// nothing; queries in the same launch made 83 us 108.
template <bool BF, int LB>
__global__ __launch_bounds__(kBlock, LB <= 4 ? 4 : 2) void blocks_kernel(const AppendArgs a) {
  constexpr int LT = 1 << LB, GROUP = Unit<LB>::GROUP, PAIRS = Unit<LB>::PAIRS;
  __shared__ __align__(16) float table[16 * 256];         // [place][cosines, sines]
  __shared__ int placed[16];
  const int lane64 = threadIdx.x & 63, lane = lane64 & (LT - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rest = blockIdx.x, head = ((rest >= a.groups ? rest - a.groups : rest) * 4 + wave) * PAIRS + lane64 / GROUP;
  const int chunks = (int)((a.tokens + 15) >> 4);
  Unit<LB> u;
  u.there = head < a.pool.heads;
  u.head = u.there ? head : 0;
  NewTokens n;
  if (rest >= a.groups) {
    for (int chunk = blockIdx.y; chunk < chunks; chunk += gridDim.y) {
      Walk w = walk_of(a, chunk, lane64);
      while (next_block(a, w, n)) {
        load_unit<LB, true>(a, u, n, lane64);
        const int page = page_of(a, n);
        if (page >= 0) store_unit<BF, LB, true>(a, u, n, page, lane64, [&](int) { return Turn{}; });
      }
    }
    return;
  }
  const int quads = a.rot / 4;
  for (int chunk = blockIdx.y; chunk < chunks; chunk += gridDim.y) {
    Walk w = walk_of(a, chunk, lane64);
    while (next_block(a, w, n)) {
      load_unit<LB, false>(a, u, n, lane64);
      const int page = page_of(a, n);
      if (a.rot > 0) {
        __syncthreads();                                  // the block before has been turned
        // 16 threads bring a token's row
        const int place = threadIdx.x >> 4;
        if (place >= n.first && place < n.last) {
          const int64_t at = a.positions[n.row0 + place];
          const bool fine = at >= 0 && at < a.table_rows;
          if (fine)
            for (int i = threadIdx.x & 15; i < quads; i += 16) reinterpret_cast<V4*>(table)[place * quads + i] = *reinterpret_cast<const V4*>(a.table + at * a.rot + i * 4);
          if ((threadIdx.x & 15) == 0) placed[place] = fine;
        }
        __syncthreads();
      }
      if (page >= 0)
        store_unit<BF, LB, false>(a, u, n, page, lane64, [&](int place) { return turn_by(a, table + place * a.rot, a.rot == 0 || placed[place], lane); });
    }
  }
}

struct ReadArgs {
  Kv8Pool pool;
  const int32_t* slots;
  int64_t tokens, slots_held, items;
  uint16_t* k;
  int64_t k_token, k_head;
  uint16_t* v;
  int64_t v_token, v_head;
};

template <bool BF>
__device__ inline Packed8 read8(uint32_t lo, uint32_t hi, float unit) {
  float x[8];
  numbers_of(lo, x);
  numbers_of(hi, x + 4);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= unit;
  return pack8<BF>(x);
}

// A group of LT lanes takes E entries of the list for one head.  Where there are 4 and they are 4 tokens in the order in which values lie together, the values come as whole
// words; else byte by byte.  Every result is exact in 32 bits and rounded once.
template <bool BF, int LB, int E>
__global__ __launch_bounds__(kBlock) void read_kernel(const ReadArgs a) {
  constexpr int LT = 1 << LB;
  const int lane = threadIdx.x & (LT - 1), dim = a.pool.dim;
  const bool mine = lane * 8 < dim;
  for (int64_t item = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> LB; item < a.items; item += (int64_t)gridDim.x * (kBlock >> LB)) {
    const int64_t quad = item / a.pool.heads;
    const int head = (int)(item - quad * a.pool.heads);
    if (!mine) continue;
    int64_t block[E];
    int at[E];
    bool there[E], wide = E == 4;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int64_t slot = quad * E + i < a.tokens ? a.slots[quad * E + i] : -1;
      there[i] = slot >= 0 && slot < a.slots_held;
      block[i] = there[i] ? kv8_block(a.pool, slot >> a.pool.page_bits, head, (int)(slot & ((1 << a.pool.page_bits) - 1))) : 0;
      at[i] = (int)(slot & 15);
      wide = wide && there[i] && block[i] == block[0] && at[i] == (at[0] & ~3) + i;
    }
    const int64_t bytes = kBlockTokens * dim;
    if (a.k) {
      W2 word[E];
      uint32_t byte[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        word[i] = W2{0, 0};
        byte[i] = 127;
        if (there[i]) {
          word[i] = *reinterpret_cast<const W2*>(a.pool.codes + block[i] * 2 * bytes + at[i] * dim + lane * 8);
          byte[i] = a.pool.scales[block[i] * 2];
        }
      }
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (quad * E + i < a.tokens) *reinterpret_cast<Packed8Any*>(a.k + (quad * E + i) * a.k_token + head * a.k_head + lane * 8) = read8<BF>(word[i][0], word[i][1], power_of(byte[i]));
    }
    if (a.v) {
      uint32_t word[E][2] = {}, byte[E];
#pragma unroll
      for (int i = 0; i < E; ++i) byte[i] = 127;
      if (wide) {
        const uint8_t* const from = a.pool.codes + (block[0] * 2 + 1) * bytes + ((at[0] >> 2) * dim + lane * 8) * 4;
        const W4 w[2] = {*reinterpret_cast<const W4*>(from), *reinterpret_cast<const W4*>(from + 16)};
        const uint32_t all = a.pool.scales[block[0] * 2 + 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t rows4[4] = {w[h][0], w[h][1], w[h][2], w[h][3]};
          uint32_t cols[4];
          turn_words(rows4, cols);
#pragma unroll
          for (int i = 0; i < E; ++i) word[i][h] = cols[i], byte[i] = all;
        }
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          if (!there[i]) continue;
          const uint8_t* const from = a.pool.codes + (block[i] * 2 + 1) * bytes + ((at[i] >> 2) * dim + lane * 8) * 4 + (at[i] & 3);
#pragma unroll
          for (int e = 0; e < 8; ++e) word[i][e >> 2] |= (uint32_t)from[e * 4] << 8 * (e & 3);
          byte[i] = a.pool.scales[block[i] * 2 + 1];
        }
      }
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (quad * E + i < a.tokens) *reinterpret_cast<Packed8Any*>(a.v + (quad * E + i) * a.v_token + head * a.v_head + lane * 8) = read8<BF>(word[i][0], word[i][1], power_of(byte[i]));
    }
  }
}

// ---- arguments ---------------------------------------------------------------

int lane_bits_of(int dim) {
  int bits = 2;
  while ((8 << bits) < dim) ++bits;
  return bits;
}

// A pool's geometry; `data`: its memory is needed too.
int pool_of(const macko_kv8_cache_t* c, bool data, Kv8Pool* p) {
  if (!c || c->pages < 0 || c->page_size < 1 || c->kv_heads < 1) return MACKO_E_INVALID_ARG;
  if (int st = check_head_dim(c->head_dim)) return st;
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0) return MACKO_E_UNSUPPORTED;
  if (c->kv_heads > 65536 || c->pages > INT32_MAX / c->page_size) return MACKO_E_UNSUPPORTED;
  if (data && c->pages > 0 && (!c->codes_dev || !aligned_to(c->codes_dev, 16) || !c->scales_dev || !aligned_to(c->scales_dev, 2))) return MACKO_E_INVALID_ARG;
  int bits = 0;
  while ((1 << bits) < c->page_size) ++bits;
  *p = Kv8Pool{static_cast<uint8_t*>(c->codes_dev), static_cast<uint8_t*>(c->scales_dev), c->pages, c->kv_heads, c->head_dim, bits};
  return MACKO_OK;
}

// From this many tokens on, with kLongTurns and more to a sequence, keys and values go by 16 rows and queries by macko_rotate's kernel.  With 32 heads on 8 of 128 channels, fp16 (by
// token, by 16): one sequence of 256 tokens 8 and 13 us, of 512 13 and 14, of 1024 22 and 15, of 4096 75 and 27; 1024 tokens of sequences with 8 each 22 and 15, with 4 23 and 23, with
// 2 23 and 38, with one 28 and 68.  512 of 32 on 32: 22 and 14; 512 of 16 on 4 of 256 channels 23 and 19; of 40 on 8 of 64 channels 11 and 13.
constexpr int64_t kManyTokens = 512, kLongTurns = 4;

template <bool BF, int LB>
int launch_append(AppendArgs& a, hipStream_t stream) {
  constexpr int LT = 1 << LB, PAIRS = Unit<LB>::PAIRS;
  a.groups = (a.pool.heads + PAIRS - 1) / PAIRS;
  const dim3 block(kBlock);
  if (a.start && a.tokens >= kManyTokens && a.tokens >= kLongTurns * a.batch) {
    a.rows = 16;
    a.groups = (a.groups + 3) / 4;
    hipLaunchKernelGGL((blocks_kernel<BF, LB>), dim3((unsigned)(2 * a.groups), (unsigned)std::min<int64_t>(kMostGrid, (a.tokens + 15) / 16)), block, 0, stream, a);
    MACKO_HIP_TRY(hipGetLastError());
    if (a.heads == 0) return MACKO_OK;
    const macko_rotation_t r{a.positions, a.table, a.table_rows, a.rot, a.interleaved, a.eps};
    return macko_rotate(a.tokens, a.heads, a.dim, BF ? MACKO_BF16 : MACKO_FP16, a.q, a.q_token, a.q_head, &r, a.q_weight, a.out, a.out_token, a.out_head, stream);
  }
  a.rows = 1;
  a.q_groups = (a.heads + kBlock / LT - 1) / (kBlock / LT);
  const dim3 grid((unsigned)(a.q_groups + (2 * a.groups + kBlock / kWave - 1) / (kBlock / kWave)), (unsigned)std::min<int64_t>(kMostGrid, a.tokens));
  hipLaunchKernelGGL((append_kernel<BF, LB>), grid, block, 0, stream, a);
  MACKO_HIP_TRY(hipGetLastError());
  return MACKO_OK;
}
template <bool BF>
int launch_append_type(AppendArgs& a, hipStream_t stream) {
  switch (lane_bits_of(a.dim)) {
    case 2: return launch_append<BF, 2>(a, stream);
    case 3: return launch_append<BF, 3>(a, stream);
    case 4: return launch_append<BF, 4>(a, stream);
    default: return launch_append<BF, 5>(a, stream);
  }
}

template <bool BF, int E>
void launch_read(ReadArgs& a, hipStream_t stream) {
  a.items = (a.tokens + E - 1) / E * a.pool.heads;
  const int bits = lane_bits_of(a.pool.dim);
  const int64_t groups = kBlock >> bits;
  const dim3 grid((unsigned)std::min(kMostBlocks, (a.items + groups - 1) / groups)), block(kBlock);
  switch (bits) {
    case 2: hipLaunchKernelGGL((read_kernel<BF, 2, E>), grid, block, 0, stream, a); break;
    case 3: hipLaunchKernelGGL((read_kernel<BF, 3, E>), grid, block, 0, stream, a); break;
    case 4: hipLaunchKernelGGL((read_kernel<BF, 4, E>), grid, block, 0, stream, a); break;
    default: hipLaunchKernelGGL((read_kernel<BF, 5, E>), grid, block, 0, stream, a); break;
  }
}
// Few entries: one to a group of lanes, whose loads are a fourth as many.  Entries in order and in no order, one to a group and four, us: 257 of 8 heads of 256 channels 4.2, 4.2 and 4.5, 7.9;
// 1024 of 8 of 64 3.8, 3.8 and 4.4, 7.8; of 8 of 128 (131072 lanes) 4.8, 4.9 and 4.7, 8.2; of 8 of 256 7.4, 7.4 and 5.3, 8.6.
constexpr int64_t kFewLanes = 1 << 17;
template <bool BF>
void launch_read_type(ReadArgs& a, hipStream_t stream) {
  if (a.tokens * a.pool.heads << lane_bits_of(a.pool.dim) <= kFewLanes) launch_read<BF, 1>(a, stream);
  else launch_read<BF, 4>(a, stream);
}

// The attention's arguments are those of the 4-bit cache.
int attention_of(const macko_kv8_cache_t* cache, const macko_kv_attention_args_t* g, bool pointers, Kv8Attention* a) {
  Kv8Pool pool;
  if (int st = pool_of(cache, pointers, &pool)) return st;
  a->scales = pool.scales;
  return kv_attention_of(KvPool{pool.codes, pool.pages, pool.heads, pool.dim, pool.page_bits}, g, pointers, &a->a);
}

}  // namespace
}  // namespace macko

extern "C" {

using namespace macko;

int64_t macko_kv8_cache_bytes(const macko_kv8_cache_t* cache, int64_t* scale_bytes) {
  Kv8Pool p;
  if (scale_bytes) *scale_bytes = 0;
  if (int st = pool_of(cache, false, &p)) return st;
  const int64_t blocks = (p.pages * p.heads) << (p.page_bits - kBlockBits);
  if (scale_bytes) *scale_bytes = blocks * 2;
  return blocks * 2 * kBlockTokens * p.dim;
}

int macko_kv8_append(const macko_kv8_cache_t* cache, const macko_kv8_append_args_t* g, void* stream) {
  if (!g || g->tokens < 0 || g->heads < 0 || g->batch < 0 || g->table_width < 0 || g->table_stride < 0 || (g->type != MACKO_FP16 && g->type != MACKO_BF16)) return MACKO_E_INVALID_ARG;
  Kv8Pool pool;
  if (int st = pool_of(cache, true, &pool)) return st;
  if (int st = check_rotation(g->rotation, pool.dim, g->tokens)) return st;
  if (!g->start_dev && g->tokens != g->batch) return MACKO_E_INVALID_ARG;
  if (g->tokens == 0) return MACKO_OK;
  if (g->tokens > INT32_MAX - 64 || g->heads > 65536) return MACKO_E_UNSUPPORTED;
  if (!heads_fine(g->k_dev, g->k_token, g->k_head) || !heads_fine(g->v_dev, g->v_token, g->v_head) || !aligned_to(g->q_weight_dev, 2) || !aligned_to(g->k_weight_dev, 2) ||
      !aligned_to(g->start_dev, 4) || !aligned_to(g->lengths_dev, 4) || !aligned_to(g->tables_dev, 4) || (g->batch > 0 && !g->lengths_dev) ||
      (g->batch > 0 && g->table_width > 0 && !g->tables_dev))
    return MACKO_E_INVALID_ARG;
  if (g->heads > 0 && (!heads_fine(g->q_dev, g->q_token, g->q_head) || !heads_fine(g->q_out_dev, g->q_out_token, g->q_out_head))) return MACKO_E_INVALID_ARG;
  AppendArgs a{};
  a.q = static_cast<const uint16_t*>(g->q_dev), a.q_token = g->q_token, a.q_head = g->q_head;
  a.k = static_cast<const uint16_t*>(g->k_dev), a.k_token = g->k_token, a.k_head = g->k_head;
  a.v = static_cast<const uint16_t*>(g->v_dev), a.v_token = g->v_token, a.v_head = g->v_head;
  a.out = static_cast<uint16_t*>(g->q_out_dev), a.out_token = g->q_out_token, a.out_head = g->q_out_head;
  a.q_weight = static_cast<const uint16_t*>(g->q_weight_dev), a.k_weight = static_cast<const uint16_t*>(g->k_weight_dev);
  a.positions = g->rotation.positions_dev, a.table = g->rotation.table_dev, a.table_rows = g->rotation.table_rows;
  a.rot = g->rotation.rot, a.interleaved = g->rotation.interleaved != 0, a.eps = g->rotation.eps;
  a.tables = g->tables_dev, a.lengths = g->lengths_dev, a.start = g->start_dev, a.table_stride = g->table_stride;
  a.table_width = g->table_width, a.batch = g->batch;
  a.pool = pool;
  a.tokens = g->tokens, a.heads = g->heads, a.dim = pool.dim;
  return g->type == MACKO_BF16 ? launch_append_type<true>(a, static_cast<hipStream_t>(stream)) : launch_append_type<false>(a, static_cast<hipStream_t>(stream));
}

int macko_kv8_read(const macko_kv8_cache_t* cache, int64_t tokens, const int32_t* slots_dev, int type, void* k_out_dev, int64_t k_token, int64_t k_head,
                   void* v_out_dev, int64_t v_token, int64_t v_head, void* stream) {
  if (tokens < 0 || (type != MACKO_FP16 && type != MACKO_BF16)) return MACKO_E_INVALID_ARG;
  Kv8Pool pool;
  if (int st = pool_of(cache, true, &pool)) return st;
  if (tokens == 0 || (!k_out_dev && !v_out_dev)) return MACKO_OK;
  if (tokens > INT32_MAX) return MACKO_E_UNSUPPORTED;
  if (!slots_dev || !aligned_to(slots_dev, 4) || (k_out_dev && !heads_fine(k_out_dev, k_token, k_head)) || (v_out_dev && !heads_fine(v_out_dev, v_token, v_head)))
    return MACKO_E_INVALID_ARG;
  ReadArgs a{pool, slots_dev, tokens, pool.pages << pool.page_bits, 0, static_cast<uint16_t*>(k_out_dev), k_token, k_head,
                   static_cast<uint16_t*>(v_out_dev), v_token, v_head};
  if (type == MACKO_BF16) launch_read_type<true>(a, static_cast<hipStream_t>(stream));
  else launch_read_type<false>(a, static_cast<hipStream_t>(stream));
  MACKO_HIP_TRY(hipGetLastError());
  return MACKO_OK;
}

int64_t macko_kv8_attention_workspace(const macko_kv8_cache_t* cache, const macko_kv_attention_args_t* args) {
  Kv8Attention a;
  if (int st = attention_of(cache, args, false, &a)) return st;
  return 4 * kv8_attention_workspace(a.a);
}

int macko_kv8_attention(const macko_kv8_cache_t* cache, const macko_kv_attention_args_t* args, void* workspace_dev, int64_t workspace_bytes, void* stream) {
  Kv8Attention a;
  if (int st = attention_of(cache, args, true, &a)) return st;
  if (a.a.tokens == 0 || a.a.batch == 0) return MACKO_OK;
  const int64_t need = 4 * kv8_attention_workspace(a.a);
  if (need > 0 && (!workspace_dev || !aligned_to(workspace_dev, 16) || workspace_bytes < need)) return MACKO_E_INVALID_ARG;
  return launch_kv8_attention(a, static_cast<float*>(workspace_dev), static_cast<hipStream_t>(stream));
}

}  // extern "C"
