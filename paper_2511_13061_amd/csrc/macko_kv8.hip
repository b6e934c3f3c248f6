// The 8-bit key/value cache: new tokens into it (macko_kv8_append) and its values back (macko_kv8_read); the C entry points of these and of the attention
// over the cache.
//
// A value takes 2 bytes in and 1 out, or the other way round, and some ten operations: memory bounds long calls, a launch short ones.
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
  int64_t tokens, q_items, q_waves, waves;       // of queries: bundles of heads; wavefronts of queries, and of the launch
  int32_t table_width, batch, heads, bundles, dim, rot, interleaved;
  int32_t rows;              // of a wavefront that stores: it takes the blocks that begin in them
  int32_t pair_waves;        // wavefronts that share a token's keys and values out
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
__device__ inline Turn turn_of(const AppendArgs& a, int64_t token, int lane) {
  Turn t;
  const int half = a.rot >> 4;                            // lanes of half a turned part
  t.other = lane >= 2 * half ? lane : lane < half ? lane + half : lane - half;
  t.placed = true;
  int64_t at = 0;
  if (a.rot > 0) {
    at = a.positions[token];
    t.placed = at >= 0 && at < a.table_rows;
  }
  t.turned = t.placed && lane < 2 * half;
  if (t.turned) {
    const float* const row = a.table + at * a.rot + (a.interleaved ? lane * 4 : (lane < half ? lane : t.other) * 8);
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

// A wavefront either turns queries (groups of LT lanes take BUNDLE heads of a token) or stores: it takes the blocks of 16 places of a sequence whose first new
// token is one of its `rows` rows, for keys or values of one head or, where a block takes fewer lanes, of several.  In a block lane (t, l) has 8 channels of TPL
// places, so that the values' words, 4 places of a channel, are made without another lane; all of a block's new tokens are there at once, and the largest
// magnitude takes one round of exchanges.  Only where the byte of scale grows are the block's earlier tokens read at all.
template <bool BF, int LB, int BUNDLE>
__global__ __launch_bounds__(kBlock) void append_kernel(const AppendArgs a) {
  constexpr int LT = 1 << LB, TG = LT <= 16 ? 4 : 2, GROUP = LT * TG, TPL = 16 / TG, PAIRS = kWave / GROUP;
  const int lane64 = threadIdx.x & 63, lane = lane64 & (LT - 1);
  const bool mine = lane * 8 < a.dim;
  for (int64_t wave = (int64_t)blockIdx.x * (kBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); wave < a.waves; wave += (int64_t)gridDim.x * (kBlock / kWave)) {
    if (wave < a.q_waves) {
      const int64_t item = wave * (kWave / LT) + (lane64 >> LB), token = min(item / a.bundles, a.tokens - 1);
      const int head = (int)(item - item / a.bundles * a.bundles) * BUNDLE;
      const bool there = item < a.q_items;
      Packed8 raw[BUNDLE];
#pragma unroll
      for (int i = 0; i < BUNDLE; ++i) {
        raw[i] = Packed8{0, 0, 0, 0};
        if (there && mine && head + i < a.heads) raw[i] = *reinterpret_cast<const Packed8Any*>(a.q + token * a.q_token + (head + i) * a.q_head + lane * 8);
      }
      const Turn t = turn_of(a, token, lane);
#pragma unroll
      for (int i = 0; i < BUNDLE; ++i) {
        float y[8];
        finish<BF, LT>(a, raw[i], a.q_weight, t, lane, y);
        if (there && mine && head + i < a.heads) *reinterpret_cast<Packed8Any*>(a.out + token * a.out_token + (head + i) * a.out_head + lane * 8) = pack8<BF>(y);
      }
      continue;
    }
    const int64_t unit = wave - a.q_waves, chunk = unit / a.pair_waves;
    const int pair = (int)(unit - chunk * a.pair_waves) * PAIRS + lane64 / GROUP;        // keys' heads, then values'
    const bool there = pair < 2 * a.pool.heads, value = pair >= a.pool.heads && there;
    const int head = there ? pair - (value ? a.pool.heads : 0) : 0;
    const int first_place = (lane64 / LT) % TG * TPL;
    const int row_end = (int)min((chunk + 1) * a.rows, a.tokens);
    int row = (int)(chunk * a.rows);
    int b = a.start ? sequence_at(a.start, a.batch, row, lane64) : row;
    if (b < 0) b = 0, row = min(max(a.start[0], 0), row_end);
    while (row < row_end && b < a.batch) {
      const int from = a.start ? min(max(a.start[b], 0), (int)a.tokens) : row, to = a.start ? min(max(a.start[b + 1], 0), (int)a.tokens) : row + 1;
      if (row >= to) {                                    // the sequence's rows are over, or it has none
        ++b;
        continue;
      }
      const int length = min(max(a.lengths[b], 0), kMostTokens);
      int place = length - (to - row);
      if (place < 0) {                                    // more rows than tokens: these have no place
        row = min(to, row - place);
        if (row >= to) ++b;
        continue;
      }
      const int first = place & 15, last = min(16, first + (to - row));      // places of the block that are new
      const int row0 = row - first, sequence = b;
      const bool begins = first == 0 || row == from;
      row = row0 + last;
      if (row >= to) ++b;
      if (!begins) continue;                              // the block begins in rows before these
      const int index = place >> a.pool.page_bits;
      const int page = index < a.table_width ? a.tables[sequence * a.table_stride + index] : -1;
      if (page < 0 || page >= a.pool.pages) continue;

      const int64_t block = kv8_block(a.pool, page, head, place & ((1 << a.pool.page_bits) - 1));
      uint8_t* const scale = a.pool.scales + block * 2 + value;
      uint8_t* const codes = a.pool.codes + (block * 2 + value) * (int64_t)(kBlockTokens * a.dim);
      const uint32_t had = first > 0 ? *scale : 0u;
      const uint16_t* const src = value ? a.v + head * a.v_head + lane * 8 : a.k + head * a.k_head + lane * 8;
      const int64_t stride = value ? a.v_token : a.k_token;
      Packed8 raw[TPL];
#pragma unroll
      for (int r = 0; r < TPL; ++r) {
        const int p = first_place + r;
        raw[r] = Packed8{0, 0, 0, 0};
        if (there && mine && p >= first && p < last) raw[r] = *reinterpret_cast<const Packed8Any*>(src + (int64_t)(row0 + p) * stride);
      }
      float y[TPL][8];
      uint32_t most = 0;
      bool odd = false;                                   // something is not finite
#pragma unroll
      for (int r = 0; r < TPL; ++r) {
        const int p = first_place + r;
        if (value) {
          unpack8<BF>(raw[r], y[r]);
        } else {
          const Turn t = turn_of(a, row0 + min(max(p, first), last - 1), lane);
          finish<BF, LT>(a, raw[r], a.k_weight, t, lane, y[r]);
        }
        if (p < first || p >= last) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t bits = __builtin_bit_cast(uint32_t, y[r][e]) & 0x7FFFFFFFu;
          odd = odd || bits >= 0x7F800000u;
          most = max(most, bits >= 0x7F800000u ? 0u : bits);
        }
      }
      const uint32_t byte = max(scale_byte(most_over<GROUP>(most)), had);
      const bool grown = first > 0 && byte > had;
      const float down = power_of(254u - min(byte, 254u)), again = power_of(127u - min(byte - had, 127u));
      if (there && (lane64 & (GROUP - 1)) == 0 && (first == 0 || grown)) *scale = (uint8_t)byte;
      const int begin = grown ? 0 : first;                // places that are written
      if (!there || !mine) continue;
      uint32_t word[TPL][2];                              // 8 codes of a place
#pragma unroll
      for (int r = 0; r < TPL; ++r) {
        const int p = first_place + r;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = y[r][e] * down;
        word[r][0] = codes_of(x), word[r][1] = codes_of(x + 4);
        if (odd) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if ((__builtin_bit_cast(uint32_t, y[r][e]) & 0x7FFFFFFFu) >= 0x7F800000u)
              word[r][e >> 2] = (word[r][e >> 2] & ~(255u << 8 * (e & 3))) | 0x7Fu << 8 * (e & 3);
          }
        }
        if (grown && p < first) {
          uint32_t old[2];
          if (value) {
            old[0] = old[1] = 0;
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
            for (int e = 0; e < 4; ++e) z[e] *= again;
            uint32_t w = codes_of(z);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if ((old[h] >> 8 * e & 0x7Fu) == 0x7Fu) w = (w & ~(255u << 8 * e)) | 0x7Fu << 8 * e;
            }
            word[r][h] = w;
          }
        }
        if (!value && p >= begin && p < last) *reinterpret_cast<W2*>(codes + p * a.dim + lane * 8) = W2{word[r][0], word[r][1]};
      }
      if (!value) continue;
#pragma unroll
      for (int u = 0; u < TPL / 4; ++u) {
        const int p = first_place + 4 * u;
        uint8_t* const quad = codes + ((p >> 2) * a.dim + lane * 8) * 4;
        uint32_t out[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t rows4[4] = {word[4 * u][h], word[4 * u + 1][h], word[4 * u + 2][h], word[4 * u + 3][h]};
          uint32_t cols[4];
          turn_words(rows4, cols);
#pragma unroll
          for (int e = 0; e < 4; ++e) out[4 * h + e] = cols[e];
        }
        if (p >= begin && p + 4 <= last) {
          *reinterpret_cast<W4*>(quad) = W4{out[0], out[1], out[2], out[3]};
          *reinterpret_cast<W4*>(quad + 16) = W4{out[4], out[5], out[6], out[7]};
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (p + i < begin || p + i >= last) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) quad[e * 4 + i] = (uint8_t)(out[e] >> 8 * i);
          }
        }
      }
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

// A group of LT lanes takes 4 entries of the list for one head.  Where they are 4 tokens in the order in which values lie together, the values come as whole
// words; else byte by byte.
template <bool BF, int LB>
__global__ __launch_bounds__(kBlock) void read_kernel(const ReadArgs a) {
  constexpr int LT = 1 << LB;
  const int lane = threadIdx.x & (LT - 1), dim = a.pool.dim;
  const bool mine = lane * 8 < dim;
  for (int64_t item = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> LB; item < a.items; item += (int64_t)gridDim.x * (kBlock >> LB)) {
    const int64_t quad = item / a.pool.heads;
    const int head = (int)(item - quad * a.pool.heads);
    if (!mine) continue;
    int64_t block[4];
    int at[4];
    bool there[4], wide = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t slot = quad * 4 + i < a.tokens ? a.slots[quad * 4 + i] : -1;
      there[i] = slot >= 0 && slot < a.slots_held;
      block[i] = there[i] ? kv8_block(a.pool, slot >> a.pool.page_bits, head, (int)(slot & ((1 << a.pool.page_bits) - 1))) : 0;
      at[i] = (int)(slot & 15);
      wide = wide && there[i] && block[i] == block[0] && at[i] == (at[0] & ~3) + i;
    }
    const int64_t bytes = kBlockTokens * dim;
    if (a.k) {
      W2 word[4];
      uint32_t byte[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        word[i] = W2{0, 0};
        byte[i] = 127;
        if (there[i]) {
          word[i] = *reinterpret_cast<const W2*>(a.pool.codes + block[i] * 2 * bytes + at[i] * dim + lane * 8);
          byte[i] = a.pool.scales[block[i] * 2];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (quad * 4 + i < a.tokens) *reinterpret_cast<Packed8Any*>(a.k + (quad * 4 + i) * a.k_token + head * a.k_head + lane * 8) = read8<BF>(word[i][0], word[i][1], power_of(byte[i]));
    }
    if (a.v) {
      uint32_t word[4][2] = {}, byte[4] = {127, 127, 127, 127};
      if (wide) {
        const uint8_t* const from = a.pool.codes + (block[0] * 2 + 1) * bytes + ((at[0] >> 2) * dim + lane * 8) * 4;
        const W4 w[2] = {*reinterpret_cast<const W4*>(from), *reinterpret_cast<const W4*>(from + 16)};
        byte[0] = byte[1] = byte[2] = byte[3] = a.pool.scales[block[0] * 2 + 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t rows4[4] = {w[h][0], w[h][1], w[h][2], w[h][3]};
          uint32_t cols[4];
          turn_words(rows4, cols);
#pragma unroll
          for (int i = 0; i < 4; ++i) word[i][h] = cols[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!there[i]) continue;
          const uint8_t* const from = a.pool.codes + (block[i] * 2 + 1) * bytes + ((at[i] >> 2) * dim + lane * 8) * 4 + (at[i] & 3);
#pragma unroll
          for (int e = 0; e < 8; ++e) word[i][e >> 2] |= (uint32_t)from[e * 4] << 8 * (e & 3);
          byte[i] = a.pool.scales[block[i] * 2 + 1];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (quad * 4 + i < a.tokens) *reinterpret_cast<Packed8Any*>(a.v + (quad * 4 + i) * a.v_token + head * a.v_head + lane * 8) = read8<BF>(word[i][0], word[i][1], power_of(byte[i]));
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

// Rows that a wavefront looks for blocks in: 16 where long sequences are likely (one block begins in them) and the launch is large, else 1.
constexpr int64_t kManyWaves = 16384;

template <bool BF, int LB>
int launch_append(AppendArgs& a, hipStream_t stream) {
  constexpr int LT = 1 << LB, PAIRS = kWave / (LT * (LT <= 16 ? 4 : 2));
  constexpr int kBundle = 4;
  const int64_t cus = device_cu_count();
  const bool bundle = (a.tokens * a.heads) / (kWave / LT) >= cus * 32;
  a.bundles = a.heads == 0 ? 1 : bundle ? (a.heads + kBundle - 1) / kBundle : a.heads;
  a.q_items = a.heads == 0 ? 0 : a.tokens * a.bundles;
  a.q_waves = (a.q_items + kWave / LT - 1) / (kWave / LT);
  a.pair_waves = (2 * a.pool.heads + PAIRS - 1) / PAIRS;
  a.rows = a.start && a.tokens * a.pair_waves >= kManyWaves ? 16 : 1;
  a.waves = a.q_waves + (a.tokens + a.rows - 1) / a.rows * a.pair_waves;
  const dim3 grid((unsigned)std::min(kMostBlocks, (a.waves + kBlock / kWave - 1) / (kBlock / kWave))), block(kBlock);
  if (bundle) hipLaunchKernelGGL((append_kernel<BF, LB, kBundle>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((append_kernel<BF, LB, 1>), grid, block, 0, stream, a);
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

template <bool BF>
void launch_read(const ReadArgs& a, hipStream_t stream) {
  const int bits = lane_bits_of(a.pool.dim);
  const int64_t groups = kBlock >> bits;
  const dim3 grid((unsigned)std::min(kMostBlocks, (a.items + groups - 1) / groups)), block(kBlock);
  switch (bits) {
    case 2: hipLaunchKernelGGL((read_kernel<BF, 2>), grid, block, 0, stream, a); break;
    case 3: hipLaunchKernelGGL((read_kernel<BF, 3>), grid, block, 0, stream, a); break;
    case 4: hipLaunchKernelGGL((read_kernel<BF, 4>), grid, block, 0, stream, a); break;
    default: hipLaunchKernelGGL((read_kernel<BF, 5>), grid, block, 0, stream, a); break;
  }
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
  const ReadArgs a{pool, slots_dev, tokens, pool.pages << pool.page_bits, (tokens + 3) / 4 * pool.heads, static_cast<uint16_t*>(k_out_dev), k_token, k_head,
                   static_cast<uint16_t*>(v_out_dev), v_token, v_head};
  if (type == MACKO_BF16) launch_read<true>(a, static_cast<hipStream_t>(stream));
  else launch_read<false>(a, static_cast<hipStream_t>(stream));
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
