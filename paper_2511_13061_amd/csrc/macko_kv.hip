// Heads between the products of a decoder layer: norm and position of queries and keys, the 4-bit key/value cache that new tokens go into
// (macko_kv_append) and its values back (macko_kv_read); the C entry points of these and of the attention over the cache.
//
// All of it moves bytes: a value takes 2 bytes in, 2 or 17/32 out and some ten operations.  A head of a token is the unit of work, a
// group of 4 to 32 lanes with 8 channels each takes it in one 16-byte load a lane; what a head needs of other lanes (the sum of a norm, the
// other half of a pair, a group's largest magnitude) goes through lane shuffles, so that nothing is read twice and in-place calls are safe.
#include <cmath>
#include <type_traits>

#include "macko_kv.h"

namespace macko {
namespace {

constexpr int kBlock = 256;
typedef float V4 __attribute__((ext_vector_type(4)));
constexpr int64_t kMostBlocks = (int64_t{1} << 24) - 1;  // a launch has fewer than 2^32 threads

struct Heads {
  const uint16_t* x;
  int64_t token, head;       // strides in elements
  const uint16_t* weight;
  int32_t heads;
  int32_t bundles;           // of a token: heads that a group of lanes takes together
  int64_t blocks;            // that the launch has for these heads
};
// Results of a large call leave the caches to others: they are larger than those, and what is read stays longer.
template <bool STREAM>
__device__ inline void put8(uint16_t* to, Packed8 x) {
  if (STREAM) __builtin_nontemporal_store((Packed8Any)x, reinterpret_cast<Packed8Any*>(to));
  else *reinterpret_cast<Packed8Any*>(to) = x;
}

struct TurnArgs {
  Heads part[3];             // queries, keys, values
  uint16_t* out;
  int64_t out_token, out_head;
  const int32_t* positions;
  const int32_t* slots;
  const float* table;
  int64_t table_rows;
  KvPool pool;
  int64_t tokens, slots_held, blocks;
  int32_t dim, rot, interleaved;
  int32_t lane_bits;         // log2 of the lanes of a head
  float eps;
};

template <int CTRL>
__device__ inline uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;      // quad_perm [1,0,3,2] and [2,3,0,1], row_half_mirror, row_mirror

// The sum over a group of 4 to 32 lanes, in all of them.
__device__ inline float group_sum(float x, int lanes) {
  auto with = [](float y, uint32_t far) { return y + __builtin_bit_cast(float, far); };
  x = with(x, dpp<kSwap1>(__builtin_bit_cast(uint32_t, x)));
  x = with(x, dpp<kSwap2>(__builtin_bit_cast(uint32_t, x)));
  if (lanes > 4) x = with(x, dpp<kMirror8>(__builtin_bit_cast(uint32_t, x)));      // quads hold one sum each: any lane of the other will do
  if (lanes > 8) x = with(x, dpp<kMirror16>(__builtin_bit_cast(uint32_t, x)));
  if (lanes > 16) x += __shfl_xor(x, 16);
  return x;
}

// The 4-bit codes of 8 channels of a group that 4 neighbouring lanes hold, 2 to a byte, and the group's byte.
__device__ inline uint32_t encode8(const float* y, uint32_t* byte) {
  uint32_t bits = 0;                                     // magnitudes are ordered as their bits are, infinities and NaN above all
#pragma unroll
  for (int i = 0; i < 8; ++i) bits = max(bits, __builtin_bit_cast(uint32_t, y[i]) & 0x7FFFFFFFu);
  bits = max(bits, dpp<kSwap1>(bits));
  bits = max(bits, dpp<kSwap2>(bits));
  // the exponent of most / 7, rounded up: 7 = 1.75 * 2^2, and a mantissa above 1.75 carries
  const uint32_t e = (bits + 0x1FFFFFu) >> 23;
  const uint32_t b = bits >= 0x7F800000u ? 255u : e > 2u ? min(e - 2u, kMostByte) : 0u;
  *byte = b;
  const float unit = __builtin_bit_cast(float, b << 23);
  uint32_t word = 0;
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[0], y[1], unit, 0);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[2], y[3], unit, 1);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[4], y[5], unit, 2);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[6], y[7], unit, 3);
  return word;
}

// Lanes 4g + 2u + v hold the codes of channels 32g + 16u + 8v + e as keys are stored, 8 of them in a word; a byte of the values' layout takes
// the same e from u = 0 and u = 1.  The word of lane 4g + 2u + v here: bytes m = 8v + 4u + (0 .. 3) of group g.  And back.
__device__ inline uint32_t pair_values(uint32_t word, bool upper) {
  const uint32_t far = dpp<kSwap2>(word);
  const uint32_t low = upper ? far >> 16 : word & 0xFFFFu, high = upper ? word >> 16 : far & 0xFFFFu;
  // 4 codes to the low halves of 4 bytes, 4 to the high ones
  const uint32_t a = (low | low << 8) & 0x00FF00FFu, b = (high | high << 8) & 0x00FF00FFu;
  return ((a | a << 4) & 0x0F0F0F0Fu) | ((b | b << 4) & 0x0F0F0F0Fu) << 4;
}
__device__ inline uint32_t unpair_values(uint32_t word, bool upper) {
  uint32_t a = word & 0x0F0F0F0Fu, b = word >> 4 & 0x0F0F0F0Fu;
  a = (a | a >> 4) & 0x00FF00FFu, b = (b | b >> 4) & 0x00FF00FFu;
  a = (a | a >> 8) & 0xFFFFu, b = (b | b >> 8) & 0xFFFFu;
  const uint32_t give = upper ? a : b, far = dpp<kSwap2>(give);
  return upper ? far | b << 16 : a | far << 16;
}
// A 4 x 4 matrix of bytes, a row in each of the lanes whose numbers differ in bits 2 and 3, turned over.
__device__ inline uint32_t turn_bytes(uint32_t word, int lane) {
  uint32_t far = (uint32_t)__shfl_xor((int)word, 4);
  word = __builtin_amdgcn_perm(far, word, lane & 4 ? 0x03070105u : 0x06020400u);
  far = (uint32_t)__shfl_xor((int)word, 8);
  return __builtin_amdgcn_perm(far, word, lane & 8 ? 0x03020706u : 0x05040100u);
}

// Memory bounds it: 8191 tokens of 40 heads with 128 channels, normalised and turned, 33 us (5.1 TB/s; a copy reaches 4.8 to 5.2); 16384 tokens of 32 heads into
// the cache, q, k and v, 74 us.  One token takes 3 us, a launch's own time.  By width (1024 channels of keys a token, 4 times as many of queries; TB/s): 32 channels
// 3.7, 64 4.7, 96 4.1, 128 4.9, 160 3.7, 192 3.9, 224 4.1, 256 4.8: value codes go in whole words with 128 channels and byte by byte otherwise, and with
// other than powers of two some lanes have no channels (4 of 16 with 96, 4 to 12 of 32 with 160 to 224).
// Queries, keys and values have workgroups of their own.  A group of lanes takes BUNDLE heads of a token, whose loads are under way together;
// position, table row and weight serve all of them.
template <bool BF, int BUNDLE>
__global__ __launch_bounds__(kBlock) void turn_kernel(const TurnArgs a) {
#pragma clang fp contract(off)     // products are rounded before they are added: keys near the edge of two codes take the same one everywhere
  const int lanes = 1 << a.lane_bits, lane = threadIdx.x & (lanes - 1), groups = kBlock >> a.lane_bits, n = a.dim / 32;
  const bool mine = lane * 8 < a.dim;
  for (int64_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
    const int kind = block < a.part[0].blocks ? 0 : block < a.part[0].blocks + a.part[1].blocks ? 1 : 2;
    const Heads& part = a.part[kind];
    const int64_t first = (block - (kind > 0 ? a.part[0].blocks : 0) - (kind > 1 ? a.part[1].blocks : 0)) * groups;
    const int64_t first_token = first / part.bundles;
    const uint32_t at_bundle = (uint32_t)(first - first_token * part.bundles) + (threadIdx.x >> a.lane_bits), skip = at_bundle / (uint32_t)part.bundles;
    const int64_t token = first_token + skip;
    const int head = (int)(at_bundle - skip * part.bundles) * BUNDLE;
    if (token >= a.tokens) continue;                      // the same for all lanes of a group

    Packed8 raw[BUNDLE];
    const uint16_t* const src = part.x + token * part.token + head * part.head + lane * 8;
#pragma unroll
    for (int i = 0; i < BUNDLE; ++i) {
      raw[i] = Packed8{0, 0, 0, 0};
      if (mine && head + i < part.heads) raw[i] = *reinterpret_cast<const Packed8Any*>(src + i * part.head);
    }
    bool placed = true;
    int64_t at = 0, slot = 0;
    if (a.rot > 0) {
      at = a.positions[token];
      placed = at >= 0 && at < a.table_rows;
    }
    if (kind > 0) slot = a.slots[token];
    const int half = a.rot >> 4;                          // lanes of half a turned part
    const bool turned = kind < 2 && placed && lane < 2 * half;
    const int other = lane >= 2 * half ? lane : lane < half ? lane + half : lane - half;      // the lane that holds the other channels of this one's pairs
    float c[8], s[8], w[8] = {};
    if (turned) {
      const float* const row = a.table + at * a.rot + (a.interleaved ? lane * 4 : (lane < half ? lane : other) * 8);
      *reinterpret_cast<V4*>(c) = *reinterpret_cast<const V4*>(row);
      *reinterpret_cast<V4*>(s) = *reinterpret_cast<const V4*>(row + a.rot / 2);
      if (!a.interleaved) {
        *reinterpret_cast<V4*>(c + 4) = *reinterpret_cast<const V4*>(row + 4);
        *reinterpret_cast<V4*>(s + 4) = *reinterpret_cast<const V4*>(row + a.rot / 2 + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = lane < half ? -s[i] : s[i];
      }
    }
    if (part.weight && mine) unpack8<BF>(*reinterpret_cast<const Packed8Any*>(part.weight + lane * 8), w);

    // A head of the bundle, normalised and turned; what varies by call and not by lane is settled outside the loops.
    auto finish = [&](Packed8 x, float* y, auto normed, auto interleaved) {
      unpack8<BF>(x, y);
      if constexpr (normed) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(y[e], y[e], sum);
        const float r = rsqrtf(group_sum(sum, lanes) / (float)a.dim + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = y[e] * r * w[e];
      }
      if (a.rot == 0) return;
      if constexpr (interleaved) {
        if (turned) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float u = y[2 * e], v = y[2 * e + 1];
            y[2 * e] = u * c[e] - v * s[e];
            y[2 * e + 1] = u * s[e] + v * c[e];
          }
        }
      } else {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], other, lanes);
        if (turned) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = y[e] * c[e] + z[e] * s[e];
        }
      }
    };
    const bool stored = placed && slot >= 0 && slot < a.slots_held;
    const KvToken to = kv_token(a.pool, kind > 0 && stored ? slot >> a.pool.page_bits : 0, head, kind > 0 && stored ? (int)(slot & ((1 << a.pool.page_bits) - 1)) : 0);
    const int64_t piece = kv_piece_bytes(int64_t{1} << a.pool.page_bits, a.dim);
    auto heads = [&](auto normed, auto interleaved) {
      uint16_t* const out = a.out + token * a.out_token + head * a.out_head + lane * 8;
#pragma unroll
      for (int i = 0; i < BUNDLE; ++i) {
        if (head + i >= part.heads) break;
        float y[8];
        finish(raw[i], y, normed, interleaved);
        if (kind == 0) {
          Packed8 x = pack8<BF>(y);
          if (__any(!placed) && !placed) x = Packed8{0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu};      // NaN in both types
          if (mine) put8<(BUNDLE > 1)>(out + i * a.out_head, x);
        } else {
          uint32_t byte;
          const uint32_t word = encode8(y, &byte);
          if (stored && mine) {
            reinterpret_cast<uint32_t*>(to.keys + i * piece)[lane] = word;
            if ((lane & 3) == 0) to.key_bytes[i * piece + (lane >> 2)] = (uint8_t)byte;
          }
        }
      }
    };
    typedef std::integral_constant<bool, true> Yes;
    typedef std::integral_constant<bool, false> No;
    if (kind < 2) {
      if (part.weight) a.interleaved ? heads(Yes{}, Yes{}) : heads(Yes{}, No{});
      else a.interleaved ? heads(No{}, Yes{}) : heads(No{}, No{});
      continue;
    }
    uint8_t* const at_m = to.values + ((lane & 1) * 8 + (lane & 2) * 2) * 4 * n + (n == 4 ? (lane >> 2) * 16 : lane >> 2);
#pragma unroll
    for (int i = 0; i < BUNDLE; ++i) {
      if (head + i >= part.heads) break;
      float y[8];
      unpack8<BF>(raw[i], y);
      uint32_t byte;
      uint32_t word = pair_values(encode8(y, &byte), lane & 2);
      if (n == 4) word = turn_bytes(word, lane);
      if (!stored || !mine) continue;
      if (n == 4) {                                       // a whole word a lane
        *reinterpret_cast<uint32_t*>(at_m + i * piece) = word;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) at_m[i * piece + e * 4 * n] = (uint8_t)(word >> (8 * e));
      }
      if ((lane & 3) == 0) to.value_bytes[i * piece + (lane >> 2)] = (uint8_t)byte;
    }
  }
}

struct ReadArgs {
  KvPool pool;
  const int32_t* slots;
  int64_t tokens, slots_held, blocks;
  uint16_t* k;
  int64_t k_token, k_head;
  uint16_t* v;
  int64_t v_token, v_head;
  int32_t lane_bits, bundles;
};

// Two 4-bit codes as 16-bit values, times 2^(b - 127).
template <bool BF, int BYTE>
__device__ inline uint32_t decode2(uint32_t word, float unit) {
  if (BF) {
    typedef __bf16 B2 __attribute__((ext_vector_type(2)));
    const B2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, BYTE);
    return __builtin_bit_cast(uint32_t, x);
  }
  typedef _Float16 H2 __attribute__((ext_vector_type(2)));
  const H2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, unit, BYTE);
  return __builtin_bit_cast(uint32_t, x);
}
template <bool BF>
__device__ inline Packed8 decode8(uint32_t word, uint32_t byte) {
  const float unit = __builtin_bit_cast(float, byte << 23);
  return {decode2<BF, 0>(word, unit), decode2<BF, 1>(word, unit), decode2<BF, 2>(word, unit), decode2<BF, 3>(word, unit)};
}

// Memory bounds it, and it writes four fifths of what it moves: 65536 slots of 8 heads with 128 channels 52 us, 6.4 TB/s (writing alone reaches 6.9).
// By width, TB/s: 32 channels 3.8, 64 5.8, 96 5.1, 160 5.4, 192 5.7, 224 5.8, 256 6.4.
template <bool BF, int BUNDLE>
__global__ __launch_bounds__(kBlock) void read_kernel(const ReadArgs a) {
  const int lanes = 1 << a.lane_bits, lane = threadIdx.x & (lanes - 1), groups = kBlock >> a.lane_bits, n = a.pool.dim / 32;
  const bool mine = lane * 8 < a.pool.dim;
  for (int64_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
    const int64_t first = block * groups, first_token = first / a.bundles;
    const uint32_t at_bundle = (uint32_t)(first - first_token * a.bundles) + (threadIdx.x >> a.lane_bits), skip = at_bundle / (uint32_t)a.bundles;
    const int64_t token = first_token + skip;
    const int head = (int)(at_bundle - skip * a.bundles) * BUNDLE;
    if (token >= a.tokens) continue;
    const int64_t slot = a.slots[token];
    const bool there = slot >= 0 && slot < a.slots_held && mine;
    uint32_t key[BUNDLE], value[BUNDLE], key_byte[BUNDLE], value_byte[BUNDLE];
    const KvToken from = kv_token(a.pool, there ? slot >> a.pool.page_bits : 0, head, there ? (int)(slot & ((1 << a.pool.page_bits) - 1)) : 0);
    const uint8_t* const at_m = from.values + ((lane & 1) * 8 + (lane & 2) * 2) * 4 * n + (n == 4 ? (lane >> 2) * 16 : lane >> 2);
    const int64_t piece = kv_piece_bytes(int64_t{1} << a.pool.page_bits, a.pool.dim);
#pragma unroll
    for (int i = 0; i < BUNDLE; ++i) {
      key[i] = value[i] = key_byte[i] = value_byte[i] = 0;
      if (there && head + i < a.pool.heads) {
        if (a.k) {
          key[i] = reinterpret_cast<const uint32_t*>(from.keys + i * piece)[lane];
          key_byte[i] = from.key_bytes[i * piece + (lane >> 2)];
        }
        if (a.v) {
          if (n == 4) {
            value[i] = *reinterpret_cast<const uint32_t*>(at_m + i * piece);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) value[i] |= (uint32_t)at_m[i * piece + e * 4 * n] << (8 * e);
          }
          value_byte[i] = from.value_bytes[i * piece + (lane >> 2)];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < BUNDLE; ++i) {
      if (head + i >= a.pool.heads) break;
      if (a.k && mine) put8<(BUNDLE > 1)>(a.k + token * a.k_token + (head + i) * a.k_head + lane * 8, decode8<BF>(key[i], key_byte[i]));
      if (a.v) {
        const uint32_t word = unpair_values(n == 4 ? turn_bytes(value[i], lane) : value[i], lane & 2);
        if (mine) put8<(BUNDLE > 1)>(a.v + token * a.v_token + (head + i) * a.v_head + lane * 8, decode8<BF>(word, value_byte[i]));
      }
    }
  }
}

struct TableArgs {
  int64_t first, items;
  int32_t half;
  double base, factor, trained, low, high, amplitude;
  float* table;
};
__global__ __launch_bounds__(kBlock) void table_kernel(const TableArgs a) {
  for (int64_t item = (int64_t)blockIdx.x * kBlock + threadIdx.x; item < a.items; item += (int64_t)gridDim.x * kBlock) {
    const int64_t row = item / a.half;
    const int i = (int)(item - row * a.half);
    double f = pow(a.base, -(double)i / (double)a.half);
    if (a.factor != 1.0) {
      double keep = 0.0;
      if (a.high > a.low) keep = fmin(fmax((a.trained * f / 6.283185307179586476925 - a.low) / (a.high - a.low), 0.0), 1.0);
      f = f * keep + f / a.factor * (1.0 - keep);
    }
    const double angle = (double)(a.first + row) * f;
    a.table[row * 2 * a.half + i] = (float)(cos(angle) * a.amplitude);
    a.table[row * 2 * a.half + a.half + i] = (float)(sin(angle) * a.amplitude);
  }
}

// ---- arguments ---------------------------------------------------------------

bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int check_dim(int64_t dim) { return dim < 1 ? MACKO_E_INVALID_ARG : dim % 32 != 0 || dim > 256 ? MACKO_E_UNSUPPORTED : MACKO_OK; }

// A pool's geometry; `data`: its memory is needed too.
int pool_of(const macko_kv_cache_t* c, bool data, KvPool* p) {
  if (!c || c->pages < 0 || c->page_size < 1 || c->kv_heads < 1) return MACKO_E_INVALID_ARG;
  if (int st = check_dim(c->head_dim)) return st;
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0) return MACKO_E_UNSUPPORTED;
  if (c->kv_heads > 65536 || c->pages > INT32_MAX / c->page_size) return MACKO_E_UNSUPPORTED;
  if (data && c->pages > 0 && (!c->data_dev || !aligned_to(c->data_dev, 16))) return MACKO_E_INVALID_ARG;
  int bits = 0;
  while ((1 << bits) < c->page_size) ++bits;
  *p = KvPool{static_cast<uint8_t*>(c->data_dev), c->pages, c->kv_heads, c->head_dim, bits};
  return MACKO_OK;
}

// 16-bit heads of a call: there, on 2 bytes, with strides that stay far from 64 bits.
constexpr int64_t kMostStride = int64_t{1} << 31;        // times at most 2^31 tokens
bool heads_fine(const void* p, int64_t token, int64_t head) {
  return p && aligned_to(p, 2) && token >= 0 && head >= 0 && token <= kMostStride && head <= kMostStride;
}

int check_rotation(const macko_rotation_t& r, int dim, int64_t tokens) {
  if (r.rot < 0 || r.rot > dim || r.table_rows < 0) return MACKO_E_INVALID_ARG;
  if (r.rot % 16 != 0) return MACKO_E_UNSUPPORTED;
  if (r.rot > 0 && tokens > 0 && (!r.positions_dev || !aligned_to(r.positions_dev, 4) || (r.table_rows > 0 && !r.table_dev) || !aligned_to(r.table_dev, 16))) return MACKO_E_INVALID_ARG;
  return MACKO_OK;
}

int lane_bits_of(int dim) {
  int bits = 2;
  while ((8 << bits) < dim) ++bits;
  return bits;
}

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MACKO_OK : hip_fail(e);
}

// Heads that a group of lanes takes together: 4 where that leaves enough groups to fill the device (32 heads of 128 channels, turned: 512 tokens 5.0 us in
// fours and 4.8 one by one, 1024 tokens 5.2 and 6.9, 16384 tokens 50 and 69).
constexpr int kBundle = 4;
bool bundled(int64_t items, int lane_bits) { return items >> (8 - lane_bits) >= (int64_t)device_cu_count() * 8; }

int launch_turn(TurnArgs& a, int type, hipStream_t stream) {
  a.lane_bits = lane_bits_of(a.dim);
  const int64_t groups = kBlock >> a.lane_bits;
  const int all = a.part[0].heads + a.part[1].heads + a.part[2].heads, bundle = bundled(a.tokens * all, a.lane_bits) ? kBundle : 1;
  for (Heads& h : a.part) {
    h.bundles = std::max(1, (h.heads + bundle - 1) / bundle);
    h.blocks = h.heads ? (a.tokens * h.bundles + groups - 1) / groups : 0;
    a.blocks += h.blocks;
  }
  const dim3 grid((unsigned)std::min(a.blocks, kMostBlocks)), block(kBlock);
  if (type == MACKO_BF16) {
    if (bundle > 1) hipLaunchKernelGGL((turn_kernel<true, kBundle>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((turn_kernel<true, 1>), grid, block, 0, stream, a);
  } else {
    if (bundle > 1) hipLaunchKernelGGL((turn_kernel<false, kBundle>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((turn_kernel<false, 1>), grid, block, 0, stream, a);
  }
  return launched();
}

void set_rotation(TurnArgs& a, const macko_rotation_t& r) {
  a.positions = r.positions_dev;
  a.table = r.table_dev;
  a.table_rows = r.table_rows;
  a.rot = r.rot;
  a.interleaved = r.interleaved != 0;
  a.eps = r.eps;
}

// `pointers`: they are needed too
int attention_of(const macko_kv_cache_t* cache, const macko_kv_attention_args_t* g, bool pointers, KvAttention* a) {
  if (!g) return MACKO_E_INVALID_ARG;
  KvPool pool;
  if (int st = pool_of(cache, pointers, &pool)) return st;
  if (g->tokens < 0 || g->heads < 1 || g->batch < 0 || g->most_queries < 1 || g->window < 0 || g->longest < 0 || g->table_width < 0 || g->table_stride < 0 ||
      (g->type != MACKO_FP16 && g->type != MACKO_BF16) || g->heads % pool.heads != 0 || !std::isfinite(g->scale))
    return MACKO_E_INVALID_ARG;
  if (!g->start_dev && pointers && g->tokens != g->batch) return MACKO_E_INVALID_ARG;
  if (g->tokens > INT32_MAX || g->heads > 65536 || g->longest > INT32_MAX) return MACKO_E_UNSUPPORTED;
  if (pointers && g->tokens > 0 && g->batch > 0) {
    if (!heads_fine(g->q_dev, g->q_token, g->q_head) || !heads_fine(g->out_dev, g->out_token, g->out_head) || !g->lengths_dev || !aligned_to(g->lengths_dev, 4) ||
        (g->table_width > 0 && !g->tables_dev) || !aligned_to(g->tables_dev, 4) || !aligned_to(g->start_dev, 4) || !aligned_to(g->sums_dev, 4))
      return MACKO_E_INVALID_ARG;
  }
  // A sequence has 2^30 tokens at most: a window as long is none.  A longer one, taken off a place before the first token, would not fit 32 bits.
  const int32_t window = g->window >= int32_t{1} << 30 ? 0 : g->window;
  *a = KvAttention{pool, static_cast<const uint8_t*>(g->q_dev), static_cast<uint8_t*>(g->out_dev), g->sums_dev, g->q_token, g->q_head, g->out_token, g->out_head,
                   g->tables_dev, g->table_stride, g->lengths_dev, g->start_dev, g->table_width, g->batch, g->heads, g->heads / pool.heads, window, g->scale,
                   (int32_t)std::max<int64_t>(1, std::min<int64_t>(g->most_queries, g->tokens)), g->tokens, g->longest, g->type};
  return kv_attention_fits(*a) ? MACKO_OK : MACKO_E_UNSUPPORTED;
}

}  // namespace
}  // namespace macko

extern "C" {

using namespace macko;

int64_t macko_kv_cache_bytes(const macko_kv_cache_t* cache) {
  KvPool p;
  if (int st = pool_of(cache, false, &p)) return st;
  return p.pages * p.heads * kv_piece_bytes(cache->page_size, p.dim);
}

int macko_rope_table(int64_t first, int64_t count, int rot, double base, double factor, double trained, double low, double high, double amplitude,
                     float* table_dev, void* stream) {
  if (first < 0 || count < 0 || rot < 2 || rot > 256 || rot % 2 != 0 || !(base > 0.0) || !std::isfinite(base) || !(factor > 0.0) || !std::isfinite(factor) ||
      !std::isfinite(trained) || !std::isfinite(low) || !std::isfinite(high) || !std::isfinite(amplitude) || (count > 0 && (!table_dev || !aligned_to(table_dev, 4))))
    return MACKO_E_INVALID_ARG;
  if (first > INT32_MAX || count > INT32_MAX) return MACKO_E_UNSUPPORTED;
  if (count == 0) return MACKO_OK;
  const TableArgs a{first, count * (rot / 2), rot / 2, base, factor, trained, low, high, amplitude, table_dev};
  const int64_t blocks = std::min(kMostBlocks, (a.items + kBlock - 1) / kBlock);
  hipLaunchKernelGGL(table_kernel, dim3((unsigned)blocks), dim3(kBlock), 0, static_cast<hipStream_t>(stream), a);
  return launched();
}

int macko_rotate(int64_t tokens, int heads, int head_dim, int type, const void* x_dev, int64_t x_token, int64_t x_head, const macko_rotation_t* rotation,
                 const void* weight_dev, void* out_dev, int64_t out_token, int64_t out_head, void* stream) {
  if (tokens < 0 || heads < 0 || !rotation || (type != MACKO_FP16 && type != MACKO_BF16)) return MACKO_E_INVALID_ARG;
  if (int st = check_dim(head_dim)) return st;
  if (int st = check_rotation(*rotation, head_dim, heads ? tokens : 0)) return st;
  if (tokens == 0 || heads == 0) return MACKO_OK;
  if (tokens > INT32_MAX || heads > 65536) return MACKO_E_UNSUPPORTED;
  if (!heads_fine(x_dev, x_token, x_head) || !heads_fine(out_dev, out_token, out_head) || !aligned_to(weight_dev, 2)) return MACKO_E_INVALID_ARG;
  TurnArgs a{};
  a.part[0] = Heads{static_cast<const uint16_t*>(x_dev), x_token, x_head, static_cast<const uint16_t*>(weight_dev), heads, 0, 0};
  a.out = static_cast<uint16_t*>(out_dev);
  a.out_token = out_token;
  a.out_head = out_head;
  a.tokens = tokens;
  a.dim = head_dim;
  set_rotation(a, *rotation);
  return launch_turn(a, type, static_cast<hipStream_t>(stream));
}

int macko_kv_append(const macko_kv_cache_t* cache, const macko_kv_append_args_t* g, void* stream) {
  if (!g || g->tokens < 0 || g->heads < 0 || (g->type != MACKO_FP16 && g->type != MACKO_BF16)) return MACKO_E_INVALID_ARG;
  KvPool pool;
  if (int st = pool_of(cache, true, &pool)) return st;
  if (int st = check_rotation(g->rotation, pool.dim, g->tokens)) return st;
  if (g->tokens == 0) return MACKO_OK;
  if (g->tokens > INT32_MAX || g->heads > 65536) return MACKO_E_UNSUPPORTED;
  if (!heads_fine(g->k_dev, g->k_token, g->k_head) || !heads_fine(g->v_dev, g->v_token, g->v_head) || !g->slots_dev || !aligned_to(g->slots_dev, 4) ||
      !aligned_to(g->q_weight_dev, 2) || !aligned_to(g->k_weight_dev, 2))
    return MACKO_E_INVALID_ARG;
  if (g->heads > 0 && (!heads_fine(g->q_dev, g->q_token, g->q_head) || !heads_fine(g->q_out_dev, g->q_out_token, g->q_out_head))) return MACKO_E_INVALID_ARG;
  TurnArgs a{};
  a.part[0] = Heads{static_cast<const uint16_t*>(g->q_dev), g->q_token, g->q_head, static_cast<const uint16_t*>(g->q_weight_dev), g->heads, 0, 0};
  a.part[1] = Heads{static_cast<const uint16_t*>(g->k_dev), g->k_token, g->k_head, static_cast<const uint16_t*>(g->k_weight_dev), pool.heads, 0, 0};
  a.part[2] = Heads{static_cast<const uint16_t*>(g->v_dev), g->v_token, g->v_head, nullptr, pool.heads, 0, 0};
  a.out = static_cast<uint16_t*>(g->q_out_dev);
  a.out_token = g->q_out_token;
  a.out_head = g->q_out_head;
  a.slots = g->slots_dev;
  a.pool = pool;
  a.slots_held = pool.pages << pool.page_bits;
  a.tokens = g->tokens;
  a.dim = pool.dim;
  set_rotation(a, g->rotation);
  return launch_turn(a, g->type, static_cast<hipStream_t>(stream));
}

int macko_kv_read(const macko_kv_cache_t* cache, int64_t tokens, const int32_t* slots_dev, int type, void* k_out_dev, int64_t k_token, int64_t k_head,
                  void* v_out_dev, int64_t v_token, int64_t v_head, void* stream) {
  if (tokens < 0 || (type != MACKO_FP16 && type != MACKO_BF16)) return MACKO_E_INVALID_ARG;
  KvPool pool;
  if (int st = pool_of(cache, true, &pool)) return st;
  if (tokens == 0 || (!k_out_dev && !v_out_dev)) return MACKO_OK;
  if (tokens > INT32_MAX) return MACKO_E_UNSUPPORTED;
  if (!slots_dev || !aligned_to(slots_dev, 4) || (k_out_dev && !heads_fine(k_out_dev, k_token, k_head)) || (v_out_dev && !heads_fine(v_out_dev, v_token, v_head)))
    return MACKO_E_INVALID_ARG;
  const int bits = lane_bits_of(pool.dim), groups = kBlock >> bits, bundle = bundled(tokens * pool.heads, bits) ? kBundle : 1, bundles = (pool.heads + bundle - 1) / bundle;
  const ReadArgs a{pool, slots_dev, tokens, pool.pages << pool.page_bits, (tokens * bundles + groups - 1) / groups, static_cast<uint16_t*>(k_out_dev), k_token, k_head,
                   static_cast<uint16_t*>(v_out_dev), v_token, v_head, bits, bundles};
  const dim3 grid((unsigned)std::min(a.blocks, kMostBlocks)), block(kBlock);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == MACKO_BF16) {
    if (bundle > 1) hipLaunchKernelGGL((read_kernel<true, kBundle>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_kernel<true, 1>), grid, block, 0, s, a);
  } else {
    if (bundle > 1) hipLaunchKernelGGL((read_kernel<false, kBundle>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_kernel<false, 1>), grid, block, 0, s, a);
  }
  return launched();
}

int64_t macko_kv_attention_workspace(const macko_kv_cache_t* cache, const macko_kv_attention_args_t* args) {
  KvAttention a;
  if (int st = attention_of(cache, args, false, &a)) return st;
  return 4 * kv_attention_workspace(a);
}

int macko_kv_attention(const macko_kv_cache_t* cache, const macko_kv_attention_args_t* args, void* workspace_dev, int64_t workspace_bytes, void* stream) {
  KvAttention a;
  if (int st = attention_of(cache, args, true, &a)) return st;
  if (a.tokens == 0 || a.batch == 0) return MACKO_OK;
  const int64_t need = 4 * kv_attention_workspace(a);
  if (need > 0 && (!workspace_dev || !aligned_to(workspace_dev, 16) || workspace_bytes < need)) return MACKO_E_INVALID_ARG;
  return launch_kv_attention(a, static_cast<float*>(workspace_dev), static_cast<hipStream_t>(stream));
}

}  // extern "C"
