// Heads between the products of a decoder layer: norm and position of queries and keys, the 4-bit key/value cache that new tokens go into
// (macko_kv_append) and its values back (macko_kv_read); the C entry points of these and of the attention over the cache.
//
// All of it moves bytes: a value takes 2 bytes in, 2 or 17/32 out and some ten operations.  A head of a token is the unit of work, a
// group of 4 to 32 lanes with 8 channels each takes it in one 16-byte load a lane; what a head needs of other lanes (the sum of a norm, the
// other half of a pair, a group's largest magnitude) goes through lane shuffles, so that nothing is read twice and in-place calls are safe.
#include <cmath>

#include "macko_kv.h"

namespace macko {
namespace {

constexpr int kBlock = 256;
constexpr int64_t kMostBlocks = (int64_t{1} << 24) - 1;  // a launch has fewer than 2^32 threads

struct Heads {
  const uint16_t* x;
  int64_t token, head;       // strides in elements
};
struct TurnArgs {
  Heads q, k, v;
  uint16_t* out;
  int64_t out_token, out_head;
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  const int32_t* positions;
  const int32_t* slots;
  const float* table;
  int64_t table_rows;
  KvPool pool;               // heads = 0: queries alone
  int64_t items, slots_held; // heads of all tokens; slots of the pool
  int32_t heads, all_heads;  // query heads; with key and value heads
  int32_t dim, rot, interleaved;
  int32_t lane_bits;         // log2 of the lanes of a head
  int32_t rounds;            // heads that a group of lanes takes one after the other
  float eps;
};

__device__ inline float group_sum(float x, int lanes) {
  for (int m = 1; m < lanes; m <<= 1) x += __shfl_xor(x, m);
  return x;
}

// The 4-bit codes of 8 channels of a group that 4 neighbouring lanes hold, 2 to a byte, and the group's byte.
__device__ inline uint32_t encode8(const float* y, uint32_t* byte) {
  float most = 0.f;
  bool finite = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    most = fmaxf(most, fabsf(y[i]));
    finite = finite && fabsf(y[i]) < INFINITY;           // false for a NaN
  }
  uint32_t bits = finite ? __builtin_bit_cast(uint32_t, most) : 0x7F800000u;
  bits = max(bits, (uint32_t)__shfl_xor((int)bits, 1));  // magnitudes are ordered as their bits are
  bits = max(bits, (uint32_t)__shfl_xor((int)bits, 2));
  // the exponent of most / 7, rounded up: 7 = 1.75 * 2^2, and a mantissa above 1.75 carries
  const uint32_t e = (bits + 0x1FFFFFu) >> 23;
  const uint32_t b = bits >= 0x7F800000u ? 255u : e > 2u ? e - 2u : 0u;
  *byte = b;
  const float unit = __builtin_bit_cast(float, b << 23);
  uint32_t word = 0;
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[0], y[1], unit, 0);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[2], y[3], unit, 1);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[4], y[5], unit, 2);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[6], y[7], unit, 3);
  return word;
}

template <bool BF>
__global__ __launch_bounds__(kBlock) void turn_kernel(const TurnArgs a) {
#pragma clang fp contract(off)     // products are rounded before they are added: keys near the edge of two codes take the same one everywhere
  const int lanes = 1 << a.lane_bits, lane = threadIdx.x & (lanes - 1), groups = kBlock >> a.lane_bits;
  const int64_t first = (int64_t)blockIdx.x * (groups * a.rounds) + (threadIdx.x >> a.lane_bits);
  const bool mine = lane * 8 < a.dim;
  for (int round = 0; round < a.rounds; ++round) {
    const int64_t item = first + (int64_t)round * groups;
    if (item >= a.items) return;                          // the same for all lanes of a head
    const int64_t token = item / a.all_heads;
    int head = (int)(item - token * a.all_heads);
    const int kind = head < a.heads ? 0 : head < a.heads + a.pool.heads ? 1 : 2;
    head -= kind == 0 ? 0 : kind == 1 ? a.heads : a.heads + a.pool.heads;
    const Heads src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;

    Packed8 raw = {0, 0, 0, 0};
    if (mine) raw = *reinterpret_cast<const Packed8Any*>(src.x + token * src.token + head * src.head + lane * 8);
    float y[8];
    unpack8<BF>(raw, y);
    bool placed = true;
    if (kind < 2) {
      // the lane that holds the other channels of this one's pairs
      const int half = a.rot >> 4;                        // lanes of half a turned part
      const bool turned = lane < 2 * half;
      float z[8];
      if (!a.interleaved) {
        const int other = !turned ? lane : lane < half ? lane + half : lane - half;
        Packed8 far;
#pragma unroll
        for (int i = 0; i < 4; ++i) far[i] = (uint32_t)__shfl((int)raw[i], other, lanes);
        unpack8<BF>(far, z);
      }
      const uint16_t* weight = kind == 0 ? a.q_weight : a.k_weight;
      if (weight) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += y[i] * y[i];
        const float r = 1.f / sqrtf(group_sum(sum, lanes) / (float)a.dim + a.eps);
        if (mine) {
          float w[8];
          unpack8<BF>(*reinterpret_cast<const Packed8Any*>(weight + lane * 8), w);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = y[i] * r * w[i];
          if (!a.interleaved && turned) {
            unpack8<BF>(*reinterpret_cast<const Packed8Any*>(weight + (lane < half ? lane + half : lane - half) * 8), w);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = z[i] * r * w[i];
          }
        }
      }
      if (a.rot > 0) {
        const int64_t at = a.positions[token];
        placed = at >= 0 && at < a.table_rows;
        if (placed && turned) {
          const float* row = a.table + at * a.rot;
          if (a.interleaved) {
            const float4 c = *reinterpret_cast<const float4*>(row + lane * 4), s = *reinterpret_cast<const float4*>(row + a.rot / 2 + lane * 4);
            const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float u = y[2 * i], w = y[2 * i + 1];
              y[2 * i] = u * cs[i] - w * sn[i];
              y[2 * i + 1] = u * sn[i] + w * cs[i];
            }
          } else {
            const int i0 = (lane < half ? lane : lane - half) * 8;
            const float sign = lane < half ? -1.f : 1.f;
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
              const float4 c = *reinterpret_cast<const float4*>(row + i0 + i), s = *reinterpret_cast<const float4*>(row + a.rot / 2 + i0 + i);
              const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
              for (int t = 0; t < 4; ++t) y[i + t] = y[i + t] * cs[t] + sign * (z[i + t] * sn[t]);
            }
          }
        }
      }
    }
    if (kind == 0) {
      if (!placed) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = NAN;
      }
      if (mine) *reinterpret_cast<Packed8Any*>(a.out + token * a.out_token + head * a.out_head + lane * 8) = pack8<BF>(y);
      continue;
    }
    if (kind == 2 && a.rot > 0) {
      const int64_t at = a.positions[token];
      placed = at >= 0 && at < a.table_rows;
    }
    const int64_t slot = a.slots[token];
    uint32_t byte;
    const uint32_t word = encode8(y, &byte);
    if (!placed || slot < 0 || slot >= a.slots_held) continue;
    const int n = a.dim / 32;
    const KvToken to = kv_token(a.pool, slot >> a.pool.page_bits, head, (int)(slot & ((1 << a.pool.page_bits) - 1)));
    if (kind == 1) {
      if (mine) {
        reinterpret_cast<uint32_t*>(to.keys)[lane] = word;
        if ((lane & 3) == 0) to.key_bytes[lane >> 2] = (uint8_t)byte;
      }
    } else {
      // lanes 4g + 2u + v hold channels 32g + 16u + 8v + e: a byte takes the same e from u = 0 and u = 1
      const uint32_t far = (uint32_t)__shfl_xor((int)word, 2);
      const bool upper = lane & 2;
      const uint32_t low = upper ? far >> 16 : word, high = upper ? word >> 16 : far;
      if (mine) {
        uint8_t* at = to.values + ((lane & 1) * 8 + (upper ? 4 : 0)) * 4 * n + (lane >> 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) at[e * 4 * n] = (uint8_t)((low >> (4 * e) & 15u) | (high >> (4 * e) & 15u) << 4);
        if ((lane & 3) == 0) to.value_bytes[lane >> 2] = (uint8_t)byte;
      }
    }
  }
}

struct ReadArgs {
  KvPool pool;
  const int32_t* slots;
  int64_t items, slots_held;
  uint16_t* k;
  int64_t k_token, k_head;
  uint16_t* v;
  int64_t v_token, v_head;
  int32_t lane_bits;
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

template <bool BF>
__global__ __launch_bounds__(kBlock) void read_kernel(const ReadArgs a) {
  const int lanes = 1 << a.lane_bits, lane = threadIdx.x & (lanes - 1), groups = kBlock >> a.lane_bits;
  if (lane * 8 >= a.pool.dim) return;
  for (int64_t item = (int64_t)blockIdx.x * groups + (threadIdx.x >> a.lane_bits); item < a.items; item += (int64_t)gridDim.x * groups) {
    const int64_t token = item / a.pool.heads;
    const int head = (int)(item - token * a.pool.heads), n = a.pool.dim / 32;
    const int64_t slot = a.slots[token];
    Packed8 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (slot >= 0 && slot < a.slots_held) {
      const KvToken from = kv_token(a.pool, slot >> a.pool.page_bits, head, (int)(slot & ((1 << a.pool.page_bits) - 1)));
      if (a.k) k = decode8<BF>(reinterpret_cast<const uint32_t*>(from.keys)[lane], from.key_bytes[lane >> 2]);
      if (a.v) {
        const uint8_t* at = from.values + (lane & 1) * 8 * 4 * n + (lane >> 2);
        uint32_t word = 0;
  #pragma unroll
        for (int e = 0; e < 8; ++e) word |= (uint32_t)(at[e * 4 * n] >> (lane & 2 ? 4 : 0) & 15) << (4 * e);
        v = decode8<BF>(word, from.value_bytes[lane >> 2]);
      }
    }
    if (a.k) *reinterpret_cast<Packed8Any*>(a.k + token * a.k_token + head * a.k_head + lane * 8) = k;
    if (a.v) *reinterpret_cast<Packed8Any*>(a.v + token * a.v_token + head * a.v_head + lane * 8) = v;
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

int launch_turn(TurnArgs& a, int64_t tokens, int type, hipStream_t stream) {
  a.lane_bits = lane_bits_of(a.dim);
  a.items = tokens * a.all_heads;
  const int64_t groups = kBlock >> a.lane_bits, target = (int64_t)device_cu_count() * 16;
  int64_t rounds = std::min<int64_t>(4, std::max<int64_t>(1, a.items / (groups * target)));
  rounds = std::max(rounds, (a.items + groups * kMostBlocks - 1) / (groups * kMostBlocks));
  if (rounds > INT32_MAX / kBlock) return MACKO_E_UNSUPPORTED;
  a.rounds = (int32_t)rounds;
  const int64_t blocks = (a.items + groups * rounds - 1) / (groups * rounds);
  if (type == MACKO_BF16) hipLaunchKernelGGL(turn_kernel<true>, dim3((unsigned)blocks), dim3(kBlock), 0, stream, a);
  else hipLaunchKernelGGL(turn_kernel<false>, dim3((unsigned)blocks), dim3(kBlock), 0, stream, a);
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
  *a = KvAttention{pool, static_cast<const uint8_t*>(g->q_dev), static_cast<uint8_t*>(g->out_dev), g->sums_dev, g->q_token, g->q_head, g->out_token, g->out_head,
                   g->tables_dev, g->table_stride, g->lengths_dev, g->start_dev, g->table_width, g->batch, g->heads, g->heads / pool.heads, g->window, g->scale,
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
  a.q = {static_cast<const uint16_t*>(x_dev), x_token, x_head};
  a.out = static_cast<uint16_t*>(out_dev);
  a.out_token = out_token;
  a.out_head = out_head;
  a.q_weight = static_cast<const uint16_t*>(weight_dev);
  a.heads = a.all_heads = heads;
  a.dim = head_dim;
  set_rotation(a, *rotation);
  return launch_turn(a, tokens, type, static_cast<hipStream_t>(stream));
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
  a.q = {static_cast<const uint16_t*>(g->q_dev), g->q_token, g->q_head};
  a.k = {static_cast<const uint16_t*>(g->k_dev), g->k_token, g->k_head};
  a.v = {static_cast<const uint16_t*>(g->v_dev), g->v_token, g->v_head};
  a.out = static_cast<uint16_t*>(g->q_out_dev);
  a.out_token = g->q_out_token;
  a.out_head = g->q_out_head;
  a.q_weight = static_cast<const uint16_t*>(g->q_weight_dev);
  a.k_weight = static_cast<const uint16_t*>(g->k_weight_dev);
  a.slots = g->slots_dev;
  a.pool = pool;
  a.slots_held = pool.pages << pool.page_bits;
  a.heads = g->heads;
  a.all_heads = g->heads + 2 * pool.heads;
  a.dim = pool.dim;
  set_rotation(a, g->rotation);
  return launch_turn(a, g->tokens, g->type, static_cast<hipStream_t>(stream));
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
  const int bits = lane_bits_of(pool.dim), groups = kBlock >> bits;
  const ReadArgs a{pool, slots_dev, tokens * pool.heads, pool.pages << pool.page_bits, static_cast<uint16_t*>(k_out_dev), k_token, k_head,
                   static_cast<uint16_t*>(v_out_dev), v_token, v_head, bits};
  const int64_t blocks = std::min(kMostBlocks, (a.items + groups - 1) / groups);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == MACKO_BF16) hipLaunchKernelGGL(read_kernel<true>, dim3((unsigned)blocks), dim3(kBlock), 0, s, a);
  else hipLaunchKernelGGL(read_kernel<false>, dim3((unsigned)blocks), dim3(kBlock), 0, s, a);
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
