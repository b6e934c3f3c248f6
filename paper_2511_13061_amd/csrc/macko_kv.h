// Layout of the 4-bit key/value cache, shared by the kernels that fill it and those that read it.
//
// A page holds page_size tokens (a power of two, at least 16) of every key/value head; what one head has of it is one piece of
// page_size * (D + D / 16) bytes (D channels, n = D / 32 groups of 32 channels that share a byte b, a factor 2^(b - 127)):
//   key codes    [page_size][D / 2]         channel 2i in the low half of byte i: a lane of the matrix instruction takes 16 bytes as they lie
//   value codes  [page_size / 4][16][4][n]  [token / 4][m][token % 4][g]: channels 32g + m and 32g + 16 + m in the halves of one byte, so
//                                           that a lane finds 4 tokens of "its" channels together and two channels share a conversion
//   key bytes    [page_size][n]
//   value bytes  [page_size][n]
// No byte belongs to two tokens: tokens are written without reading what is there, in any order and from any workgroup.
#pragma once

#include "macko_internal.h"

namespace macko {

constexpr uint32_t kMostByte = 252;      // that a group of numbers is stored with: 6 * 2^125 is a number in bf16 and in 32 bits, 4 * 2^126 is not

struct KvPool {
  uint8_t* data;
  int64_t pages;
  int32_t heads;             // key/value heads
  int32_t dim;
  int32_t page_bits;         // log2(page_size)
};

constexpr int64_t kv_piece_bytes(int64_t page_size, int64_t dim) { return page_size * (dim + dim / 16); }

// Pointers into the piece of one head in one page, for the token at `at` in it.
struct KvToken {
  uint8_t* keys;             // D / 2 bytes
  uint8_t* values;           // byte (m, g) at m * 4n + g
  uint8_t* key_bytes;        // n
  uint8_t* value_bytes;      // n
};
__host__ __device__ inline KvToken kv_token(const KvPool& p, int64_t page, int head, int at) {
  const int64_t size = int64_t{1} << p.page_bits;
  const int n = p.dim / 32;
  uint8_t* piece = p.data + (page * p.heads + head) * kv_piece_bytes(size, p.dim);
  uint8_t* bytes = piece + size * p.dim;
  return {piece + (int64_t)at * (p.dim / 2), piece + size * (p.dim / 2) + ((at >> 2) * 64 + (at & 3)) * n, bytes + (int64_t)at * n,
          bytes + (size + at) * n};
}

// 8 values of 16 bits, as they are loaded and stored
typedef uint32_t Packed8 __attribute__((ext_vector_type(4)));
typedef uint32_t Packed8Any __attribute__((ext_vector_type(4), aligned(2)));

template <bool BF>
__device__ inline float to_float(uint32_t bits16) {
  if (BF) return __builtin_bit_cast(float, bits16 << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
}
template <bool BF>
__device__ inline void unpack8(Packed8 p, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = to_float<BF>(p[i] & 0xFFFFu);
    x[2 * i + 1] = to_float<BF>(p[i] >> 16);
  }
}
template <bool BF>
__device__ inline uint32_t pack2(float x, float y) {   // round to nearest even
  if (BF) {
    typedef __bf16 B2 __attribute__((ext_vector_type(2)));
    const B2 p = {(__bf16)x, (__bf16)y};
    return __builtin_bit_cast(uint32_t, p);
  }
  typedef _Float16 H2 __attribute__((ext_vector_type(2)));
  const H2 p = {(_Float16)x, (_Float16)y};
  return __builtin_bit_cast(uint32_t, p);
}
template <bool BF>
__device__ inline Packed8 pack8(const float* x) {
  return {pack2<BF>(x[0], x[1]), pack2<BF>(x[2], x[3]), pack2<BF>(x[4], x[5]), pack2<BF>(x[6], x[7])};
}

struct KvAttention {
  KvPool pool;
  const uint8_t* q;
  uint8_t* out;
  float* sums;               // may be null
  int64_t q_token, q_head, out_token, out_head;      // strides in elements
  const int32_t* tables;     // [batch][table_width], rows table_stride apart
  int64_t table_stride;
  const int32_t* lengths;
  const int32_t* start;      // null: one query token a sequence
  int32_t table_width, batch, heads, shared, window;
  float scale;
  int32_t most_queries;
  int64_t tokens, longest;
  int32_t type;
};
bool kv_attention_fits(const KvAttention& a);        // in a launch
// The arguments of a call over a pool, checked; `pointers`: they are needed too.
int kv_attention_of(const KvPool& pool, const macko_kv_attention_args_t* g, bool pointers, KvAttention* a);

// Checks of arguments, in macko_kv.hip
bool aligned_to(const void* p, uintptr_t bytes);
int check_head_dim(int64_t dim);
bool heads_fine(const void* p, int64_t token, int64_t head);       // 16-bit heads of a call: there, on 2 bytes, with strides that stay far from 64 bits
int check_rotation(const macko_rotation_t& r, int dim, int64_t tokens);
// floats of workspace that the launch needs
int64_t kv_attention_workspace(const KvAttention& a);
int launch_kv_attention(const KvAttention& a, float* workspace, hipStream_t stream);

}  // namespace macko
