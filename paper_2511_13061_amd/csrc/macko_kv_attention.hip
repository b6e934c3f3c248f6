// Attention over the paged 4-bit key/value cache (layout: macko_kv.h).
//
// Rows are the queries of one sequence for one key/value head, query by query and in it head by head, 16 to a tile.  A wavefront takes
// 32 tokens at a time:
//   scores   S^T = K Q^T by mfma_scale 16x16x128: keys go to the matrix cores as they lie in memory, 4-bit codes and the group's byte as the
//            block scale, without an instruction of the vector units.  Queries are 8-bit parts, each what the ones before left over (fp16: 3,
//            bf16: 2), with a scale of their own per 32 channels: together they hold every bit of a query down to 2^-18 (2^-13) of its group's largest.
//   softmax  running maximum and sum in 32 bits.  Column r of S^T is row r, so a lane holds 8 scores of one row; the running maximum moves
//            only when a score is more than 2^8 above it, and only then do lanes talk to each other.
//   values   O^T += V^T P^T by mfma 16x16x32 bf16: codes are exact in bf16 with any scale; weights go in as two bf16 parts (16 bits).
//            The lanes of S^T that hold a token's weights are those that P^T needs: nothing moves between lanes.
// The four wavefronts of a workgroup take turns along the tokens and join their sums in LDS; long sequences are split over workgroups
// too, whose unnormalised sums a second kernel joins.
#include "macko_kv.h"

namespace macko {
namespace {

typedef int V8i __attribute__((ext_vector_type(8)));
typedef int V4i __attribute__((ext_vector_type(4)));
typedef float V4f __attribute__((ext_vector_type(4)));
typedef __bf16 B2 __attribute__((ext_vector_type(2)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4, kTile = 32;
constexpr int kMostTokens = 1 << 30;                  // of a sequence: sums of a length and a launch's steps stay in 31 bits
constexpr float kLift = 8.f;       // how far, in powers of two, a score may pass the running maximum before that moves

struct Grid {
  int32_t row_blocks, splits;      // of a sequence's rows and of its tokens, at most
  int64_t chunk;                   // tokens of a split, at least; a multiple of kWaves * kTile
  float* parts;                    // [tokens * heads][splits][D], then [tokens * heads][splits][2]: maximum and sum
};

struct Sequence {
  int length, first, queries, rows;
};
__device__ inline Sequence sequence_of(const KvAttention& a, int b) {
  Sequence s;
  s.length = min(max(0, a.lengths[b]), kMostTokens);
  s.first = a.start ? min(max(a.start[b], 0), (int)a.tokens) : b;
  s.queries = a.start ? min(max(a.start[b + 1], s.first), (int)a.tokens) - s.first : 1;
  s.rows = s.queries * a.shared;
  return s;
}

// The tokens that the rows first_row .. of a block see, and how they are split.
struct Span {
  int lo, hi, chunk, used;         // lo: a multiple of 16
  int all_lo, all_hi;              // every row of the block sees [all_lo, all_hi)
};
__device__ inline Span span_of(const KvAttention& a, const Grid& g, const Sequence& s, int first_row, int rows) {
  Span p;
  const int qa = first_row / a.shared, qb = min(first_row + rows - 1, s.rows - 1) / a.shared, offset = s.length - s.queries;
  p.hi = min(max(offset + qb + 1, 0), s.length);
  p.all_hi = min(max(offset + qa + 1, 0), s.length);
  const int lo = a.window ? max(offset + qa - a.window + 1, 0) : 0;
  p.all_lo = a.window ? max(offset + qb - a.window + 1, 0) : 0;
  p.lo = min(lo, p.hi) & ~15;
  const int range = max(p.hi - p.lo, 0), unit = kWaves * kTile;
  p.chunk = max((int)g.chunk, (range + g.splits * unit - 1) / (g.splits * unit) * unit);
  p.used = max(1, (range + p.chunk - 1) / p.chunk);
  return p;
}

// What a wavefront holds of 32 tokens: two blocks of 16.
template <int NG>
struct Tile {
  static constexpr int NK = (NG + 3) / 4;
  V4i key[2][NK];
  int key_byte[2][NK];
  uint32_t value[2][NG], value_byte[2][NG];      // [token of 4][g] bytes
};

template <int BYTE>
__device__ inline B2 decode_pair(uint32_t word, uint32_t bytes, int at) {
  // the conversion looks at the exponent field of its scale alone
  const uint32_t unit = at == 0 ? bytes << 23 : at == 1 ? bytes << 15 : at == 2 ? bytes << 7 : bytes >> 1;
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, __builtin_bit_cast(float, unit), BYTE);
}
__device__ inline B2 decode_at(uint32_t word, uint32_t bytes, int at) {
  switch (at) {
    case 0: return decode_pair<0>(word, bytes, 0);
    case 1: return decode_pair<1>(word, bytes, 1);
    case 2: return decode_pair<2>(word, bytes, 2);
    default: return decode_pair<3>(word, bytes, 3);
  }
}

template <int NG, bool BF, int RT>
__global__ __launch_bounds__(64 * kWaves) void attention_kernel(const KvAttention a, const Grid g) {
  constexpr int D = 32 * NG, NK = (NG + 3) / 4, NP = BF ? 2 : 3, R = 16 * RT, LD = D + 4;
  extern __shared__ __align__(16) float lds[];           // [kWaves][16][LD], then maxima and sums [kWaves][16] each
  float* const lds_max = lds + kWaves * 16 * LD;
  float* const lds_sum = lds_max + kWaves * 16;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  const uint32_t pairs = (uint32_t)a.batch * a.pool.heads, bh = blockIdx.x % pairs, rest = blockIdx.x / pairs;
  const int b = (int)(bh / a.pool.heads), head = (int)(bh % a.pool.heads), split = (int)(rest / g.row_blocks);
  const Sequence seq = sequence_of(a, b);
  const int32_t* const table = a.tables + b * a.table_stride;
  const int64_t piece = kv_piece_bytes(int64_t{1} << a.pool.page_bits, D), page_stride = piece * a.pool.heads;
  const uint8_t* const pool = a.pool.data + head * piece;
  const int page_size = 1 << a.pool.page_bits;
  const float scale = a.scale * 1.4426950408889634f;     // weights are powers of two

  for (int first_row = (int)(rest % g.row_blocks) * R; first_row < seq.rows; first_row += g.row_blocks * R) {
    const Span span = span_of(a, g, seq, first_row, R);
    if (split >= span.used) continue;
    const int begin = span.lo + split * span.chunk, end = min(span.hi, begin + span.chunk);

    // rows of this lane
    int see_lo[RT], see_hi[RT];
    V8i q[RT][NK][NP];
    int q_byte[RT][NK];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = first_row + rt * 16 + n, query = row / a.shared;
      const bool there = row < seq.rows;
      const int at = seq.length - seq.queries + query;
      see_hi[rt] = there ? min(max(at + 1, 0), seq.length) : 0;
      see_lo[rt] = a.window ? max(at - a.window + 1, 0) : 0;
      const uint16_t* src = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(seq.first + query) * a.q_token + (int64_t)(head * a.shared + row - query * a.shared) * a.q_head;
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
          const float unit = __builtin_bit_cast(float, (254u - top[u]) << 23);
#pragma unroll
          for (int i = 0; i < 16; ++i) x[u][i] *= unit;
#pragma unroll
          for (int p = 0; p < NP; ++p) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              int word = 0;
              word = __builtin_amdgcn_cvt_pk_fp8_f32(x[u][4 * w], x[u][4 * w + 1], word, false);
              word = __builtin_amdgcn_cvt_pk_fp8_f32(x[u][4 * w + 2], x[u][4 * w + 3], word, true);
              q[rt][kk][p][u * 4 + w] = word;
              x[u][4 * w] = (x[u][4 * w] - __builtin_amdgcn_cvt_f32_fp8(word, 0)) * 16.f;
              x[u][4 * w + 1] = (x[u][4 * w + 1] - __builtin_amdgcn_cvt_f32_fp8(word, 1)) * 16.f;
              x[u][4 * w + 2] = (x[u][4 * w + 2] - __builtin_amdgcn_cvt_f32_fp8(word, 2)) * 16.f;
              x[u][4 * w + 3] = (x[u][4 * w + 3] - __builtin_amdgcn_cvt_f32_fp8(word, 3)) * 16.f;
            }
          }
        }
        // lane j gives the scale of group j: groups 0 and 1 are those of lanes 0 and 2 (first half), 2 and 3 of the second
        const int from = n + 32 * (j & 1), t0 = __shfl((int)top[0], from), t1 = __shfl((int)top[1], from);
        const int t = j < 2 ? t0 : t1;
        q_byte[rt][kk] = t | (t - 4) << 8 | (t - 8) << 16;
      }
    }

    bool bad = end > begin && (a.table_width == 0 || a.pool.pages == 0);     // a page that is needed is missing
    const int last_block = (end - 1) >> 4;
    float top[RT], sum[RT];
    V4f out[RT][2 * NG];
    uint32_t spoilt[RT];                                  // groups in which a seen value is not a number

    auto page_of = [&](int block) {
      const int index = min(block, last_block) >> (a.pool.page_bits - 4);
      const int page = table[min(index, a.table_width - 1)];
      const bool fine = index < a.table_width && page >= 0 && page < a.pool.pages;
      bad = bad || !fine;
      return fine ? page : 0;
    };
    auto load = [&](Tile<NG>& t, int at) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int block = min((at >> 4) + u, last_block), in_page = (block << 4) & (page_size - 1);
        const uint8_t* const codes = pool + (int64_t)page_of(block) * page_stride;
        const uint8_t* const keys = codes + in_page * (D / 2);
        const uint8_t* const values = codes + page_size * (D / 2) + in_page * (D / 2);
        const uint8_t* const key_bytes = codes + page_size * D + in_page * NG;
        const uint8_t* const value_bytes = codes + page_size * (D + NG) + in_page * NG;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
          const int group = kk * 4 + j;
          t.key[u][kk] = V4i{0, 0, 0, 0};
          t.key_byte[u][kk] = 0;
          if (group < NG) {
            t.key[u][kk] = *reinterpret_cast<const V4i*>(keys + n * (D / 2) + group * 16);
            t.key_byte[u][kk] = key_bytes[n * NG + group];
          }
        }
        const uint32_t* const v = reinterpret_cast<const uint32_t*>(values + (j * 16 + n) * (4 * NG));
        const uint32_t* const vb = reinterpret_cast<const uint32_t*>(value_bytes + j * (4 * NG));
#pragma unroll
        for (int w = 0; w < NG; ++w) {
          t.value[u][w] = v[w];
          t.value_byte[u][w] = vb[w];
        }
      }
    };
    auto step = [&](Tile<NG>& t, int at, bool careful) {
      const bool masked = at < span.all_lo || at + kTile > span.all_hi;
      B8 p_hi[RT], p_lo[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          V4f s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < NK; ++kk) {
            const V8i key = {t.key[u][kk][0], t.key[u][kk][1], t.key[u][kk][2], t.key[u][kk][3], 0, 0, 0, 0};
            if (NP == 3) s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, q[rt][kk][NP - 1], s, 4, 0, 0, t.key_byte[u][kk], 2, q_byte[rt][kk]);
            s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, q[rt][kk][1], s, 4, 0, 0, t.key_byte[u][kk], 1, q_byte[rt][kk]);
            s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, q[rt][kk][0], s, 4, 0, 0, t.key_byte[u][kk], 0, q_byte[rt][kk]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) x[4 * u + i] = s[i] * scale;
        }
        if (masked) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int token = at + (i >> 2) * 16 + j * 4 + (i & 3);
            if (token < see_lo[rt] || token >= see_hi[rt]) x[i] = -INFINITY;
          }
        }
        const float most = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__any(most > top[rt] + kLift)) {
          float to = fmaxf(most, __shfl_xor(most, 16));
          to = fmaxf(to, __shfl_xor(to, 32));
          to = fmaxf(to, top[rt]);
          const float by = to == top[rt] ? 1.f : __builtin_amdgcn_exp2f(top[rt] - to);
          top[rt] = to;
          sum[rt] *= by;
#pragma unroll
          for (int c = 0; c < 2 * NG; ++c) out[rt][c] *= by;
        }
        const float base = top[rt] == -INFINITY ? 0.f : top[rt];       // nothing seen yet: weights of 2^-inf, not NaN
        uint32_t bits[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float w = __builtin_amdgcn_exp2f(x[i] - base);
          sum[rt] += w;
          bits[i] = __builtin_bit_cast(uint32_t, w);
        }
        // the first part is cut off, not rounded: it takes no instruction but the one that joins two of them
        V4i hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          hi[i] = (int)__builtin_amdgcn_perm(bits[2 * i + 1], bits[2 * i], 0x07060302u);
          const float r0 = __builtin_bit_cast(float, bits[2 * i]) - __builtin_bit_cast(float, bits[2 * i] & 0xFFFF0000u);
          const float r1 = __builtin_bit_cast(float, bits[2 * i + 1]) - __builtin_bit_cast(float, bits[2 * i + 1] & 0xFFFF0000u);
          const B2 r = {(__bf16)r0, (__bf16)r1};
          lo[i] = __builtin_bit_cast(int, r);
        }
        p_hi[rt] = __builtin_bit_cast(B8, hi);
        p_lo[rt] = __builtin_bit_cast(B8, lo);
      }
      if (careful || at + kTile > seq.length) {
        // Tokens behind the sequence's end may hold anything: their factor becomes the least one.  In a careful pass that of values that are
        // not numbers does too, and rows that see them are marked.
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int token = at + u * 16 + j * 4 + k;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
              const int byte = k * NG + i, shift = 8 * (byte & 3);
              uint32_t& word = t.value_byte[u][byte >> 2];
              const bool nan = (word >> shift & 255u) == 255u && token < seq.length;
              if (token >= seq.length || (careful && nan)) word &= ~(255u << shift);
              if (careful && nan) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                  if (token >= see_lo[rt] && token < see_hi[rt]) spoilt[rt] |= 1u << i;
              }
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        V4i lower, upper;                                 // channels 32i + n and 32i + 16 + n of 8 tokens
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int k = 0; k < 4; k += 2) {
            const int b0 = k * NG + i, b1 = (k + 1) * NG + i;
            const uint32_t v0 = __builtin_bit_cast(uint32_t, decode_at(t.value[u][b0 >> 2], t.value_byte[u][b0 >> 2], b0 & 3));
            const uint32_t v1 = __builtin_bit_cast(uint32_t, decode_at(t.value[u][b1 >> 2], t.value_byte[u][b1 >> 2], b1 & 3));
            lower[u * 2 + k / 2] = (int)__builtin_amdgcn_perm(v1, v0, 0x05040100u);
            upper[u * 2 + k / 2] = (int)__builtin_amdgcn_perm(v1, v0, 0x07060302u);
          }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          out[rt][2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, lower), p_lo[rt], out[rt][2 * i], 0, 0, 0);
          out[rt][2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, upper), p_lo[rt], out[rt][2 * i + 1], 0, 0, 0);
          out[rt][2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, lower), p_hi[rt], out[rt][2 * i], 0, 0, 0);
          out[rt][2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, upper), p_hi[rt], out[rt][2 * i + 1], 0, 0, 0);
        }
      }
    };

    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        top[rt] = -INFINITY;
        sum[rt] = 0.f;
        spoilt[rt] = 0;
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c) out[rt][c] = V4f{0.f, 0.f, 0.f, 0.f};
      }
      int at = begin + wave * kTile;
      if (at < end && !bad) {
        Tile<NG> one, two;
        load(one, at);
        for (;;) {
          int next = at + kWaves * kTile;
          if (next < end) load(two, next);
          step(one, at, pass > 0);
          at = next;
          if (at >= end) break;
          next = at + kWaves * kTile;
          if (next < end) load(one, next);
          step(two, at, pass > 0);
          at = next;
          if (at >= end) break;
        }
      }
      // A value that is not a number reaches every row of its tile, with weight 0 where it is not seen: then the tokens are gone through
      // again, carefully.  Nothing but such values gets here.
      bool nan = false;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) nan = nan || out[rt][c][i] != out[rt][c][i];
      if (!__any(nan)) break;
    }

#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      sum[rt] += __shfl_xor(sum[rt], 16);
      sum[rt] += __shfl_xor(sum[rt], 32);
      if (bad) sum[rt] = NAN;
      spoilt[rt] |= (uint32_t)__shfl_xor((int)spoilt[rt], 16);
      spoilt[rt] |= (uint32_t)__shfl_xor((int)spoilt[rt], 32);
      float* const mine = lds + (wave * 16 + n) * LD;
#pragma unroll
      for (int c = 0; c < 2 * NG; ++c) {
        V4f o = out[rt][c];
        if (spoilt[rt] >> (c / 2) & 1) o = V4f{NAN, NAN, NAN, NAN};
        *reinterpret_cast<V4f*>(mine + c * 16 + j * 4) = o;
      }
      if (j == 0) {
        lds_max[wave * 16 + n] = top[rt];
        lds_sum[wave * 16 + n] = sum[rt];
      }
      __syncthreads();
      for (int item = threadIdx.x; item < 4 * D; item += 64 * kWaves) {
        const int r = item / (D / 4), channel = item % (D / 4) * 4, row = first_row + rt * 16 + r;
        if (row >= seq.rows) continue;
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, lds_max[w * 16 + r]);
        V4f o = {0.f, 0.f, 0.f, 0.f};
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float m = lds_max[w * 16 + r], by = m == most ? 1.f : __builtin_amdgcn_exp2f(m - most);
          total += lds_sum[w * 16 + r] * by;
          o += *reinterpret_cast<const V4f*>(lds + (w * 16 + r) * LD + channel) * by;
        }
        const int query = row / a.shared, h = head * a.shared + row - query * a.shared;
        const int64_t token = seq.first + query;
        if (span.used > 1) {
          const int64_t part = (token * a.heads + h) * g.splits + split;
          *reinterpret_cast<V4f*>(g.parts + part * D + channel) = o;
          if (channel == 0) {
            float* const ms = g.parts + a.tokens * a.heads * g.splits * D + part * 2;
            ms[0] = most;
            ms[1] = total;
          }
          continue;
        }
        const float r1 = total == 0.f ? 0.f : 1.f / total;
        uint16_t* const dst = reinterpret_cast<uint16_t*>(a.out) + token * a.out_token + h * a.out_head + channel;
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[i] = (uint16_t)to_bits<BF>(o[i] * r1);
        if (a.sums && channel == 0) a.sums[token * a.heads + h] = (most + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
      }
      __syncthreads();
    }
  }
}

// The sums of a row's splits together.
template <int NG, bool BF, int RT>
__global__ __launch_bounds__(256) void join_kernel(const KvAttention a, const Grid g) {
  constexpr int D = 32 * NG, R = 16 * RT, LANES = D / 4, GROUPS = 256 / LANES;      // a group of lanes takes a split at a time
  __shared__ __align__(16) float lds[GROUPS][D];
  __shared__ float lds_sum[GROUPS];
  const int64_t id = blockIdx.x;
  const int h = (int)(id % a.heads), head = h / a.shared;
  const int64_t token = id / a.heads;
  // the sequence of a token
  int b = (int)token;
  if (a.start) {
    int lo = 0, hi = a.batch;                              // the last b with start[b] <= token
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.start[mid] <= token) lo = mid;
      else hi = mid;
    }
    b = lo;
  }
  const Sequence seq = sequence_of(a, b);
  const int query = (int)(token - seq.first);
  if (query < 0 || query >= seq.queries) return;
  const int row = query * a.shared + h - head * a.shared;
  const Span span = span_of(a, g, seq, row / R * R, R);
  if (span.used <= 1) return;
  const float* const parts = g.parts + id * g.splits * D;
  const float* const ms = g.parts + a.tokens * a.heads * g.splits * D + id * g.splits * 2;
  float most = -INFINITY;
  for (int s = 0; s < span.used; ++s) most = fmaxf(most, ms[2 * s]);
  const int group = threadIdx.x / LANES, channel = threadIdx.x % LANES * 4;
  if (group < GROUPS) {
    V4f o = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    for (int s = group; s < span.used; s += GROUPS) {
      const float by = ms[2 * s] == most ? 1.f : __builtin_amdgcn_exp2f(ms[2 * s] - most);
      total += ms[2 * s + 1] * by;
      o += *reinterpret_cast<const V4f*>(parts + (int64_t)s * D + channel) * by;
    }
    *reinterpret_cast<V4f*>(&lds[group][channel]) = o;
    if (channel == 0) lds_sum[group] = total;
  }
  __syncthreads();
  if (group > 0) return;
  V4f o = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < GROUPS; ++k) {
    o += *reinterpret_cast<const V4f*>(&lds[k][channel]);
    total += lds_sum[k];
  }
  const float r1 = total == 0.f ? 0.f : 1.f / total;
  uint16_t* const dst = reinterpret_cast<uint16_t*>(a.out) + token * a.out_token + h * a.out_head + channel;
#pragma unroll
  for (int i = 0; i < 4; ++i) dst[i] = (uint16_t)to_bits<BF>(o[i] * r1);
  if (a.sums && channel == 0) a.sums[id] = (most + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

// Two tiles of rows share the decoded values where there are more rows than one has (beyond 128 channels the registers do not hold two).
int row_tiles(const KvAttention& a) { return (int64_t)a.most_queries * a.shared > 16 && a.pool.dim <= 128 ? 2 : 1; }

Grid grid_of(const KvAttention& a) {
  Grid g{};
  const int64_t rows = 16 * row_tiles(a), unit = kWaves * kTile;
  g.row_blocks = (int32_t)(((int64_t)a.most_queries * a.shared + rows - 1) / rows);
  const int64_t others = (int64_t)a.batch * a.pool.heads * g.row_blocks, wanted = (int64_t)device_cu_count() * 4;
  const int64_t longest = std::max<int64_t>(1, std::min(a.longest, a.window ? (int64_t)a.window + a.most_queries + 15 : a.longest));
  int64_t splits = others > 0 ? (wanted + others - 1) / others : 1;
  splits = std::max<int64_t>(1, std::min({splits, (longest + 4 * unit - 1) / (4 * unit), (int64_t)256}));
  g.chunk = (longest + splits * unit - 1) / (splits * unit) * unit;
  g.splits = (int32_t)((longest + g.chunk - 1) / g.chunk);
  return g;
}

template <int NG, bool BF, int RT>
int launch_of(const KvAttention& a, const Grid& g, hipStream_t stream) {
  constexpr int lds = 4 * (kWaves * 16 * (32 * NG + 4) + 2 * kWaves * 16);
  const int64_t blocks = (int64_t)a.batch * a.pool.heads * g.row_blocks * g.splits, rows = a.tokens * a.heads;
  if (lds > 64 * 1024) MACKO_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_kernel<NG, BF, RT>), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  hipLaunchKernelGGL((attention_kernel<NG, BF, RT>), dim3((unsigned)blocks), dim3(64 * kWaves), lds, stream, a, g);
  MACKO_HIP_TRY(hipGetLastError());
  if (g.splits > 1) {
    hipLaunchKernelGGL((join_kernel<NG, BF, RT>), dim3((unsigned)rows), dim3(256), 0, stream, a, g);
    MACKO_HIP_TRY(hipGetLastError());
  }
  return MACKO_OK;
}

template <int NG>
int launch_dim(const KvAttention& a, const Grid& g, hipStream_t stream) {
  if constexpr (NG <= 4)
    if (row_tiles(a) == 2) return a.type == MACKO_BF16 ? launch_of<NG, true, 2>(a, g, stream) : launch_of<NG, false, 2>(a, g, stream);
  return a.type == MACKO_BF16 ? launch_of<NG, true, 1>(a, g, stream) : launch_of<NG, false, 1>(a, g, stream);
}

}  // namespace

bool kv_attention_fits(const KvAttention& a) {
  if (a.tokens == 0 || a.batch == 0) return true;
  constexpr int64_t kMost = (int64_t{1} << 24) - 1;       // workgroups of a launch of 256 threads each
  const int64_t rows = a.tokens * a.heads, pairs = (int64_t)a.batch * a.pool.heads;
  if (rows > kMostTokens || pairs > kMost) return false;
  const Grid g = grid_of(a);
  return pairs * g.row_blocks <= kMost && pairs * g.row_blocks * g.splits <= kMost && (g.splits == 1 || rows <= kMost);
}

int64_t kv_attention_workspace(const KvAttention& a) {
  if (a.tokens == 0 || a.batch == 0) return 0;
  const Grid g = grid_of(a);
  return g.splits > 1 ? a.tokens * a.heads * g.splits * (a.pool.dim + 2) : 0;
}

int launch_kv_attention(const KvAttention& a, float* workspace, hipStream_t stream) {
  Grid g = grid_of(a);
  g.parts = workspace;
  switch (a.pool.dim / 32) {
    case 1: return launch_dim<1>(a, g, stream);
    case 2: return launch_dim<2>(a, g, stream);
    case 3: return launch_dim<3>(a, g, stream);
    case 4: return launch_dim<4>(a, g, stream);
    case 5: return launch_dim<5>(a, g, stream);
    case 6: return launch_dim<6>(a, g, stream);
    case 7: return launch_dim<7>(a, g, stream);
    case 8: return launch_dim<8>(a, g, stream);
  }
  return MACKO_E_UNSUPPORTED;
}

}  // namespace macko
