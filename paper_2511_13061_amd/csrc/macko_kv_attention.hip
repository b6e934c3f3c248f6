// Attention over the paged 4-bit key/value cache (layout: macko_kv.h).
//
// Rows are the queries of one sequence for one key/value head, query by query and in it head by head, 16 to a tile.  A wavefront takes
// 32 tokens at a time:
//   scores   S^T = K Q^T by mfma_scale 16x16x128: keys go to the matrix cores as they lie in memory, 4-bit codes and the group's byte as the
//            block scale, without an instruction of the vector units.  Queries are 8-bit parts, each what the ones before left over (fp16: 3,
//            bf16: 2), with a scale of their own per 32 channels: together they hold every bit of a query down to 2^-18 (2^-13) of its group's largest.
//            The instruction lines its products up with the largest before it adds them.  Measured, of the sum of their magnitudes: normally distributed
//            queries and keys 2^-20 off in the mean, 2^-15.4 at worst; one product of 4000 beside 31 to 255 of about 1 2^-14.5 and 2^-12; heavy tails
//            (times e^(2x), x normal) 2^-15 and 2^-11.2.
//   softmax  running maximum and sum in 32 bits, the sum anew every 32 steps.  Column r of S^T is row r, so a lane holds 8 scores of one row; the running maximum moves
//            only when a score is more than 2^8 above it, and only then do lanes talk to each other.
//   values   O^T += V^T P^T by mfma 16x16x32 bf16: codes are exact in bf16 with any scale; weights go in as two bf16 parts (16 bits).
//            The lanes of S^T that hold a token's weights are those that P^T needs: nothing moves between lanes.
// The four wavefronts of a workgroup take turns along the tokens and join their sums in LDS; long sequences are split over workgroups
// too, whose unnormalised sums a second kernel joins.
//
// Memory bounds it for up to 16 rows: 16 sequences of 65536 tokens, 32 heads of 128 channels, 5.7 TB/s of the 6.0 that reading alone reaches; 64 of up to
// 4096 131 to 140 us (5.1 to 5.5 TB/s: workgroups that begin, and the last to end); one of 131072 35 to 38 us, 5 of them to begin and 4.5 to join.
#include <cmath>

#include "macko_kv_attention.h"

namespace macko {
namespace {

// What a wavefront holds of 32 tokens: two blocks of 16.
template <int NG>
struct Tile {
  static constexpr int NK = (NG + 3) / 4;
  V4i key[2][NK];
  int key_byte[2][NK];
  uint32_t value[2][NG], value_byte[2][NG];      // [token of 4][g] bytes
};

// Wavefronts on a SIMD that the registers are to leave room for, as many as they can without spills (several parts of a query in an instruction made room for
// one more of narrow heads).  Two for 160 and 192 channels a head: 3.3 to 5.2 and 4.0 to 6.1 TB/s.
constexpr int waves_wanted(int ng, int rt) { return rt == 2 ? (ng == 1 ? 4 : ng == 2 ? 3 : 2) : ng <= 2 ? 4 : ng <= 4 ? 3 : ng <= 6 ? 2 : 1; }

template <int NG, bool BF, int RT>
__global__ __launch_bounds__(64 * kWaves, waves_wanted(NG, RT)) void attention_kernel(const Launch args) {
  const KvAttention& a = args.a;
  const Grid& g = args.g;
  constexpr int D = 32 * NG, NK = (NG + 3) / 4, NP = BF ? 2 : 3, R = 16 * RT, LD = D + 4;
  // Narrow heads leave room in an instruction: it takes the same keys against SHARE parts of a query, channel 0 of part p at p D (64 sequences of up
  // to 4096 tokens, 32 heads of 64 channels 135 to 127 us, 64 rows on 64 of 2048 61 to 54).
  constexpr int SHARE = NG <= 2 ? 4 / NG : 1, NI = (NP + SHARE - 1) / SHARE;
  extern __shared__ __align__(16) float lds[];           // [kWaves][16][LD], maxima and sums [kWaves][16] each, and below
  float* const lds_max = lds + kWaves * 16 * LD;
  float* const lds_sum = lds_max + kWaves * 16;
  uint32_t* const lds_spoilt = reinterpret_cast<uint32_t*>(lds_sum + kWaves * 16);      // [RT][kWaves][16]: groups in which a row sees what is not a number
  uint32_t* const lds_q = lds_spoilt + RT * kWaves * 16;                                // [RT][NK][NP][64][8]
  // [RT][thread]: a lane's sum up to the last 32 steps, out of the registers' way.  A token that is far ahead of very many others would lose them, step by step.
  float* const lds_whole = reinterpret_cast<float*>(lds_q + RT * NK * NP * 512);
  uint8_t* const lds_byte = reinterpret_cast<uint8_t*>(lds_whole + RT * 64 * kWaves);   // [R][NG]

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x, split = g.splits == 1 ? 0 : g.row_blocks == 1 ? (int)blockIdx.z : (int)blockIdx.z / g.row_blocks, row_block = (int)blockIdx.z - split * g.row_blocks;
  int b = blockIdx.y;
  if (g.ordered) b = nth_longest(a, b, threadIdx.x & 63);
  const Sequence seq = sequence_of(a, b);
  const int32_t* const table = a.tables + b * a.table_stride;
  const int64_t piece = kv_piece_bytes(int64_t{1} << a.pool.page_bits, D), page_stride = piece * a.pool.heads;
  const uint8_t* const pool = a.pool.data + head * piece;
  const int page_size = 1 << a.pool.page_bits;
  // Weights are 2^(score * unit - maximum); the scale's sign goes into the queries, so that the largest score has the largest weight.
  const float unit = a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.4426950408889634f, sign = a.scale < 0.f ? -1.f : a.scale == 0.f ? 0.f : 1.f;
  const float lift = fminf(kLift / unit, 0x1p127f);      // finite: nothing is above -infinity by an infinity, and the first maximum would never be taken
  const uint32_t reach = a.window ? (uint32_t)a.window : 0x7FFFFFFFu;

  // the last rows see most and start first
  for (int first_row = (g.row_blocks - 1 - row_block) * R; first_row < seq.rows; first_row += g.row_blocks * R) {
    const Rows rows = rows_of(a, first_row);
    const Span span = span_of(a, g, seq, rows);
    if (split >= span.used) continue;
    // What follows from the lane is worked out here and again behind the steps (later(...)): kept from outside the loop it would hold registers.
    const int lane = later(threadIdx.x) & 63, n = lane & 15, j = lane >> 4;
    const int begin = span.lo + split * span.chunk, end = span.hi - begin > span.chunk ? begin + span.chunk : span.hi;

    bool bad = end > begin && (a.table_width == 0 || a.pool.pages == 0);     // a page that is needed is missing
    const int last_block = (end - 1) >> 4;
    float top[RT], sum[RT];
    V4f out[RT][2 * NG];
    auto gather = [&] {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        lds_whole[rt * 64 * kWaves + later(threadIdx.x)] += sum[rt];
        sum[rt] = 0.f;
      }
    };

    // A lane holds the page of one block of the wavefront's next 32 steps: one load for all of them, ahead of the loads that need it.
    int pages = 0;
    auto look_up = [&](int at) {
      const int block = min((at >> 4) + (lane >> 1) * (kWaves * 2) + (lane & 1), last_block), index = block >> (a.pool.page_bits - 4);
      const int page = table[min(index, a.table_width - 1)];
      const bool fine = index < a.table_width && page >= 0 && page < a.pool.pages;
      bad = bad || __any(!fine);
      pages = fine ? page : 0;
    };
    const int key_group = SHARE > 1 ? j % NG : j;
    const uint32_t key_lane = n * (D / 2) + key_group * 16, key_byte_lane = n * NG + key_group, value_lane = (j * 16 + n) * (4 * NG), value_byte_lane = j * (4 * NG);
    auto load = [&](Tile<NG>& t, int at, int slot) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int block = min((at >> 4) + u, last_block), in_page = (block << 4) & (page_size - 1);
        const uint8_t* const codes = pool + (int64_t)__builtin_amdgcn_readlane(pages, slot * 2 + u) * page_stride + in_page * (D / 2);
        const uint8_t* const bytes = codes + page_size * D - in_page * (D / 2 - NG);
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
          const int group = kk * 4 + key_group;
          t.key[u][kk] = V4i{0, 0, 0, 0};
          t.key_byte[u][kk] = 0;
          if (group < NG) {
            t.key[u][kk] = *reinterpret_cast<const V4i*>(codes + key_lane + kk * 64);
            t.key_byte[u][kk] = bytes[key_byte_lane + kk * 4];
          }
        }
        const uint32_t* const v = reinterpret_cast<const uint32_t*>(codes + page_size * (D / 2) + value_lane);
        const uint32_t* const vb = reinterpret_cast<const uint32_t*>(bytes + page_size * NG + value_byte_lane);
#pragma unroll
        for (int w = 0; w < NG; ++w) {
          t.value[u][w] = v[w];
          t.value_byte[u][w] = vb[w];
        }
      }
    };
    Tile<NG> one, two;
    const int mine = begin + wave * kTile;                // the wavefront's first step
    const bool any = mine < end && !bad;
    if (any) {                                            // on its way while the queries are made ready
      look_up(mine);
      load(one, mine, 0);
    }

    if (lane < 16) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) lds_spoilt[(rt * kWaves + wave) * 16 + lane] = 0;
    }
    int place[RT];                                        // of a row's query: it sees the tokens t with 0 <= place - t < reach
    V8i q[RT][NK][NI];
    int q_byte[RT][NK];
    // The queries' operand (load_queries says what it is), 8 channels of a row by each thread, through LDS to the lanes of all wavefronts.
    constexpr int kChunks = R * 4 * NG, kTurns = (kChunks + 64 * kWaves - 1) / (64 * kWaves);
#pragma unroll
    for (int turn = 0; turn < kTurns; ++turn) {
      const int chunk = turn * 64 * kWaves + (wave * 64 + lane), r = chunk / (4 * NG), c = chunk % (4 * NG);
      if (chunk >= kChunks) break;
      const int row = first_row + r, query = rows.query_of(a, g, row);
      Packed8 raw = {0, 0, 0, 0};
      if (row < seq.rows)
        raw = *reinterpret_cast<const Packed8Any*>(reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(seq.first + query) * a.q_token +
                                                   (int64_t)(head * a.shared + row - query * a.shared) * a.q_head + c * 8);
      float x[8];
      unpack8<BF>(raw, x);
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu);
      most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xF, 0xF, true));      // the quad has a group
      most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4E, 0xF, 0xF, true));
      const uint32_t byte = max(most >> 23, 20u) - 7u;
      const float up = __builtin_bit_cast(float, (254u - byte) << 23) * sign;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= up;
      uint32_t* to = lds_q + (((r >> 4) * NK + (c >> 4)) * NP * 64 + ((c & 7) >> 1) * 16 + (r & 15)) * 8 + ((c & 8) >> 1) + (c & 1) * 2;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        uint2 words;
        words.x = (uint32_t)part_of(x);
        words.y = (uint32_t)part_of(x + 4);
        *reinterpret_cast<uint2*>(to + p * 512) = words;
      }
      if ((c & 3) == 0) lds_byte[r * NG + (c >> 2)] = (uint8_t)byte;
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = first_row + rt * 16 + n;
      place[rt] = row < seq.rows ? seq.length - seq.queries + rows.query_of(a, g, row) : -1;
      if constexpr (SHARE > 1) {
        auto part_at = [&](int p, int lane_of) { return *reinterpret_cast<const V4i*>(lds_q + ((rt * NP + p) * 64 + lane_of) * 8); };
        const int t = lds_byte[(rt * 16 + n) * NG + key_group];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          // part by group of lanes: the low half of the operand has channels 16 j of it, the high half 64 on
          const int p = i * SHARE + (NG == 1 ? j >> 1 : 0), p_high = NG == 1 ? 2 + (j >> 1) : i * SHARE + 1, from = NG == 1 ? (j & 1) * 16 + n : lane;
          const V4i low = part_at(min(p, NP - 1), from), high = part_at(min(p_high, NP - 1), from);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            q[rt][0][i][w] = p < NP ? low[w] : 0;
            q[rt][0][i][4 + w] = p_high < NP ? high[w] : 0;
          }
        }
        q_byte[rt][0] = (t - 4 * min(j / NG, NP - 1)) | (t - 8) << 8;
      } else {
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const V4i* const from = reinterpret_cast<const V4i*>(lds_q + (((rt * NK + kk) * NP + p) * 64 + lane) * 8);
            V4i half[2] = {from[0], from[1]};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              if (NG % 4 != 0 && kk * 128 + u * 64 + j * 16 >= D) half[u] = V4i{0, 0, 0, 0};      // no such channels
#pragma unroll
              for (int w = 0; w < 4; ++w) q[rt][kk][p][u * 4 + w] = half[u][w];
            }
          }
          const int t = kk * 4 + j < NG ? lds_byte[(rt * 16 + n) * NG + kk * 4 + j] : 20;
          q_byte[rt][kk] = t | (t - 4) << 8 | (t - 8) << 16;
        }
      }
    }

    auto step = [&](Tile<NG>& t, int at, bool careful) {
      const bool masked = at < span.all_lo || at + kTile > span.all_hi;
      V4i p_hi[RT], p_lo[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          V4f s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < NK; ++kk) {
            const V8i key = {t.key[u][kk][0], t.key[u][kk][1], t.key[u][kk][2], t.key[u][kk][3], 0, 0, 0, 0};
            if (NI == 3) s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, q[rt][kk][NI - 1], s, 4, 0, 0, t.key_byte[u][kk], 2, q_byte[rt][kk]);
            if (NI >= 2) s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, q[rt][kk][NI >= 2 ? 1 : 0], s, 4, 0, 0, t.key_byte[u][kk], 1, q_byte[rt][kk]);
            s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, q[rt][kk][0], s, 4, 0, 0, t.key_byte[u][kk], 0, q_byte[rt][kk]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) x[4 * u + i] = s[i];
        }
        if (masked) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int token = at + (i >> 2) * 16 + j * 4 + (i & 3);
            if ((uint32_t)(place[rt] - token) >= reach) x[i] = -INFINITY;
          }
        }
        const float most = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__any(most > top[rt] + lift)) {
          float to = fmaxf(most, __shfl_xor(most, 16));
          to = fmaxf(to, __shfl_xor(to, 32));
          to = fmaxf(to, top[rt]);
          const float by = to == top[rt] ? 1.f : __builtin_amdgcn_exp2f((top[rt] - to) * unit);
          top[rt] = to;
          sum[rt] *= by;
          lds_whole[rt * 64 * kWaves + later(threadIdx.x)] *= by;
#pragma unroll
          for (int c = 0; c < 2 * NG; ++c) out[rt][c] *= by;
        }
        const float base = top[rt] == -INFINITY ? 0.f : -top[rt] * unit;       // nothing seen yet: weights of 2^-inf, not NaN
        float weight[8], more = 0.f;                       // `more`: of the step alone, for the same reason as lds_whole
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          weight[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], unit, base));
          more = i == 0 ? weight[0] : more + weight[i];
        }
        sum[rt] += more;
        parts_of<false>(weight, p_hi[rt], p_lo[rt]);
      }
      if (careful || at + kTile > seq.length) {
        // Tokens behind the sequence's end may hold anything: their factor becomes the least one.  In a careful pass that of values that may
        // not be numbers does too, and rows that see them are marked.
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int token = at + u * 16 + j * 4 + k;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
              const int byte = k * NG + i, shift = 8 * (byte & 3);
              uint32_t& word = t.value_byte[u][byte >> 2];
              const bool nan = (word >> shift & 255u) >= kNoNumber && token < seq.length;
              if (token >= seq.length || (careful && nan)) word &= ~(255u << shift);
              if (careful && nan) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                  if ((uint32_t)(place[rt] - token) < reach) atomicOr(lds_spoilt + (rt * kWaves + wave) * 16 + n, 1u << i);
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
            const uint32_t v0 = decode_at<false>(t.value[u][b0 >> 2], t.value_byte[u][b0 >> 2], b0 & 3);
            const uint32_t v1 = decode_at<false>(t.value[u][b1 >> 2], t.value_byte[u][b1 >> 2], b1 & 3);
            lower[u * 2 + k / 2] = (int)__builtin_amdgcn_perm(v1, v0, 0x05040100u);
            upper[u * 2 + k / 2] = (int)__builtin_amdgcn_perm(v1, v0, 0x07060302u);
          }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          out[rt][2 * i] = multiply<false>(lower, p_lo[rt], out[rt][2 * i]);
          out[rt][2 * i + 1] = multiply<false>(upper, p_lo[rt], out[rt][2 * i + 1]);
          out[rt][2 * i] = multiply<false>(lower, p_hi[rt], out[rt][2 * i]);
          out[rt][2 * i + 1] = multiply<false>(upper, p_hi[rt], out[rt][2 * i + 1]);
        }
      }
    };

    bool again, marked = false;
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        top[rt] = -INFINITY;
        sum[rt] = lds_whole[rt * 64 * kWaves + later(threadIdx.x)] = 0.f;
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c) out[rt][c] = V4f{0.f, 0.f, 0.f, 0.f};
      }
      if (any) {
        int at = mine, slot = 0;
        if (pass > 0) {
          look_up(at);
          load(one, at, 0);
        }
        auto ahead = [&](Tile<NG>& t, int next) {
          if (next >= end) return;
          if (++slot == 32) {
            look_up(next);
            slot = 0;
            gather();
          }
          load(t, next, slot);
        };
        for (;;) {
          ahead(two, at + kWaves * kTile);
          step(one, at, pass > 0);
          at += kWaves * kTile;
          if (at >= end) break;
          ahead(one, at + kWaves * kTile);
          step(two, at, pass > 0);
          at += kWaves * kTile;
          if (at >= end) break;
        }
      }
      // A value that is not a number, or infinite, reaches every row of its tile, with weight 0 where it is not seen: then the tokens are gone
      // through again, carefully.  (A row's own NaN, of its query or a key that it sees, gets here too, and costs time alone.)
      float all[4] = {0.f, 0.f, 0.f, 0.f};                // infinities of both signs make one too: time alone
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) all[i] += out[rt][c][i];
      const float one_of = (all[0] + all[1]) + (all[2] + all[3]);
      again = pass == 0 && __any(one_of != one_of);
      if (!again) break;
      marked = true;
    }

    // What the results need of the arguments is read again here, rather than kept in registers through the steps.
    LaunchPtr e = (LaunchPtr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(e));
    const int rows_of_sequence = seq.rows, first_of_sequence = seq.first;
    const int thread = later(threadIdx.x), row16 = thread & 15, quad = thread >> 4 & 3;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      sum[rt] += lds_whole[rt * 64 * kWaves + thread];
      sum[rt] += __shfl_xor(sum[rt], 16);
      sum[rt] += __shfl_xor(sum[rt], 32);
      if (bad) sum[rt] = NAN;
      if (marked) {
        const uint32_t spoilt = lds_spoilt[(rt * kWaves + wave) * 16 + row16];
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c)
          if (spoilt >> (c / 2) & 1) out[rt][c] = V4f{NAN, NAN, NAN, NAN};
      }
      float* const mine = lds + (wave * 16 + row16) * LD;
#pragma unroll
      for (int c = 0; c < 2 * NG; ++c) *reinterpret_cast<V4f*>(mine + c * 16 + quad * 4) = out[rt][c];
      if (quad == 0) {
        lds_max[wave * 16 + row16] = top[rt] * unit;
        lds_sum[wave * 16 + row16] = sum[rt];
      }
      __syncthreads();
      for (int item = thread; item < 4 * D; item += 64 * kWaves) {
        const int r = item / (D / 4), channel = item % (D / 4) * 4, row = first_row + rt * 16 + r;
        if (row >= rows_of_sequence) continue;
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
        const int query = rows.query_of(a, g, row), h = head * e->a.shared + row - query * e->a.shared;
        const int64_t token = first_of_sequence + query;
        if (span.used > 1) {
          const int64_t part = (token * e->a.heads + h) * e->g.splits + split;
          *reinterpret_cast<V4f*>(e->g.parts + part * D + channel) = o;
          if (channel == 0) {
            float* const ms = e->g.parts + e->a.tokens * e->a.heads * e->g.splits * D + part * 2;
            ms[0] = most;
            ms[1] = total;
            if (split == 0) used_splits(e->a, e->g)[token * e->a.heads + h] = span.used;
          }
          continue;
        }
        const float r1 = total == 0.f ? 0.f : 1.f / total;
        typedef uint32_t Pair __attribute__((ext_vector_type(2), aligned(2)));
        *reinterpret_cast<Pair*>(reinterpret_cast<uint16_t*>(e->a.out) + token * e->a.out_token + h * e->a.out_head + channel) =
            Pair{pack2<BF>(o[0] * r1, o[1] * r1), pack2<BF>(o[2] * r1, o[3] * r1)};
        if (e->g.splits > 1 && channel == 0) used_splits(e->a, e->g)[token * e->a.heads + h] = 1;
        if (e->a.sums && channel == 0) e->a.sums[token * e->a.heads + h] = (most + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
      }
      __syncthreads();
    }
  }
}

// The sums of a row's splits together; the rows whose tokens were not split have their results already.
template <bool BF>
__device__ inline void write_joined(const KvAttention& a, int64_t id, int channel, V4f o, float most, float total) {
  const int h = (int)(id % a.heads);
  const int64_t token = id / a.heads;
  const float r = total == 0.f ? 0.f : 1.f / total;
  typedef uint32_t Pair __attribute__((ext_vector_type(2), aligned(2)));
  *reinterpret_cast<Pair*>(reinterpret_cast<uint16_t*>(a.out) + token * a.out_token + h * a.out_head + channel) = Pair{pack2<BF>(o[0] * r, o[1] * r), pack2<BF>(o[2] * r, o[3] * r)};
  if (a.sums && channel == 0) a.sums[id] = (most + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

// Few splits: a wavefront has a row, a lane the maximum and the sum of one split.  512 rows of 32 heads with 64 channels in 4 parts: 96 us with the attention,
// 111 with a workgroup a row; with more parts a row's reads take longer than a wavefront's share is worth (8 rows in 32 parts 14.6 and 13.6).
constexpr int kFewSplits = 16;
template <int NG, bool BF>
__global__ __launch_bounds__(256) void join_few_kernel(const KvAttention a, const Grid g) {
  constexpr int D = 32 * NG, LANES = D / 4, GROUPS = LANES > 32 ? 1 : LANES > 16 ? 2 : LANES > 8 ? 4 : 8;      // a group of lanes takes a split at a time
  const int64_t rows = a.tokens * a.heads, id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= rows) return;
  const int lane = threadIdx.x & 63, group = lane / LANES, channel = lane % LANES * 4;
  const float* const parts = g.parts + id * g.splits * D;
  const float* const ms = g.parts + rows * g.splits * D + id * g.splits * 2;
  // on their way before it is known how many splits there are
  float top = -INFINITY, sum = 0.f;
  if (lane < g.splits) top = ms[2 * lane], sum = ms[2 * lane + 1];
  const int used = min(used_splits(a, g)[id], g.splits);
  if (used <= 1) return;
  if (lane >= used) top = -INFINITY, sum = 0.f;
  float most = top;
  for (int m = 1; m < kFewSplits; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
  most = __shfl(most, 0);
  const float by = top == most ? 1.f : __builtin_amdgcn_exp2f(top - most);
  float total = sum * by;
  for (int m = 1; m < kFewSplits; m <<= 1) total += __shfl_xor(total, m);
  total = __shfl(total, 0);
  V4f o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < used; s0 += 4 * GROUPS) {
    V4f part[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int s = s0 + k * GROUPS + group;
      part[k] = V4f{0.f, 0.f, 0.f, 0.f};
      if (group < GROUPS && s < used) part[k] = *reinterpret_cast<const V4f*>(parts + (int64_t)s * D + channel);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int s = s0 + k * GROUPS + group;
      const float w = __shfl(by, s & 63);
      if (s < used) o += part[k] * w;
    }
  }
#pragma unroll
  for (int m = GROUPS / 2; m > 0; m /= 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl(o[i], (lane + m * LANES) & 63);
  }
  if (group == 0) write_joined<BF>(a, id, channel, o, most, total);
}

template <int NG, bool BF>
__global__ __launch_bounds__(256) void join_kernel(const KvAttention a, const Grid g) {
  constexpr int D = 32 * NG, LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ __align__(16) float lds[GROUPS][D];
  __shared__ float weight[kMostSplits], most_of[4], total_of[4];
  const int64_t id = blockIdx.x, rows = a.tokens * a.heads;
  const float* const parts = g.parts + id * g.splits * D;
  const float* const ms = g.parts + rows * g.splits * D + id * g.splits * 2;
  const int mine = threadIdx.x, wave = mine >> 6, group = mine / LANES, channel = mine % LANES * 4;
  float top = -INFINITY, sum = 0.f;
  static_assert(kMostSplits == 256, "a thread has one split's maximum");
  if (mine < g.splits) top = ms[2 * mine], sum = ms[2 * mine + 1];
  const int used = min(used_splits(a, g)[id], g.splits);
  if (used <= 1) return;
  if (mine >= used) top = -INFINITY, sum = 0.f;
  float most = top;
  for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
  if ((mine & 63) == 0) most_of[wave] = most;
  __syncthreads();
  most = fmaxf(fmaxf(most_of[0], most_of[1]), fmaxf(most_of[2], most_of[3]));
  const float by = top == most ? 1.f : __builtin_amdgcn_exp2f(top - most);
  weight[mine] = by;
  float total = sum * by;
  for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
  if ((mine & 63) == 0) total_of[wave] = total;
  __syncthreads();
  V4f o = {0.f, 0.f, 0.f, 0.f};
  if (group < GROUPS) {
#pragma unroll 4
    for (int s = group; s < used; s += GROUPS) o += *reinterpret_cast<const V4f*>(parts + (int64_t)s * D + channel) * weight[s];
    *reinterpret_cast<V4f*>(&lds[group][channel]) = o;
  }
  __syncthreads();
  if (group > 0) return;
  o = V4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < GROUPS; ++k) o += *reinterpret_cast<const V4f*>(&lds[k][channel]);
  write_joined<BF>(a, id, channel, o, most, (total_of[0] + total_of[1]) + (total_of[2] + total_of[3]));
}

// Two tiles of rows share the decoded values where there are more rows than one has (beyond 128 channels the registers do not hold two): 32 rows on 16
// sequences of 4096 tokens, 8 heads of 128 channels 32 us, 35 with one tile; 20 rows 30 and 32, 128 rows 72 and 99.
int row_tiles(const KvAttention& a) { return (int64_t)a.most_queries * a.shared > 16 && a.pool.dim <= 128 ? 2 : 1; }
// Rows up to which the kernel for many rows is not thought of: half of a workgroup's have none there (64 rows on 16 sequences of 4096 tokens, 8 heads of 128
// channels: 73 us, 47 here).
constexpr int kPromptRows = 64;
// Rows of a workgroup
int rows_of_block(const KvAttention& a, bool prompt) { return prompt ? 16 * kWaves * prompt_row_tiles(a.pool.dim) : 16 * row_tiles(a); }
bool is_prompt(const Grid& g) { return g.rows >= 64; }

constexpr int64_t kMostGrid = 65535;       // of a launch's second and third dimension

bool may_join(const KvAttention& a) { return a.tokens * a.heads < int64_t{1} << 24; }      // a join has a workgroup a row, and a launch fewer than 2^32 threads

struct Dealt {
  int64_t splits;
  double time;
};
// How many parts the tokens of a sequence are dealt out to: the number with the shortest estimate, in microseconds.  A workgroup goes on by 128 tokens (one
// step of each wavefront, two for many rows) in the time that it takes alone, or that the workgroups of a compute unit take for one each where that is
// longer: from memory (6 TB/s, once for all rows of a sequence) or on the vector units and matrix cores.  Workgroups take turns where more of them come than fit, and each has 5 to begin and
// to end.  Joining costs a launch, the sums' way through memory and something for each part.  Constants from 75 calls of 1 to 64 sequences of 256 to 131072
// tokens, 1 to 1024 queries, heads of 32 to 256 channels, with 1 to 128 parts each and, of 96 to 2048 rows, by both kernels; the choice of parts and kernel
// took 2 % longer than the best of these in the mean, 14 % at worst.  What it chooses for 16 sequences of 4096, 8 heads of 128
// channels in bf16 (this kernel / the one for many rows): 128 rows 66 us (66 / 67), 256 rows 113 (124 / 112), 512 rows 172 (232 / 172).
Dealt deal(const KvAttention& a, bool prompt, int64_t row_blocks, int64_t units, int64_t unit_bytes) {
  static constexpr int kTry[] = {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256};
  static_assert(kMostSplits == 256, "the last one tried");
  const int64_t others = (int64_t)a.batch * a.pool.heads * row_blocks;
  const double cus = device_cu_count(), rows = (double)a.tokens * a.heads;
  const bool two = !prompt && row_tiles(a) == 2, wide = a.pool.dim > 128, narrow = a.pool.dim <= 64, one_part = prompt && a.type == MACKO_BF16;
  const double alone = prompt ? (wide ? 6.4 : narrow ? 4.5 : 5.1) * (one_part ? 0.82 : 1.0) : two ? 1.3 : wide ? 1.4 : 0.9;
  const double busy_share = prompt ? (narrow ? 2.2 : 3.2) * (one_part ? 0.82 : 1.0) : two ? (narrow ? 0.65 : 0.86) : wide ? 0.82 : 0.45;
  const double room = two && narrow ? 3 : prompt || two ? 2 : a.pool.dim > 192 ? 1 : wide ? 2 : 3, share = std::max((double)unit_bytes * cus / 6.0e6 / (double)row_blocks, busy_share);
  auto time = [&](int64_t splits) {
    const double groups = (double)(others * splits) / cus, steps = (double)((units + splits - 1) / splits), busy = std::min(std::ceil(groups), room);
    const double turns = groups <= 4.0 * room ? std::ceil(groups / room) : groups / room + 0.5;
    const double join = splits > 1 ? 3.4 + 0.02 * (double)splits + rows * (double)splits * (a.pool.dim + 2) * 8.0 / 4.0e6 : 0.0;
    return turns * (5.0 + steps * std::max(alone, busy * share)) + join;
  };
  Dealt best{1, time(1)};
  if (!may_join(a)) return best;
  for (const int splits : kTry) {
    if (splits > units) break;
    const double t = time(splits);
    if (t < best.time) best = Dealt{splits, t};
  }
  return best;
}

Grid grid_of(const KvAttention& a) {
  Grid g{};
  g.unit = kWaves * kTile;
  g.shared_inverse = a.shared == 1 ? 0u : (uint32_t)(((uint64_t{1} << 32) + a.shared - 1) / a.shared);
  const int64_t unit = g.unit, most_rows = (int64_t)a.most_queries * a.shared;
  const int64_t longest = std::max<int64_t>(1, std::min({a.longest, (int64_t)kMostTokens, a.window ? (int64_t)a.window + a.most_queries + 15 : a.longest}));
  auto blocks_of = [&](bool prompt) { return (most_rows + rows_of_block(a, prompt) - 1) / rows_of_block(a, prompt); };
  auto dealt = [&](bool prompt) { return deal(a, prompt, std::max<int64_t>(1, blocks_of(prompt)), (longest + unit - 1) / unit, kv_piece_bytes(unit, a.pool.dim)); };
  const Tuning& knobs = tuning();
  bool prompt = knobs.attention_kernel == 2;
  Dealt dealt_out = dealt(prompt);
  if (knobs.attention_kernel == 0 && most_rows > kPromptRows) {
    const Dealt as_prompt = dealt(true);
    if (as_prompt.time < dealt_out.time) dealt_out = as_prompt, prompt = true;
  }
  if (knobs.attention_parts > 0 && may_join(a)) dealt_out.splits = std::min({knobs.attention_parts, (longest + unit - 1) / unit, (int64_t)kMostSplits});
  const int64_t splits = dealt_out.splits, row_blocks = blocks_of(prompt), others = (int64_t)a.batch * a.pool.heads * row_blocks;
  g.rows = rows_of_block(a, prompt);
  g.chunk = (longest + splits * unit - 1) / (splits * unit) * unit;
  g.splits = (int32_t)((longest + g.chunk - 1) / g.chunk);
  g.row_blocks = (int32_t)std::min(row_blocks, kMostGrid / g.splits);      // of a launch: a workgroup goes on to others
  g.ordered = a.batch > 1 && a.batch <= 64 && others * g.splits > 3 * (int64_t)device_cu_count();
  return g;
}

template <int NG, bool BF, int RT>
int launch_of(const KvAttention& a, const Grid& g, hipStream_t stream) {
  constexpr int lds = 4 * (kWaves * 16 * (32 * NG + 4) + (2 + RT) * kWaves * 16 + RT * ((NG + 3) / 4) * (BF ? 2 : 3) * 512 + RT * 64 * kWaves) + 16 * RT * NG;
  if (lds > 64 * 1024) MACKO_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_kernel<NG, BF, RT>), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  hipLaunchKernelGGL((attention_kernel<NG, BF, RT>), dim3((unsigned)a.pool.heads, (unsigned)a.batch, (unsigned)(g.row_blocks * g.splits)), dim3(64 * kWaves), lds, stream, Launch{a, g});
  MACKO_HIP_TRY(hipGetLastError());
  return MACKO_OK;
}

template <int NG, bool BF>
int launch_type(const KvAttention& a, const Grid& g, hipStream_t stream) {
  int status = MACKO_OK;
  bool one = true;
  if (is_prompt(g)) {
    status = launch_prompt(a, g, stream);
    one = false;
  } else if constexpr (NG <= 4) {
    if (row_tiles(a) == 2) {
      status = launch_of<NG, BF, 2>(a, g, stream);
      one = false;
    }
  }
  if (one) status = launch_of<NG, BF, 1>(a, g, stream);
  if (status == MACKO_OK && g.splits > 1) {
    const int64_t rows = a.tokens * a.heads;
    if (g.splits <= kFewSplits) hipLaunchKernelGGL((join_few_kernel<NG, BF>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, a, g);
    else hipLaunchKernelGGL((join_kernel<NG, BF>), dim3((unsigned)rows), dim3(256), 0, stream, a, g);
    MACKO_HIP_TRY(hipGetLastError());
  }
  return status;
}

template <int NG>
int launch_dim(const KvAttention& a, const Grid& g, hipStream_t stream) {
  return a.type == MACKO_BF16 ? launch_type<NG, true>(a, g, stream) : launch_type<NG, false>(a, g, stream);
}

}  // namespace

bool kv_attention_fits(const KvAttention& a) {
  if (a.tokens == 0 || a.batch == 0) return true;
  const int64_t rows = a.tokens * a.heads;
  return rows <= kMostTokens && a.batch <= kMostGrid && a.shared <= 32768;
}

int64_t kv_attention_workspace(const KvAttention& a) {
  if (a.tokens == 0 || a.batch == 0) return 0;
  const Grid g = grid_of(a);
  return g.splits > 1 ? a.tokens * a.heads * (g.splits * (int64_t)(a.pool.dim + 2) + 1) : 0;
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
