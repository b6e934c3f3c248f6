// Attention over the paged 8-bit key/value cache (layout: macko_kv8.h), few rows.
//
// Rows are the queries of one sequence for one key/value head, query by query and in it head by head, 16 to a tile.  A wavefront takes
// 32 tokens at a time, two blocks, straight from memory into the operands of mfma 16x16x32:
//   scores   S^T = K Q^T in the queries' type, which holds every code exactly; products of 16 bits, sums of 32.  A block's power of two goes onto its codes (bf16, where
//            it changes nothing but the exponent) or onto its scores (fp16, whose exponents do not reach as far).
//   softmax  running maximum and sum in 32 bits.  Column r of S^T is row r, so a lane holds 8 scores of one row; the running maximum moves only when a score
//            is more than 2^8 above it, and only then do lanes talk to each other.  The sum is taken anew every 32 steps.
//   values   O^T += V^T P^T in bf16, which holds codes exactly with any of the scales; weights go in as two bf16 parts (16 bits).  The lanes of S^T that hold a
//            token's weights are those that P^T needs, and a lane's 4 tokens of a channel are a word of the cache: nothing moves between lanes.
// The four wavefronts of a workgroup take turns along the tokens and join their sums in LDS; long sequences are split over workgroups
// too, whose unnormalised sums a second kernel joins.
// Memory bounds long calls: one token over 131072, 32 query heads on 8 of 128 channels, 46 us (5.8 TB/s with the joining; 54 from Python); 64 sequences of 4096 with 32 heads of 128 channels 385 us
// (5.6 TB/s); 16 of 4096 tokens with 8 heads 28 us (4.7).  50 tokens take 5.5 us, a launch and the chain length, table, keys.
#include <cmath>

#include "macko_kv8_attention.h"

namespace macko {
namespace {

// What a wavefront holds of 32 tokens: two blocks of 16.
template <int NG>
struct Tile8 {
  uint32_t key[2][2 * NG], value[2][2 * NG];
  uint32_t scale[2];
};

constexpr int waves_wanted(int ng, int rt) { return rt == 2 ? (ng == 1 ? 3 : 2) : ng == 1 ? 4 : ng == 2 ? 3 : ng <= 4 ? 2 : 1; }

template <int NG, bool BF, int RT>
__global__ __launch_bounds__(64 * kWaves, waves_wanted(NG, RT)) void attention8_kernel(const Launch8 args) {
  const KvAttention& a = args.a;
  const Grid& g = args.g;
  constexpr int D = 32 * NG, R = 16 * RT, LD = D + 4, FULL = NG / 2, REST = NG % 2;      // groups of 64 channels, and of 32
  extern __shared__ __align__(16) float lds[];           // [kWaves][16][LD], maxima and sums [kWaves][16] each, and below
  float* const lds_max = lds + kWaves * 16 * LD;
  float* const lds_sum = lds_max + kWaves * 16;
  int* const lds_place = reinterpret_cast<int*>(lds_sum + kWaves * 16);                 // [R]
  uint32_t* const lds_spoilt = reinterpret_cast<uint32_t*>(lds_place + R);              // [R][NG]: channels in which a row sees what is not a number
  // [RT][thread]: a lane's sum up to the last 32 steps, out of the registers' way.  A token that is far ahead of very many others would lose them, step by step.
  float* const lds_whole = reinterpret_cast<float*>(lds_spoilt + R * NG);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x, split = g.splits == 1 ? 0 : g.row_blocks == 1 ? (int)blockIdx.z : (int)blockIdx.z / g.row_blocks, row_block = (int)blockIdx.z - split * g.row_blocks;
  int b = blockIdx.y;
  if (g.ordered) b = nth_longest(a, b, threadIdx.x & 63);
  const Sequence seq = sequence_of(a, b);
  const int32_t* const table = a.tables + b * a.table_stride;
  const int block_bits = a.pool.page_bits - kBlockBits;  // log2 of a page's blocks
  // Weights are 2^(score * unit - maximum); the scale's sign goes into the queries, so that the largest score has the largest weight.
  const float unit = scalar(a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.4426950408889634f);
  const float lift = scalar(fminf(kLift / unit, 0x1p127f));      // finite: nothing is above -infinity by an infinity, and the first maximum would never be taken
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : 0xFFFFFFFFu;
  const uint32_t reach = a.window ? (uint32_t)a.window : 0x7FFFFFFFu;

  // the last rows see most and start first
  for (int first_row = (g.row_blocks - 1 - row_block) * R; first_row < seq.rows; first_row += g.row_blocks * R) {
    const Rows rows = rows_of(a, first_row);
    const Span span = span_of(a, g, seq, rows);
    if (split >= span.used) continue;
    const int lane = later(threadIdx.x) & 63, n = lane & 15, j = lane >> 4;
    const int begin = span.lo + split * span.chunk, end = span.hi - begin > span.chunk ? begin + span.chunk : span.hi;
    bool bad = end > begin && (a.table_width == 0 || a.pool.pages == 0);     // a page that is needed is missing
    const int last_block = (end - 1) >> 4;

    // A lane holds the page of one block of the wavefront's next 32 steps: one load for all of them, ahead of the loads that need it.
    int pages = 0;
    auto look_up = [&](int at) {
      const int block = min((at >> 4) + (lane >> 1) * (kWaves * 2) + (lane & 1), last_block), index = block >> block_bits;
      const int page = table[min(index, a.table_width - 1)];
      const bool fine = index < a.table_width && page >= 0 && page < a.pool.pages;
      bad = bad || __any(!fine);
      pages = fine ? page : 0;
    };
    const uint32_t key_lane = n * D + j * 16, key_rest = n * D + FULL * 64 + j * 8, value_lane = 16 * D + j * 4 * D + n * 16, value_rest = 16 * D + j * 4 * D + FULL * 256 + n * 8;
    auto load = [&](Tile8<NG>& t, int at, int slot) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int block = min((at >> 4) + u, last_block);
        const int64_t index = (((int64_t)__builtin_amdgcn_readlane(pages, slot * 2 + u) * a.pool.heads + head) << block_bits) + (block & ((1 << block_bits) - 1));
        const uint8_t* const codes = a.pool.data + index * (32 * D);
        t.scale[u] = *reinterpret_cast<const uint16_t*>(args.scales + index * 2);
#pragma unroll
        for (int i = 0; i < FULL; ++i) load_words<4>(t.key[u] + 4 * i, codes + key_lane + i * 64);
        if (REST) load_words<2>(t.key[u] + 4 * FULL, codes + key_rest);
#pragma unroll
        for (int i = 0; i < FULL; ++i) load_words<4>(t.value[u] + 4 * i, codes + value_lane + i * 256);
        if (REST) load_words<2>(t.value[u] + 4 * FULL, codes + value_rest);
      }
    };
    Tile8<NG> one, two;
    const int mine = begin + wave * kTile;                // the wavefront's first step
    const bool any = mine < end && !bad;
    if (any) {                                            // on its way while the queries are made ready
      look_up(mine);
      load(one, mine, 0);
    }

    // Queries as the operand: a lane has the channels that a lane of the keys has.
    V4i q[RT][NG];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = first_row + rt * 16 + n, query = rows.query_of(a, g, row);
      const bool there = row < seq.rows;
      const uint16_t* const src = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(seq.first + query) * a.q_token + (int64_t)(head * a.shared + row - query * a.shared) * a.q_head;
#pragma unroll
      for (int s = 0; s < NG; ++s) {
        Packed8 raw = {0, 0, 0, 0};
        if (there) raw = *reinterpret_cast<const Packed8Any*>(src + (s < 2 * FULL ? (s / 2) * 64 + j * 16 + (s & 1) * 8 : FULL * 64 + j * 8));
#pragma unroll
        for (int i = 0; i < 4; ++i) q[rt][s][i] = (int)((raw[i] ^ flip) & keep);
      }
      // of a row's query: it sees the tokens t with 0 <= place - t < reach
      if (wave == 0 && j == 0) lds_place[rt * 16 + n] = there ? seq.length - seq.queries + query : -1;
    }
    for (int i = threadIdx.x; i < R * NG; i += 64 * kWaves) lds_spoilt[i] = 0;
    __syncthreads();

    float top[RT], sum[RT];
    V4f out[RT][2 * NG];
    auto gather = [&] {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        lds_whole[rt * 64 * kWaves + later(threadIdx.x)] += sum[rt];
        sum[rt] = 0.f;
      }
    };
    auto step = [&](Tile8<NG>& t, int at, bool careful) {
      const bool masked = at < span.all_lo || at + kTile > span.all_hi;
      V4i p_hi[RT], p_lo[RT];
      float x[RT][8];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float key_unit = scalar(power_of((uint32_t)__builtin_amdgcn_readfirstlane((int)t.scale[u]) & 255u));
        V4f s[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt] = V4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NG; ++k) {
          const V4i key = operand_of<BF>(t.key[u][2 * k], t.key[u][2 * k + 1], BF ? key_unit : 1.f);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[rt] = multiply<!BF>(key, q[rt][k], s[rt]);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[rt][4 * u + i] = BF ? s[rt][i] : s[rt][i] * key_unit;
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        if (masked) {
          const int place = lds_place[rt * 16 + n];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int token = at + (i >> 2) * 16 + j * 4 + (i & 3);
            if ((uint32_t)(place - token) >= reach) x[rt][i] = -INFINITY;
          }
        }
        const float* const y = x[rt];
        const float most = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
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
        float weight[8], more = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          weight[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[i], unit, base));
          more = i == 0 ? weight[0] : more + weight[i];
        }
        sum[rt] += more;                                  // `more`: of the step alone, for the same reason as lds_whole
        parts_of<false>(weight, p_hi[rt], p_lo[rt]);
      }
      if (careful || at < span.first || at + kTile > span.hi) {
        // What no row sees may be anything: its codes become zeros.  In a careful pass those of values that are not numbers do too, and the rows that see
        // them are marked.
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int token = at + u * 16 + j * 4;
          uint32_t mask = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) mask |= token + i >= span.first && token + i < span.hi ? 255u << 8 * i : 0u;
#pragma unroll
          for (int w = 0; w < 2 * NG; ++w) {
            t.value[u][w] &= mask;
            const uint32_t odd = careful ? not_numbers(t.value[u][w]) : 0u;
            if (odd) {
              const int channel = w < 4 * FULL ? (w / 4) * 64 + n * 4 + w % 4 : FULL * 64 + n * 2 + (w - 4 * FULL);
#pragma unroll 1
              for (int i = 0; i < 4; ++i) {
                if (!(odd >> 8 * i & 1)) continue;
#pragma unroll 1
                for (int r = 0; r < R; ++r)
                  if ((uint32_t)(lds_place[r] - (token + i)) < reach) atomicOr(lds_spoilt + r * NG + (channel >> 5), 1u << (channel & 31));
              }
              t.value[u][w] &= ~(odd * 255u);
            }
          }
        }
      }
      const float unit0 = scalar(power_of((uint32_t)__builtin_amdgcn_readfirstlane((int)t.scale[0]) >> 8)), unit1 = scalar(power_of((uint32_t)__builtin_amdgcn_readfirstlane((int)t.scale[1]) >> 8));
#pragma unroll
      for (int w = 0; w < 2 * NG; ++w) {
        const V4i v = {pair_of<true>(t.value[0][w], unit0, false), pair_of<true>(t.value[0][w], unit0, true), pair_of<true>(t.value[1][w], unit1, false),
                       pair_of<true>(t.value[1][w], unit1, true)};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          out[rt][w] = multiply<false>(v, p_lo[rt], out[rt][w]);
          out[rt][w] = multiply<false>(v, p_hi[rt], out[rt][w]);
        }
      }
    };

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
        auto ahead = [&](Tile8<NG>& t, int next) {
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
      // A value that is not a number reaches every row of its tile, with weight 0 where it is not seen: then the tokens are gone through again, carefully.
      // (A row's own NaN, of its query or a key that it sees, gets here too, and costs time alone; so do infinities of both signs.)
      float all[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) all[i] += out[rt][c][i];
      const float one_of = (all[0] + all[1]) + (all[2] + all[3]);
      if (!__any(one_of != one_of)) break;
    }

    // What the results need of the arguments is read again here, rather than kept in registers through the steps.
    typedef const __attribute__((address_space(4))) Launch8* Launch8Ptr;
    Launch8Ptr e = (Launch8Ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(e));
    const int thread = later(threadIdx.x), row16 = thread & 15, quad = thread >> 4 & 3;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float total_of_row = sum[rt] + lds_whole[rt * 64 * kWaves + thread];
      total_of_row += __shfl_xor(total_of_row, 16);
      total_of_row += __shfl_xor(total_of_row, 32);
      if (bad) total_of_row = NAN;
      float* const to = lds + (wave * 16 + row16) * LD;
#pragma unroll
      for (int i = 0; i < FULL; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) *reinterpret_cast<V4f*>(to + i * 64 + quad * 16 + r * 4) = V4f{out[rt][4 * i][r], out[rt][4 * i + 1][r], out[rt][4 * i + 2][r], out[rt][4 * i + 3][r]};
      if (REST) {
#pragma unroll
        for (int r = 0; r < 4; r += 2)
          *reinterpret_cast<V4f*>(to + FULL * 64 + quad * 8 + r * 2) = V4f{out[rt][4 * FULL][r], out[rt][4 * FULL + 1][r], out[rt][4 * FULL][r + 1], out[rt][4 * FULL + 1][r + 1]};
      }
      if (quad == 0) {
        lds_max[wave * 16 + row16] = top[rt] * unit;
        lds_sum[wave * 16 + row16] = total_of_row;
      }
      __syncthreads();
      for (int item = thread; item < 4 * D; item += 64 * kWaves) {
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
        const uint32_t spoilt = lds_spoilt[(rt * 16 + r) * NG + (channel >> 5)] >> (channel & 31);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = spoilt >> i & 1 ? NAN : o[i];
        const int query = rows.query_of(a, g, row), h = head * e->a.shared + row - query * e->a.shared;
        const int64_t token = seq.first + query;
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

// Two tiles of rows share the decoded values where there are more rows than one has.
int row_tiles(const KvAttention& a) { return (int64_t)a.most_queries * a.shared > 16 && a.pool.dim <= 128 ? 2 : 1; }

// Rows of a sequence up to which the kernel for few rows takes a call; beyond, the estimates decide.
constexpr int kFewRows = 64;

struct Dealt {
  int64_t splits;
  double time;
};
// How many parts the tokens of a sequence are dealt out to: the number with the shortest estimate, in microseconds.  A workgroup goes on by 128 tokens in the
// time that it takes alone, or that the workgroups of a compute unit take for one each where that is longer: from memory (5.6 TB/s, once for all rows of a sequence)
// or on the vector units and matrix cores.  Workgroups take turns where more of them come than fit.  Joining costs a launch and the sums' way through memory.
// Constants from 1828 timings, of 1 to 64 sequences of 1024 to 131072 tokens, 1 to 1024 rows on a key/value head of 64, 128 and 256 channels, with 1 to 128
// parts, by both kernels where there are more than 16 rows; what it chooses took 0.7 % longer than the best of these in the mean, 20 % at worst.  (Wide heads by the kernel for many
// rows: from 16 sequences of 4096 tokens with 256 and 512 rows.)
Dealt deal(const KvAttention& a, bool many, int64_t row_blocks, int64_t units) {
  static constexpr int kTry[] = {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256};
  static_assert(kMostSplits == 256, "the last one tried");
  const int64_t others = (int64_t)a.batch * a.pool.heads * row_blocks;
  const double cus = device_cu_count(), rows = (double)a.tokens * a.heads, width = a.pool.dim / 128.0;
  const bool two = row_tiles(a) == 2;
  const double begin = many ? 1.9 : 2.8, alone = many ? 4.3 * (0.4 + 0.6 * width) : (two ? 1.3 : 1.1) * (0.5 + 0.5 * width);
  const double memory = 128.0 * a.pool.dim * 2 * cus / 5.6e6 / (double)row_blocks, work = many && width > 1.0 ? 0.65 * alone : (many ? 0.97 : two ? 0.96 : 1.03) * (0.3 + 0.7 * width);
  const double share = many ? work : std::max(memory, work), room = many ? (a.pool.dim <= 192 ? 2 : 1) : a.pool.dim <= 64 ? 3 : a.pool.dim <= 128 ? 2 : 1;
  auto time = [&](int64_t splits) {
    const double groups = (double)(others * splits) / cus, steps = (double)((units + splits - 1) / splits), busy = std::min(std::ceil(groups), room);
    const double turns = groups <= 4.0 * room ? std::ceil(groups / room) : groups / room + 0.5;
    return turns * (begin + steps * std::max(alone, busy * share)) + (splits > 1 ? 3.7 + rows * (double)splits * (a.pool.dim + 2) * 8.0 / 3.7e6 : 0.0);
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
  auto block_rows = [&](bool many) { return many ? 32 * kWaves : 16 * row_tiles(a); };
  auto dealt = [&](bool many) { return deal(a, many, std::max<int64_t>(1, (most_rows + block_rows(many) - 1) / block_rows(many)), (longest + unit - 1) / unit); };
  const Tuning& knobs = tuning();
  bool many = knobs.attention_kernel == 2;
  Dealt best = dealt(many);
  if (knobs.attention_kernel == 0 && most_rows > kFewRows) {
    const Dealt other = dealt(true);
    if (other.time < best.time) best = other, many = true;
  }
  if (knobs.attention_parts > 0 && may_join(a)) best.splits = std::min({knobs.attention_parts, (longest + unit - 1) / unit, (int64_t)kMostSplits});
  g.rows = block_rows(many);
  const int64_t splits = best.splits, row_blocks = (most_rows + g.rows - 1) / g.rows, others = (int64_t)a.batch * a.pool.heads * row_blocks;
  g.chunk = (longest + splits * unit - 1) / (splits * unit) * unit;
  g.splits = (int32_t)((longest + g.chunk - 1) / g.chunk);
  g.row_blocks = (int32_t)std::min(row_blocks, kMostGrid / g.splits);      // of a launch: a workgroup goes on to others
  g.ordered = a.batch > 1 && a.batch <= 64 && others * g.splits > 3 * (int64_t)device_cu_count();
  return g;
}

template <int NG, bool BF, int RT>
int launch_of(const Launch8& l, hipStream_t stream) {
  constexpr int lds = 4 * (kWaves * 16 * (32 * NG + 4) + 2 * kWaves * 16 + 16 * RT + 16 * RT * NG + RT * 64 * kWaves);
  const KvAttention& a = l.a;
  if (lds > 64 * 1024) MACKO_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&attention8_kernel<NG, BF, RT>), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  hipLaunchKernelGGL((attention8_kernel<NG, BF, RT>), dim3((unsigned)a.pool.heads, (unsigned)a.batch, (unsigned)(l.g.row_blocks * l.g.splits)), dim3(64 * kWaves), lds, stream, l);
  MACKO_HIP_TRY(hipGetLastError());
  return MACKO_OK;
}

template <int NG, bool BF>
int launch_type(const Launch8& l, hipStream_t stream) {
  if constexpr (NG <= 4) {
    if (row_tiles(l.a) == 2) return launch_of<NG, BF, 2>(l, stream);
  }
  return launch_of<NG, BF, 1>(l, stream);
}

template <int NG>
int launch_dim(const Launch8& l, hipStream_t stream) {
  return l.a.type == MACKO_BF16 ? launch_type<NG, true>(l, stream) : launch_type<NG, false>(l, stream);
}

int launch_width(const Launch8& l, hipStream_t stream) {
  switch (l.a.pool.dim / 32) {
    case 1: return launch_dim<1>(l, stream);
    case 2: return launch_dim<2>(l, stream);
    case 3: return launch_dim<3>(l, stream);
    case 4: return launch_dim<4>(l, stream);
    case 5: return launch_dim<5>(l, stream);
    case 6: return launch_dim<6>(l, stream);
    case 7: return launch_dim<7>(l, stream);
    case 8: return launch_dim<8>(l, stream);
  }
  return MACKO_E_UNSUPPORTED;
}

}  // namespace

int64_t kv8_attention_workspace(const KvAttention& a) {
  if (a.tokens == 0 || a.batch == 0) return 0;
  const Grid g = grid_of(a);
  return g.splits > 1 ? a.tokens * a.heads * (g.splits * (int64_t)(a.pool.dim + 2) + 1) : 0;
}

int launch_kv8_attention(const Kv8Attention& a, float* workspace, hipStream_t stream) {
  Launch8 l{a.a, grid_of(a.a), a.scales};
  l.g.parts = workspace;
  const int status = l.g.rows >= 64 ? launch_kv8_rows(l, stream) : launch_width(l, stream);
  return status == MACKO_OK && l.g.splits > 1 ? launch_join(a.a, l.g, stream) : status;
}

}  // namespace macko
