// Attention over the 4-bit cache for many rows of a sequence (a part of a prompt): there the vector units and the matrix cores are what bounds a
// step, not memory.  The four wavefronts of a workgroup have rows of their own and go along the tokens together, 64 at a time:
//   values   are decoded once for all of them, a quarter by each, into LDS, as the operand of the matrix instruction: a lane's 8 tokens of one
//            channel lie together.  The steps are staggered: while step t is multiplied, t + 1 is decoded and t + 2 is on its way from memory.
//            In bf16, which holds them exactly; for results in bf16 alone in fp16, which does so for factors from 2^-19 to 2^12.
//   weights  are two bf16 parts (16 bits).  For results in bf16 alone, whose sums nobody asks for, they are one fp16 part: 11 bits from 2^-24 of a row's
//            maximum on, and below that 2^-35 of it at most too much or too little.  Rows for which that may be too coarse, and factors beyond fp16, are found
//            behind the steps, and their block is done again in bf16.  One fp16 part takes 303 us where two bf16 parts take 386 (the case below).
//   scores   as in macko_kv_attention.hip: keys as they lie in memory.
//   sums     of the weights come from the matrix cores too (a row of ones), 512 tokens at a time; those are added up with what rounding leaves out.
// 64 tokens, because their keys and a step's scores are what the registers hold of two tiles of rows for two wavefronts on a SIMD; that is what hides one
// wavefront's softmax behind another's products, as far as it is hidden.  1024 queries on each of 2 sequences of 8192 tokens, 32 heads on 8 of 128 channels, bf16:
// 303 us, 850 TFLOP/s of the 1340 to 1385 that a product of 8192 x 8192 matrices reaches.  Of the 6200 cycles in which a SIMD does a step of each of its
// wavefronts the matrix core is busy for 2180 (a score takes two parts of its query, at twice the rate of 16 bits) and the vector unit for 2640
// (profiles/kv_prompt_kernel_counters.txt), so that what is left is their overlap.  Tried for that, without gain: priorities of wavefronts around either half (1.5 % here, 9 % slower with 256 channels), all
// of a step's scores before its first weight (256 registers), loads a step earlier, eight wavefronts to a workgroup, three workgroups for narrow heads.
#include "macko_kv_attention.h"

namespace macko {
namespace {

constexpr int kStep = 64, kBlocks = kStep / 16, kWide = 1, kNan = 2;
// Weights in fp16, which goes from 2^-24 to 2^16: the running maximum is at 2^10, and a weight may be 2^5 times that before it moves (2^12 and 2^3: up to 4 % slower).
constexpr float kHalfTop = 10.f, kHalfLift = 5.f;
constexpr float kHalfFar = 0x1.8p14f;                     // the largest value that goes to fp16

// Wavefronts on a SIMD: 64 channels leave room for a third (4096 queries of 2 sequences, bf16: 211 us, 280 with two).
constexpr int prompt_waves(int ng, bool bf) { return ng == 2 && bf ? 3 : 2; }

template <int NG, bool BF, int RT>
__global__ __launch_bounds__(64 * kWaves, prompt_waves(NG, BF)) void prompt_kernel(const Launch args) {
  const KvAttention& a = args.a;
  const Grid& g = args.g;
  constexpr int D = 32 * NG, NK = (NG + 3) / 4, NP = BF ? 2 : 3, R = 16 * RT * kWaves;
  constexpr int SHARE = NG <= 2 ? 4 / NG : 1, NI = (NP + SHARE - 1) / SHARE;      // parts of a query that one instruction takes; instructions
  extern __shared__ __align__(16) V4i lds[];             // [2][2][2 NG][64]: 8 tokens of one channel, for a step, 32 of its tokens, 16 channels and a lane
  uint32_t* const outside = reinterpret_cast<uint32_t*>(lds + 2 * 2 * 2 * NG * 64);     // [2][kWaves]: what look_over has found in a step's values
  uint32_t* const lds_spoilt = outside + 2 * kWaves;     // [kWaves][RT][16]: groups in which a row sees what is not a number

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x, split = g.splits == 1 ? 0 : g.row_blocks == 1 ? (int)blockIdx.z : (int)blockIdx.z / g.row_blocks, row_block = (int)blockIdx.z - split * g.row_blocks;
  int b = blockIdx.y;
  if (g.ordered) b = nth_longest(a, b, threadIdx.x & 63);
  const Sequence seq = sequence_of(a, b);
  const int32_t* const table = a.tables + b * a.table_stride;
  const int64_t piece = kv_piece_bytes(int64_t{1} << a.pool.page_bits, D), page_stride = piece * a.pool.heads;
  const uint8_t* const pool = a.pool.data + head * piece;
  const int page_size = 1 << a.pool.page_bits;
  const float unit = a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.4426950408889634f, sign = a.scale < 0.f ? -1.f : a.scale == 0.f ? 0.f : 1.f;
  const uint32_t reach = a.window ? (uint32_t)a.window : 0x7FFFFFFFu;

  bool in_half = BF && !a.sums;                           // the way that a block of rows is done in
  // The last rows see most: they start first, and what is left for the end is short (4096 rows of 32 heads 299 to 247 us).
  for (int first_row = (g.row_blocks - 1 - row_block) * R; first_row < seq.rows;) {
    const Rows rows = rows_of(a, first_row);
    const Span span = span_of(a, g, seq, rows);
    if (split >= span.used) {
      first_row += g.row_blocks * R;
      continue;
    }
    const int lane = later(threadIdx.x) & 63, n = lane & 15, j = lane >> 4, group = SHARE > 1 ? j % NG : j;
    const int begin = span.lo + split * span.chunk, end = span.hi - begin > span.chunk ? begin + span.chunk : span.hi;
    const int last_block = (end - 1) >> 4;
    bool bad = end > begin && (a.table_width == 0 || a.pool.pages == 0);
    const bool any = end > begin && !bad;

    V4i key[kBlocks][NK];
    int key_byte[kBlocks][NK];
    uint32_t value[NG], value_byte[NG];                  // of the wavefront's own block of a step
    // A lane has the page of one block of 16 steps; they are looked up anew, half of them again, every 8.
    int pages = 0;
    auto entry = [&](int at) { return table[min(min((at >> 4) + lane, last_block) >> (a.pool.page_bits - 4), a.table_width - 1)]; };
    auto take = [&](int at, int page) {
      const bool fine = min((at >> 4) + lane, last_block) >> (a.pool.page_bits - 4) < a.table_width && page >= 0 && page < a.pool.pages;
      bad = bad || __any(!fine);
      pages = fine ? page : 0;
    };
    // Codes of a block, and how far behind them its factors lie
    auto codes_of = [&](int at, int u, int slot, int64_t& bytes) {
      const int in_page = (min((at >> 4) + u, last_block) << 4) & (page_size - 1);
      bytes = page_size * D - in_page * (D / 2 - NG);
      return pool + (int64_t)__builtin_amdgcn_readlane(pages, slot * kBlocks + u) * page_stride + in_page * (D / 2);
    };
    auto load_keys = [&](int at, int slot) {
#pragma unroll
      for (int u = 0; u < kBlocks; ++u) {
        int64_t bytes;
        const uint8_t* const codes = codes_of(at, u, slot, bytes);
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
          key[u][kk] = V4i{0, 0, 0, 0};
          key_byte[u][kk] = 0;
          if (SHARE > 1 || kk * 4 + j < NG) {
            key[u][kk] = *reinterpret_cast<const V4i*>(codes + (uint32_t)(n * (D / 2) + group * 16) + kk * 64);
            key_byte[u][kk] = (codes + bytes)[(uint32_t)(n * NG + group) + kk * 4];
          }
        }
      }
    };
    auto load_values = [&](int at, int slot) {
      int64_t bytes;
      const uint8_t* const codes = codes_of(at, wave, slot, bytes);
      const uint32_t* const v = reinterpret_cast<const uint32_t*>(codes + page_size * (D / 2) + (uint32_t)((j * 16 + n) * (4 * NG)));
      const uint32_t* const vb = reinterpret_cast<const uint32_t*>(codes + bytes + page_size * NG + (uint32_t)(j * (4 * NG)));
#pragma unroll
      for (int w = 0; w < NG; ++w) {
        value[w] = v[w];
        value_byte[w] = vb[w];
      }
    };
    // What there is to see to in the wavefront's values of a step, of tokens that a row may see: kWide, factors beyond 2^-19 to 2^12 (bytes 108 to 139; 0 is
    // a group of zeros), kNan, values that may not be numbers.
    auto look_over = [&](int at, int parity) {
      uint32_t far = 0;                                   // each byte 0 to 31 once 108 is taken off (one below borrows, and shows that itself)
#pragma unroll
      for (int w = 0; w < NG; ++w) far |= value_byte[w] - 0x6C6C6C6Cu;
      int what = 0;
      if (__any((far & 0xE0E0E0E0u) != 0)) {
        bool wide = false, nan = false;
#pragma unroll
        for (int k = 0; k < 4 * NG; ++k) {
          const uint32_t byte = value_byte[k >> 2] >> 8 * (k & 3) & 255u;
          const int token = at + wave * 16 + j * 4 + k / NG;
          const bool counts = token >= span.first && token < end;
          nan = nan || (counts && byte >= kNoNumber);
          wide = wide || (counts && byte < kNoNumber && byte > 139u) || (counts && byte < 108u && byte != 0u);
        }
        what = (__any(wide) ? kWide : 0) | (__any(nan) ? kNan : 0);
      }
      if (lane == 0) outside[parity * kWaves + wave] = what;
    };
    auto found = [&](int parity) {
      const uint32_t* const o = outside + parity * kWaves;
      return __builtin_amdgcn_readfirstlane((int)(o[0] | o[1] | o[2] | o[3]));
    };
    auto decode = [&](int at, int parity, int what, auto half) {
      constexpr bool HALF = decltype(half)::value;
      if (at < span.first || at + kStep > end || (what & kNan)) {      // what no row sees may be anything, values that are not numbers are left out
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int token = at + wave * 16 + j * 4 + k;
#pragma unroll
          for (int i = 0; i < NG; ++i) {
            const int byte = k * NG + i, shift = 8 * (byte & 3);
            if (token < span.first || token >= end || (value_byte[byte >> 2] >> shift & 255u) >= kNoNumber) value_byte[byte >> 2] &= ~(255u << shift);
          }
        }
      }
      uint2* const to = reinterpret_cast<uint2*>(lds + (parity * 2 + (wave >> 1)) * 2 * NG * 64 + lane) + (wave & 1);
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        uint32_t v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = decode_at<HALF>(value[(k * NG + i) >> 2], value_byte[(k * NG + i) >> 2], (k * NG + i) & 3);
        to[(2 * i) * 128] = uint2{__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u)};
        to[(2 * i + 1) * 128] = uint2{__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u)};
      }
    };

    // the rows of this lane
    int place[RT];
    V8i q[RT][NK][NI];
    int q_byte[RT][NK];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = first_row + (wave * RT + rt) * 16 + n, query = rows.query_of(a, g, row);
      const bool there = row < seq.rows;
      place[rt] = there ? seq.length - seq.queries + query : -1;
      const uint16_t* const src = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(seq.first + query) * a.q_token + (int64_t)(head * a.shared + row - query * a.shared) * a.q_head;
      V8i part[NK][NP];
      load_queries<NG, BF>(src, there, sign, n, j, part, q_byte[rt]);
      if constexpr (SHARE == 1) {
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
#pragma unroll
          for (int p = 0; p < NP; ++p) q[rt][kk][p] = part[kk][p];
      } else {
        // Narrow heads leave room: an instruction takes the same keys against SHARE parts, channel 0 of part p at p D.
        const uint32_t bytes = (uint32_t)__shfl(q_byte[rt][0], n + 16 * group);
        const int p = j / NG;
        q_byte[rt][0] = (int)((bytes >> 8 * min(p, NP - 1) & 255u) | (bytes >> 16 & 255u) << 8);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if (NG == 1) {
            const int second = __shfl(part[0][1][w], lane & 31);
            q[rt][0][0][w] = j < 2 ? part[0][0][w] : second;
            q[rt][0][0][4 + w] = NP == 3 && j < 2 ? part[0][NP - 1][w] : 0;
          } else {
            q[rt][0][0][w] = part[0][0][w];
            q[rt][0][0][4 + w] = part[0][1][w];
            if (NP == 3) {
              q[rt][0][NI - 1][w] = part[0][2 % NP][w];
              q[rt][0][NI - 1][4 + w] = 0;
            }
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);                  // one tile of rows at a time, or the registers do not hold what lies between
      if (lane < 16) lds_spoilt[(wave * RT + rt) * 16 + lane] = 0;
    }

    // Of a row: what its scores are lifted by, and how large they may then be, in powers of two; nothing seen yet: 0 and -infinity.
    float base[RT], limit[RT];
    V4f out[RT][2 * NG], total[RT];                      // the sum of the weights since it last went into `whole`, the same in every row
    // The sum up to there and what its roundings left out: a token that is far ahead of very many others would lose them, step by step.
    float whole[RT], rest[RT];
    auto gather = [&] {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float more = total[rt][0], sum = whole[rt] + more, by = sum - whole[rt];
        rest[rt] += (whole[rt] - (sum - by)) + (more - by);
        whole[rt] = sum;
        total[rt] = V4f{0.f, 0.f, 0.f, 0.f};
      }
    };
    // All steps; true: in fp16, which did not hold all values.
    auto go = [&](auto half) {
      constexpr bool HALF = decltype(half)::value;
      constexpr float kTop = HALF ? kHalfTop : 0.f, kMost = kTop + (HALF ? kHalfLift : kLift);      // where the running maximum is put, and where it moves
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        base[rt] = 0.f;
        limit[rt] = -INFINITY;
        whole[rt] = rest[rt] = 0.f;
        total[rt] = V4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c) out[rt][c] = V4f{0.f, 0.f, 0.f, 0.f};
      }
      if (!any) return false;
      // what is loaded ahead of the last step is its last block again
      take(begin, entry(begin));
      load_values(begin, 0);
      load_keys(begin, 0);
      look_over(begin, 0);
      __syncthreads();
      int now = found(0);
      int all = now;
      decode(begin, 0, now, half);
      load_values(begin + kStep, 1);
      look_over(begin + kStep, 1);
      __syncthreads();
      int ahead = 0;                                      // table entries on their way
      for (int at = begin, parity = 0, slot = 0; at < end; at += kStep, parity ^= 1) {
        const bool more = at + kStep < end;
        const int next = more ? found(parity ^ 1) : 0;
        all |= next;
        if (more) decode(at + kStep, parity ^ 1, next, half);
        if (now & kNan) {                                 // values that are not numbers have been left out: the rows that see them are marked
#pragma unroll 1
          for (int u = 0; u < kBlocks; ++u) {
            const int in_page = (min((at >> 4) + u, last_block) << 4) & (page_size - 1);
            const uint8_t* const piece_of = pool + (int64_t)__builtin_amdgcn_readlane(pages, slot * kBlocks + u) * page_stride;
            const uint8_t* const vb = piece_of + page_size * (D + NG) + (in_page + j * 4) * NG;
#pragma unroll 1
            for (int k = 0; k < 4 * NG; ++k) {
              const int token = at + u * 16 + j * 4 + k / NG;
              if (vb[k] < kNoNumber || token >= end) continue;
#pragma unroll
              for (int rt = 0; rt < RT; ++rt)
                if ((uint32_t)(place[rt] - token) < reach) atomicOr(lds_spoilt + (wave * RT + rt) * 16 + n, 1u << k % NG);
            }
          }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {                     // 32 tokens at a time: weights, then products
          V4i p_hi[RT], p_lo[RT];
          float scores[RT][8];                            // of all tiles of rows first: the matrix cores are at the next one's while one is weighed
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              V4f sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int kk = 0; kk < NK; ++kk) {
                const V4i k4 = key[2 * s + u][kk];
                const V8i k8 = {k4[0], k4[1], k4[2], k4[3], 0, 0, 0, 0};
                if (NI == 3) sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k8, q[rt][kk][NI - 1], sum, 4, 0, 0, key_byte[2 * s + u][kk], 2, q_byte[rt][kk]);
                if (NI >= 2) sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k8, q[rt][kk][NI >= 2 ? 1 : 0], sum, 4, 0, 0, key_byte[2 * s + u][kk], 1, q_byte[rt][kk]);
                sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k8, q[rt][kk][0], sum, 4, 0, 0, key_byte[2 * s + u][kk], 0, q_byte[rt][kk]);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) scores[rt][4 * u + i] = sum[i];
            }
          }
          if (s == 1) {                                   // in the registers of this step's, and in those that the next one's values have left
            if (more) load_keys(at + kStep, slot + 1);
            if (at + 2 * kStep < end) load_values(at + 2 * kStep, slot + 2);
          }
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            float(&x)[8] = scores[rt];
            if (at < span.all_lo || at + kStep > span.all_hi) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int token = at + s * 32 + (i >> 2) * 16 + j * 4 + (i & 3);
                if ((uint32_t)(place[rt] - token) >= reach) x[i] = -INFINITY;
              }
            }
            float y[8];                                   // against the running maximum as it was
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(x[i], unit, base[rt]);
            const float most = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
            if (__any(most > limit[rt])) {
              float by = fmaxf(most, __shfl_xor(most, 16));
              by = fmaxf(by, __shfl_xor(by, 32));
              if (limit[rt] > -INFINITY) by = fmaxf(by, kTop);
              if (by > -INFINITY) {
                const float to = base[rt] - (by - kTop);
                by = limit[rt] > -INFINITY ? __builtin_amdgcn_exp2f(to - base[rt]) : 1.f;
                base[rt] = to;
                limit[rt] = kMost;
              } else {
                by = 1.f;
              }
              total[rt] *= by;
              whole[rt] *= by;
              rest[rt] *= by;
#pragma unroll
              for (int c = 0; c < 2 * NG; ++c) out[rt][c] *= by;
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(x[i], unit, base[rt]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_exp2f(y[i]);
            parts_of<HALF>(y, p_hi[rt], p_lo[rt]);
          }
          constexpr bool ONE = HALF && BF;
          const int one = HALF ? 0x3C003C00 : 0x3F803F80;
          const V4i ones = {one, one, one, one};
          const V4i* const from = lds + (parity * 2 + s) * 2 * NG * 64 + lane;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            if (!ONE) total[rt] = multiply<HALF>(ones, p_lo[rt], total[rt]);
            total[rt] = multiply<HALF>(ones, p_hi[rt], total[rt]);
          }
#pragma unroll
          for (int c = 0; c < 2 * NG; ++c) {
            const V4i v = from[c * 64];
#pragma unroll
            for (int rt = 0; rt < RT && !ONE; ++rt) out[rt][c] = multiply<HALF>(v, p_lo[rt], out[rt][c]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) out[rt][c] = multiply<HALF>(v, p_hi[rt], out[rt][c]);
          }
        }
        if (slot == 4) ahead = entry(at + 4 * kStep);
        now = next;
        look_over(at + 2 * kStep, parity);
        if (++slot == 8) {
          take(at + kStep, ahead);
          slot = 0;
          gather();
        }
        __syncthreads();
      }
      gather();
      return HALF && (all & kWide);
    };
    if (BF && in_half) {
      const bool wide = go(std::integral_constant<bool, BF>{});
      float least = wide ? -1.f : INFINITY;               // the largest result of a row that sees something, of the row where that is smallest
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float large = 0.f;
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) large = fmaxf(large, fabsf(out[rt][c][i]));
        large = fmaxf(large, __shfl_xor(large, 16));
        large = fmaxf(large, __shfl_xor(large, 32));
        if (whole[rt] > 0.f) least = fminf(least, large);
      }
      // A weight below fp16's normal numbers is off by 2^-25 at most.  Whether that, with no value larger than `far`, may come to more than half a unit in the
      // last place of a row's largest result, in any wavefront.
      auto left_out = [&](float far) {
        const bool much = __any(least < (float)(end - begin) * far * 0x1p-25f * 0x1p9f);
        if (lane == 0) outside[wave] = much;
        __syncthreads();
        return found(0) != 0;
      };
      // The largest magnitude that a value of [span.first, end) can have by the factors of all groups.
      auto largest_value = [&] {
        uint32_t top = 0;
#pragma unroll 1
        for (int block = (begin >> 4) + wave * 64 + lane; block <= last_block; block += 64 * kWaves) {
          const int index = block >> (a.pool.page_bits - 4), page = table[min(index, a.table_width - 1)];
          const uint8_t* const piece_of = pool + (index < a.table_width && page >= 0 && page < a.pool.pages ? page : 0) * page_stride;
          const V4i* const vb = reinterpret_cast<const V4i*>(piece_of + page_size * (D + NG) + ((block << 4) & (page_size - 1)) * NG);
#pragma unroll 1
          for (int w = 0; w < NG; ++w) {
            const V4i word = vb[w];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const uint32_t byte = (uint32_t)word[k >> 2] >> 8 * (k & 3) & 255u;
              const int token = (block << 4) + (w * 16 + k) / NG;
              if (token >= span.first && token < end && byte < kNoNumber) top = max(top, byte);
            }
          }
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        if (lane == 0) outside[kWaves + wave] = top;
        __syncthreads();
        const uint32_t* const o = outside + kWaves;
        return 6.f * __builtin_bit_cast(float, max(max(o[0], o[1]), max(o[2], o[3])) << 23);
      };
      if (left_out(kHalfFar) && (wide || left_out(largest_value()))) {
        in_half = false;
        __syncthreads();
        continue;
      }
    } else {
      go(std::integral_constant<bool, false>{});
    }

    LaunchPtr e = (LaunchPtr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(e));
    const int thread = later(threadIdx.x), row16 = thread & 15, quad = thread >> 4 & 3;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = first_row + (wave * RT + rt) * 16 + row16;
      const uint32_t spoilt = lds_spoilt[(wave * RT + rt) * 16 + row16];
      if (row >= seq.rows) continue;
      const int query = rows.query_of(a, g, row), h = head * e->a.shared + row - query * e->a.shared;
      const int64_t token = seq.first + query;
      const float sum = bad ? NAN : whole[rt] + rest[rt], most = limit[rt] > -INFINITY ? -base[rt] : -INFINITY;
      const int64_t part = (token * e->a.heads + h) * e->g.splits + split;
      const float r = span.used > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
      uint16_t* const dst = reinterpret_cast<uint16_t*>(e->a.out) + token * e->a.out_token + h * e->a.out_head + quad * 4;
      float* const partial = e->g.parts + part * D + quad * 4;
#pragma unroll
      for (int c = 0; c < 2 * NG; ++c) {
        V4f o = out[rt][c] * r;
        if (spoilt >> (c / 2) & 1) o = V4f{NAN, NAN, NAN, NAN};
        if (span.used > 1) {
          *reinterpret_cast<V4f*>(partial + c * 16) = o;
        } else {
          typedef uint32_t Pair __attribute__((ext_vector_type(2), aligned(2)));
          *reinterpret_cast<Pair*>(dst + c * 16) = Pair{pack2<BF>(o[0], o[1]), pack2<BF>(o[2], o[3])};
        }
      }
      if (quad > 0) continue;
      if (span.used > 1) {
        float* const ms = e->g.parts + e->a.tokens * e->a.heads * e->g.splits * D + part * 2;
        ms[0] = most;
        ms[1] = sum;
        if (split == 0) used_splits(e->a, e->g)[token * e->a.heads + h] = span.used;
        continue;
      }
      if (e->g.splits > 1) used_splits(e->a, e->g)[token * e->a.heads + h] = 1;
      if (e->a.sums) e->a.sums[token * e->a.heads + h] = (most + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    }
    in_half = BF && !a.sums;
    first_row += g.row_blocks * R;
    __syncthreads();                                      // the marks are cleared for the next rows
  }
}

template <int NG, bool BF>
int launch_of(const KvAttention& a, const Grid& g, hipStream_t stream) {
  constexpr int RT = NG <= 4 ? 2 : 1, lds = 16 * 2 * 2 * 2 * NG * 64 + 4 * (2 * kWaves + kWaves * RT * 16);
  const void* const kernel = reinterpret_cast<const void*>(&prompt_kernel<NG, BF, RT>);
  if (lds > 64 * 1024) MACKO_HIP_TRY(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  hipLaunchKernelGGL((prompt_kernel<NG, BF, RT>), dim3((unsigned)a.pool.heads, (unsigned)a.batch, (unsigned)(g.row_blocks * g.splits)), dim3(64 * kWaves), lds, stream, Launch{a, g});
  MACKO_HIP_TRY(hipGetLastError());
  return MACKO_OK;
}

template <int NG>
int launch_dim(const KvAttention& a, const Grid& g, hipStream_t stream) {
  return a.type == MACKO_BF16 ? launch_of<NG, true>(a, g, stream) : launch_of<NG, false>(a, g, stream);
}

}  // namespace

int prompt_row_tiles(int dim) { return dim <= 128 ? 2 : 1; }

int launch_prompt(const KvAttention& a, const Grid& g, hipStream_t stream) {
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
