// Causal attention of packed sequences over keys and values in 16 bits (macko_prompt_attention), by the kernel of macko_rows.h.
#include <cmath>

#include "macko_rows.h"

namespace macko {
namespace {

template <int NG, bool BF, int WAVES>
int launch_waves(LaunchRows& l, int64_t blocks, hipStream_t stream) {
  l.g.rows = 32 * WAVES;
  l.g.row_blocks = (int32_t)blocks;
  return launch_rows<NG, BF, false, WAVES>(l, dim3((unsigned)(blocks * l.a.pool.heads)), stream);
}

// Heads of 96 and 128 channels: eight wavefronts, which bring a step's keys and values for 256 rows, where those blocks fill the device twice and rows see some 512 tokens
// in the mean, else four, which waste less at both ends of what a block sees.  128 channels, 32 heads on 8: bf16, one sequence of 4096 tokens 151 us, 174 with four;
// of 8192 543 and 610, of 1024 tokens 39 and 36; fp16, 12800 tokens in sequences of 2048 274 us, 292 with four; of 1024 181 and 180; of 512 140 and 128; of 64 101 and 79.
template <int NG, bool BF>
int launch_type(LaunchRows& l, hipStream_t stream) {
  const int64_t rows = l.a.tokens * l.a.shared;
  if constexpr (NG == 3 || NG == 4) {
    const int64_t blocks = (rows + 255) / 256;
    const int64_t seen = l.a.window ? std::min<int64_t>(l.a.window, l.a.longest / 2) : l.a.longest / 2;
    if (seen >= 512 && blocks * l.a.pool.heads >= 2 * (int64_t)device_cu_count()) return launch_waves<NG, BF, 8>(l, blocks, stream);
  }
  return launch_waves<NG, BF, 4>(l, (rows + 127) / 128, stream);
}

template <int NG>
int launch_dim(LaunchRows& l, hipStream_t stream) {
  return l.a.type == MACKO_BF16 ? launch_type<NG, true>(l, stream) : launch_type<NG, false>(l, stream);
}

}  // namespace
}  // namespace macko

extern "C" {

using namespace macko;

int macko_prompt_attention(const macko_prompt_args_t* g, void* stream) {
  if (!g || g->tokens < 0 || g->heads < 1 || g->kv_heads < 1 || g->batch < 0 || g->window < 0 || g->longest < 0 || (g->type != MACKO_FP16 && g->type != MACKO_BF16) ||
      g->heads % g->kv_heads != 0 || !std::isfinite(g->scale))
    return MACKO_E_INVALID_ARG;
  if (int st = check_head_dim(g->head_dim)) return st;
  if (g->tokens > INT32_MAX || g->heads > 65536 || g->tokens * g->heads > kMostTokens || g->heads / g->kv_heads > 32768) return MACKO_E_UNSUPPORTED;
  if (g->tokens == 0 || (g->start_dev && g->batch == 0)) return MACKO_OK;
  if (!heads_fine(g->q_dev, g->q_token, g->q_head) || !heads_fine(g->k_dev, g->k_token, g->k_head) || !heads_fine(g->v_dev, g->v_token, g->v_head) ||
      !heads_fine(g->out_dev, g->out_token, g->out_head) || !aligned_to(g->start_dev, 4) || !aligned_to(g->sums_dev, 4))
    return MACKO_E_INVALID_ARG;
  LaunchRows l{};
  KvAttention& a = l.a;
  a.pool.heads = g->kv_heads, a.pool.dim = g->head_dim;
  a.q = static_cast<const uint8_t*>(g->q_dev), a.out = static_cast<uint8_t*>(g->out_dev), a.sums = g->sums_dev;
  a.q_token = g->q_token, a.q_head = g->q_head, a.out_token = g->out_token, a.out_head = g->out_head;
  a.start = g->start_dev, a.batch = g->batch;
  a.heads = g->heads, a.shared = g->heads / g->kv_heads, a.window = g->window;
  a.scale = g->scale, a.tokens = g->tokens, a.type = g->type;
  a.longest = g->start_dev ? std::min(g->longest, g->tokens) : g->tokens;
  l.k = static_cast<const uint16_t*>(g->k_dev), l.k_token = g->k_token, l.k_head = g->k_head;
  l.v = static_cast<const uint16_t*>(g->v_dev), l.v_token = g->v_token, l.v_head = g->v_head;
  l.g.splits = 1;
  l.g.shared_inverse = a.shared == 1 ? 0u : (uint32_t)(((uint64_t{1} << 32) + a.shared - 1) / a.shared);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  switch (g->head_dim / 32) {
    case 1: return launch_dim<1>(l, s);
    case 2: return launch_dim<2>(l, s);
    case 3: return launch_dim<3>(l, s);
    case 4: return launch_dim<4>(l, s);
    case 5: return launch_dim<5>(l, s);
    case 6: return launch_dim<6>(l, s);
    case 7: return launch_dim<7>(l, s);
    case 8: return launch_dim<8>(l, s);
  }
  return MACKO_E_UNSUPPORTED;
}

}  // extern "C"
