// Attention over the 8-bit cache for many rows of a sequence (a part of a prompt), by the kernel of macko_rows.h.
#include "macko_rows.h"

namespace macko {
namespace {

template <int NG, bool BF>
int launch_type(const Launch8& l8, hipStream_t stream) {
  LaunchRows l{};
  l.a = l8.a, l.g = l8.g, l.scales = l8.scales;
  const dim3 grid((unsigned)l.a.pool.heads, (unsigned)l.a.batch, (unsigned)(l.g.row_blocks * l.g.splits));
  return launch_rows<NG, BF, true, kWaves>(l, grid, stream);
}

template <int NG>
int launch_dim(const Launch8& l, hipStream_t stream) {
  return l.a.type == MACKO_BF16 ? launch_type<NG, true>(l, stream) : launch_type<NG, false>(l, stream);
}

}  // namespace

int launch_kv8_rows(const Launch8& l, hipStream_t stream) {
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

}  // namespace macko
