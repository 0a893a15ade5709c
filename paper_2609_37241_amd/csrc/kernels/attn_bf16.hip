// Attention over pages on the matrix cores, bfloat16.
#include "../internal.h"
#include "attn.h"

namespace tri {
using namespace dev;

template <int HDP>
__global__ __launch_bounds__(64 * rows_waves(HDP), 1) void k_pa_rows_bf16(PagedArgs a) {
  body_pa_rows<kBF16, HDP>(a);
}

template <int HDP>
__global__ __launch_bounds__(256, HDP == 256 ? 1 : 2) void k_pa_tile_bf16(PagedArgs a) {
  body_pa_tile<kBF16, HDP, 1>(a);
}

template <int HDP>
__global__ __launch_bounds__(512, 1) void k_pa_pair_bf16(PagedArgs a) {
  body_pa_tile<kBF16, HDP, 2>(a);
}

// hdp: the head size rounded up to 64, 128 or 256 (PA_PAIR: to 64 or 128).
const void *attn_kernel_bf16(int32_t variant, int32_t hdp) {
  const void *rows[3] = {reinterpret_cast<const void *>(&k_pa_rows_bf16<64>),
                         reinterpret_cast<const void *>(&k_pa_rows_bf16<128>),
                         reinterpret_cast<const void *>(&k_pa_rows_bf16<256>)};
  const void *tile[3] = {reinterpret_cast<const void *>(&k_pa_tile_bf16<64>),
                         reinterpret_cast<const void *>(&k_pa_tile_bf16<128>),
                         reinterpret_cast<const void *>(&k_pa_tile_bf16<256>)};
  const void *pair[3] = {reinterpret_cast<const void *>(&k_pa_pair_bf16<64>),
                         reinterpret_cast<const void *>(&k_pa_pair_bf16<128>), nullptr};
  if (hdp != 64 && hdp != 128 && hdp != 256) return nullptr;
  const int i = hdp == 64 ? 0 : hdp == 128 ? 1 : 2;
  switch (variant) {
    case PA_ROWS: return rows[i];
    case PA_TILE: return tile[i];
    case PA_PAIR: return pair[i];
    default: return nullptr;
  }
}

}  // namespace tri
