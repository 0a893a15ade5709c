// Attention over pages of 8-bit codes on the matrix cores, many rows per request: float32.
#include "../internal.h"
#include "attn_q8.h"

namespace tri {
using namespace dev;

template <int CT, int HDP>
__global__ __launch_bounds__(256, 1) void k_pa8_tile_f32(PagedQ8Args a) {
  body_pa8_tile<kF32, CT, HDP, 1>(a);
}

namespace {
template <int CT>
const void *kernel(int32_t hdp) {
  switch (hdp) {
    case 64: return reinterpret_cast<const void *>(&k_pa8_tile_f32<CT, 64>);
    case 128: return reinterpret_cast<const void *>(&k_pa8_tile_f32<CT, 128>);
    case 256: return reinterpret_cast<const void *>(&k_pa8_tile_f32<CT, 256>);
    default: return nullptr;
  }
}
}  // namespace

// As attn_q8_tile_bf16.
const void *attn_q8_tile_f32(int32_t code, int32_t hdp) {
  return code == TRI_E4M3 ? kernel<kE4M3>(hdp) : kernel<kInt8>(hdp);
}

}  // namespace tri
