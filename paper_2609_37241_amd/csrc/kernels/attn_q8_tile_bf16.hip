// Attention over pages of 8-bit codes on the matrix cores, many rows per request: bfloat16.
#include "../internal.h"
#include "attn_q8.h"

namespace tri {
using namespace dev;

template <int CT, int HDP>
__global__ __launch_bounds__(256, HDP == 256 ? 1 : 2) void k_pa8_tile_bf16(PagedQ8Args a) {
  body_pa8_tile<kBF16, CT, HDP, 1>(a);
}

template <int CT, int HDP>
__global__ __launch_bounds__(512, 1) void k_pa8_pair_bf16(PagedQ8Args a) {
  body_pa8_tile<kBF16, CT, HDP, 2>(a);
}

namespace {
template <class F>
const void *sym(F *f) {
  return reinterpret_cast<const void *>(f);
}

template <int CT>
const void *kernel(bool pair, int32_t hdp) {
  switch (hdp) {
    case 64: return pair ? sym(&k_pa8_pair_bf16<CT, 64>) : sym(&k_pa8_tile_bf16<CT, 64>);
    case 128: return pair ? sym(&k_pa8_pair_bf16<CT, 128>) : sym(&k_pa8_tile_bf16<CT, 128>);
    case 256: return pair ? nullptr : sym(&k_pa8_tile_bf16<CT, 256>);
    default: return nullptr;
  }
}
}  // namespace

// hdp: the head size rounded up to 64, 128 or 256 (pairs: to 64 or 128).
const void *attn_q8_tile_bf16(bool pair, int32_t code, int32_t hdp) {
  return code == TRI_E4M3 ? kernel<kE4M3>(pair, hdp) : kernel<kInt8>(pair, hdp);
}

}  // namespace tri
