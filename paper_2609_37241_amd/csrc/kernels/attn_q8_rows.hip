// Attention over pages of 8-bit codes on the matrix cores, few rows per request.
#include "../internal.h"
#include "attn_q8.h"

namespace tri {
using namespace dev;

template <int DT, int CT, int HDP>
__global__ __launch_bounds__(64 * rows_waves(HDP), 1) void k_pa8_rows(PagedQ8Args a) {
  body_pa8_rows<DT, CT, HDP>(a);
}

namespace {
template <int DT, int CT>
const void *rows_of(int32_t hdp) {
  switch (hdp) {
    case 64: return reinterpret_cast<const void *>(&k_pa8_rows<DT, CT, 64>);
    case 128: return reinterpret_cast<const void *>(&k_pa8_rows<DT, CT, 128>);
    case 256: return reinterpret_cast<const void *>(&k_pa8_rows<DT, CT, 256>);
    default: return nullptr;
  }
}
}  // namespace

// hdp: the head size rounded up to 64, 128 or 256.
const void *attn_q8_rows(uint32_t dtype, int32_t code, int32_t hdp) {
  if (dtype == TRI_F32)
    return code == TRI_E4M3 ? rows_of<kF32, kE4M3>(hdp) : rows_of<kF32, kInt8>(hdp);
  return code == TRI_E4M3 ? rows_of<kBF16, kE4M3>(hdp) : rows_of<kBF16, kInt8>(hdp);
}

}  // namespace tri
