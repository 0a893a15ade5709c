// Attention over pages of 8-bit codes on the matrix cores, few rows per request.
#include "../internal.h"
#include "attn_q8.h"

namespace tri {
using namespace dev;

template <int DT, int CT, int HDP, int HG>
__global__ __launch_bounds__(64 * rows_waves(HDP), 1) void k_pa8_rows(PagedQ8Args a) {
  body_pa8_rows<DT, CT, HDP, HG>(a);
}

namespace {
template <int DT, int CT, int HDP>
const void *rows_of(int32_t heads) {
  switch (heads) {
    case 1: return reinterpret_cast<const void *>(&k_pa8_rows<DT, CT, HDP, 1>);
    case 2: return reinterpret_cast<const void *>(&k_pa8_rows<DT, CT, HDP, 2>);
    case 4: return reinterpret_cast<const void *>(&k_pa8_rows<DT, CT, HDP, 4>);
    default: return nullptr;
  }
}

template <int DT, int CT>
const void *rows_of(int32_t hdp, int32_t heads) {
  return hdp == 64    ? rows_of<DT, CT, 64>(heads)
         : hdp == 128 ? rows_of<DT, CT, 128>(heads)
         : hdp == 256 ? rows_of<DT, CT, 256>(heads)
                      : nullptr;
}
}  // namespace

// hdp: the head size rounded up to 64, 128 or 256; heads: K heads of a tile.
const void *attn_q8_rows(uint32_t dtype, int32_t code, int32_t hdp, int32_t heads) {
  if (dtype == TRI_F32)
    return code == TRI_E4M3 ? rows_of<kF32, kE4M3>(hdp, heads) : rows_of<kF32, kInt8>(hdp, heads);
  return code == TRI_E4M3 ? rows_of<kBF16, kE4M3>(hdp, heads) : rows_of<kBF16, kInt8>(hdp, heads);
}

}  // namespace tri
