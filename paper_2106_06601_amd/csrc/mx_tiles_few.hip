// Products of some tens of rows, whose sums go on in parts: tiles of 64 rows and 128 columns, eight waves
// of 64 rows and 16 columns.  Between the kernel for few rows, whose every workgroup converts all of the
// rows for 16 or 32 columns, and the larger tiles, which would be half empty.
#include "mx_tiles.hpp"

namespace costa {
namespace {

template <int SRC, int BBITS>
__global__ __launch_bounds__(kLanes) void tiles_few(Args p, uint32_t nn) {
  TileSums<4, 1> t;
  tile_sums<SRC, false, BBITS, 64, 128, 1, 2, true, 0>(p, 1, nn, t);
  put_wave<4, 1>(p, t.acc, t.shared, t.wave, t.row, t.col);
}

template <int SRC>
hipError_t launch(const Args& p, int splits, hipStream_t stream) {
  const uint32_t nn = (uint32_t)up_div(p.n, 128);
  if (p.b.bits == 4) tiles_few<SRC, 4><<<dim3(nn, splits), kLanes, 0, stream>>>(p, nn);
  else tiles_few<SRC, 8><<<dim3(nn, splits), kLanes, 0, stream>>>(p, nn);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tiles_few(int src, const Args& p, int splits, hipStream_t stream) {
  if (src == SRC_BF16) return launch<SRC_BF16>(p, splits, stream);
  if (src == SRC_F16) return launch<SRC_F16>(p, splits, stream);
  return launch<SRC_F32>(p, splits, stream);
}

}  // namespace costa
