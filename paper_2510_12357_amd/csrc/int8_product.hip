// Which kernel computes an 8-bit product.  All end with the same arithmetic on an exact sum (scaled in int8_device.h), so the choice does not
// show in the result.
#include "internal.h"

namespace mm {
namespace {

}  // namespace

int launch_int8_product(const Int8Args& a, hipStream_t s) {
  ProfScope ps(kProfInt8Product, s);
  if (int8_streams(a.T, a.K)) return launch_int8_stream(a, s);
  const int64_t wide = (int64_t)((a.T + 255) / 256) * ((a.N + 255) / 256);
  if (wide >= 128) return launch_int8_wide(a, a.T > 192 ? 4 : (a.T + 63) / 64, s);
  return launch_int8_tile(a, 64, s);
}

}  // namespace mm
