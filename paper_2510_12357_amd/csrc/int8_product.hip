// An 8-bit product on the kernel that int8_route.cpp chooses, by launches of kLaunchRows tokens.
#include <algorithm>

#include "internal.h"

namespace mm {

int launch_int8_product(const Int8Args& all, hipStream_t s) {
  ProfScope ps(kProfInt8Product, s);
  if (int8_streams(all.T, all.K)) return launch_int8_stream(all, s);
  int rc = MOE_OK;
  for (int64_t t = 0; t < all.T && !rc; t += kLaunchRows) {
    Int8Args a = all;
    a.T = (int)std::min<int64_t>(all.T - t, kLaunchRows);
    a.x += t * a.ldx;
    a.x_scale += t;
    a.out = static_cast<char*>(a.out) + t * a.ldo * (a.out_dtype == MOE_FP32 ? 4 : 2);
    const Int8Route r = int8_route(a.T, a.N, a.K, device_cu_count());
    rc = r.blocks ? launch_int8_wide(a, r.blocks, s) : launch_int8_tile(a, r.tile, s);
  }
  return rc;
}

}  // namespace mm
