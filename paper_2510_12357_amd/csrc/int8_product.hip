// Which kernel computes an 8-bit product.  All end with the same arithmetic on an exact sum (scaled in int8_device.h), so the choice does not
// show in the result.
#include "internal.h"

namespace mm {
namespace {

// Up to 64 tokens (whose codes fit the registers of a workgroup) stream the weights: int8_stream.hip.  Beyond, tiles of 128, 192 or 256 tokens x 256 weight
// rows, one workgroup per CU and all of a round in step (int8_wide.hip), or of 64 x 128, two workgroups per CU (int8_tile.hip): the smaller
// estimate of time, from rounds, chunks of 128 k and what a tile costs beside them, all in us as measured.
// us, 64 x 128 / 128 x 256 / 192 x 256 / 256 x 256: 65 x 50257 x 1971 42 / 37 / - / -, 200 x 50257 x 2048 57 / 49 / 51 / 45, 333 x 50257 x 1971 88 / 75 / 68 / 69,
// 700 x 8192 x 2048 25 / 26 / 31 / 36, 1000 x 4096 x 4096 26 / 34 / 37 / 49, 1000 x 14336 x 4096 98 / 72 / 77 / 62, 2000 x 5000 x 1000 31 / 33 / 26 / 30,
// 4096 x 600 x 1000 14 / 18 / 22 / 27, 4096 x 4096 x 1024 37 / 26 / 32 / 24, 4096 x 131072 x 4096 3477 / - / 1946 / 1796.
// Two groups of waves per tile of 64 x 128 that share K: where there is no tile for every CU, and 1024 k.  us, one / two: 700 x 2048 x 5632 24 / 20, 128 x
// 2048 x 8192 28 / 22, 65 x 2048 x 2048 10.4 / 9.4, 300 x 4000 x 1000 10.0 / 10.2, 1500 x 1000 x 300 7.8 / 8.6, 1000 x 4096 x 4096 26 / 30.
// (Panels of 64 or 32 tokens by the streaming kernel, each reading all weights: 128 x 2048 x 8192 16.5, but 700 x 2048 x 5632 30, 200 x 8192 x 2048 19, 333 x
// 50257 x 1971 79, and 65 tokens as tiles; not kept.)
struct Route { int blocks; bool share_k; };              // blocks: of 64 tokens of a wide tile; 0: 64 x 128
Route route(int T, int N, int K) {
  const int64_t cus = device_cu_count();
  const double chunks = (K + 127) / 128;
  const int64_t tiles = (int64_t)((T + 63) / 64) * ((N + 127) / 128);
  Route best = {0, tiles <= cus && chunks >= 8};
  double least = best.share_k ? 6 + 0.3 * chunks : 4 + ((tiles + 2 * cus - 1) / (2 * cus)) * (0.73 * chunks + 3.7);
  constexpr double kChunk[5] = {0, 0, 1.0, 1.2, 1.46}, kTile[5] = {0, 0, 4.5, 6.0, 8.2};
  for (int b = 2; b <= 4; ++b) {
    const int64_t n = (int64_t)((T + 64 * b - 1) / (64 * b)) * ((N + 255) / 256);
    const double t = 8 + ((n + cus - 1) / cus) * (kChunk[b] * chunks + kTile[b]);
    if (t < least) { least = t; best = {b, false}; }
  }
  return best;
}

}  // namespace

int launch_int8_product(const Int8Args& a, hipStream_t s) {
  ProfScope ps(kProfInt8Product, s);
  if (int8_streams(a.T, a.K)) return launch_int8_stream(a, s);
  const Route r = route(a.T, a.N, a.K);
  return r.blocks ? launch_int8_wide(a, r.blocks, s) : launch_int8_tile(a, r.share_k, s);
}

}  // namespace mm
