// Plain host C++; the rules' arithmetic is in 64 bits, so that the largest sizes do not overflow.
#include "int8_route.h"

#include <stdint.h>

#include <algorithm>

namespace mm {

bool int8_streams(int T, int K) { return T <= 64 && (K + kStreamChunk - 1) / kStreamChunk <= kStreamWaves * stream_chunks(T <= 16 ? 1 : (T <= 32 ? 2 : 4)); }

// Wherever their codes fit beside the rings: a launch in front of the product costs a caller 3.7 us (eager, from Python), and the GPU, in a graph, us inside / in a
// launch of its own on 2048 | 32000 outputs: bf16 1 x 2048 5.5 / 6.5 | 14.5 / 16.3, 1 x 16384 12.1 / 18.4 | 84 / 90, 4 x 4096 7.4 / 8.1 | 25.5 / 27.0, 8 x 2048 6.7 / 7.0 |
// 16.1 / 16.6, 16 x 1024 6.7 / 6.9 | 11.6 / 12.1; fp32 1 x 16384 13.7 / 20.3 | 87 / 93, 2 x 8192 10.7 / 11.8 | 46.8 / 48.4, 8 x 1024 6.3 / 6.9 | 10.7 / 11.6, 16 x 512 6.2 / 6.5 |
// 8.8 / 9.1.  The other way round where more than two rows are longer than their threads hold, and so are read twice: fp32 4 x 4096 8.8 / 8.4 | 27.6 / 27.4,
// 8 x 2048 8.0 / 7.3 | 17.9 / 16.7, 16 x 1024 8.0 / 6.9 | 13.2 / 12.0, bf16 12 x 1344 7.8 / 6.7 | 15.2 / 14.5, 9 x 1792 8.2 / 6.8 | 16.7 / 15.4.
bool int8_quantises_itself(int T, int K) { return T <= 16 && (int64_t)T * K <= kMaxFused; }

// Up to 64 tokens (whose codes fit the registers of a workgroup) stream the weights: int8_stream.hip.  Beyond, tiles of 64 tokens x 64 or 128 weight
// rows, several workgroups per CU or one whose two groups of waves share K (int8_tile.hip), or of 128, 192 or 256 x 256, one workgroup per CU and
// all of a round in step (int8_wide.hip).
// From 13 chunks of 128 k on and with a CU for every tile, shared K: 64 x 64, else 64 x 128.  us, 64 x 64 shared / 64 x 64 / 64 x 128 shared / 64 x 128: 65 x 2048 x 2048
// 7.2 / 8.0 / 9.3 / 10.4, 128 x 2048 x 8192 16.2 / 20.6 / 21.9 / 27.4; 1024 x 2048 x 2048 14.9 / 11.7 / 11.0 / 11.7, 256 x 8192 x 4096 21.0 / 17.7 / 16.0 / 18.7,
// 700 x 2048 x 5632 25.8 / 20.5 / 19.9 / 22.1; fewer chunks: 500 x 2048 x 1500 9.1 / 8.5 / 11.3 / 11.1, 300 x 2048 x 1000 6.7 / 6.6 / 8.7 / 8.5.
// Up to 16 chunks, and all tiles of 64 x 64 under way at once, three to a CU: these.  us, 64 x 64 / the same in two stages / 64 x 128: 300 x 4000 x 1000 8.7 / 9.9 / 9.8,
// 700 x 2048 x 1500 10.6 / 12.6 / 11.7, 555 x 3712 x 1920 12.2 / 13.9 / 12.6, 100 x 16384 x 512 6.5 / 7.2 / 7.8, 787 x 3215 x 175 6.1 / 6.1 / 7.2.
// More tiles: the smallest estimate of time, from rounds, chunks and what a tile costs beside them, all in us as measured; two stages up to 5 chunks.
// us, 64 x 64 in two stages / 64 x 128 / 128 x 256 / 192 x 256 / 256 x 256: 179 x 101674 x 114 26 / 30 / 44 / 36 / -, 514 x 21096 x 75 15 / 17 / 21 / 20 / 22, 2231 x 40884 x 98
// 107 / 114 / 94 / 93 / 84, 1000 x 4096 x 600 10.8 / 11.6 / 16 / 16 / 24, 130 x 33000 x 300 12.5 / 14.2 / 17 / 19 / -, 1000 x 30000 x 500 60 / 59 / 50 / 42 / 45;
// - / 64 x 128 / ...: 65 x 50257 x 1971 39 / 35 / - / -, 200 x 50257 x 2048 56 / 48 / 51 / 44, 333 x 50257 x 1971 85 / 73 / 67 / 70,
// 700 x 8192 x 2048 24 / 25 / 30 / 35, 1000 x 4096 x 4096 26 / 34 / 38 / 49, 1000 x 14336 x 4096 98 / 72 / 77 / 62, 2000 x 5000 x 1000 29 / 31 / 25 / 29,
// 4096 x 4096 x 1024 37 / 26 / 32 / 24, 4096 x 131072 x 4096 3477 / - / 1946 / 1796.
// (Panels of 64 or 32 tokens by the streaming kernel, each reading all weights: 128 x 2048 x 8192 16.5, 700 x 2048 x 5632 30, 200 x 8192 x 2048 19, 333 x 50257 x
// 1971 79; not kept.)
Int8Route int8_route(int T, int N, int K, int device_cus) {
  const int64_t cus = device_cus, panels = (T + 63) / 64, narrow = panels * ((N + 63) / 64), tiles = panels * ((N + 127) / 128);
  const int chunks = (K + 127) / 128;
  if (chunks > 12 && narrow <= cus) return {0, Int8Tile::k64Shared};
  if (chunks > 12 && tiles <= cus) return {0, Int8Tile::k128Shared};
  if (chunks <= 16 && narrow <= 3 * cus) return {0, Int8Tile::k64};
  Int8Route best = {0, Int8Tile::k128};
  double least = 4 + (double)((tiles + 2 * cus - 1) / (2 * cus)) * (0.73 * chunks + 3.7);
  const double brief = 3 + (double)narrow / (double)cus * (1.0 + 0.19 * chunks);
  if (chunks <= 5 && brief < least) { least = brief; best = {0, Int8Tile::k64Short}; }
  constexpr double kChunk[5] = {0, 0, 1.0, 1.2, 1.46}, kTile[5] = {0, 0, 4.5, 6.0, 8.2};
  for (int b = 2; b <= 4; ++b) {
    const int64_t n = (int64_t)((T + 64 * b - 1) / (64 * b)) * ((N + 255) / 256);
    const double t = 8 + (double)((n + cus - 1) / cus) * (kChunk[b] * std::max(chunks, 3) + kTile[b]);   // it goes through three chunks at least
    if (t < least) { least = t; best = {b, Int8Tile::k128}; }
  }
  return best;
}

}  // namespace mm
