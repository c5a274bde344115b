// Which kernel an 8-bit product runs on: plain host C++ (no HIP), from sizes alone, so that the rules can be checked without a GPU.  All
// kernels end with the same arithmetic on an exact sum (scaled in int8_device.h), so the choice does not show in the result.
#pragma once

namespace mm {

// ---- up to 64 tokens: int8_stream.hip ----
constexpr int kStreamWaves = 8;                            // of a workgroup
constexpr int kStreamChunk = 256;                          // k of a chunk
constexpr int stream_chunks(int TB) { return 8 / TB; }     // chunks of a wave's part of K with TB blocks of 16 tokens: 128 registers of codes
constexpr int kMaxFused = 16384;                           // elements of float tokens that every workgroup quantises: codes of more have no room in LDS
bool int8_streams(int T, int K);
// whether moe_linear_int8 leaves the quantisation to the product's workgroups
bool int8_quantises_itself(int T, int K);

// ---- beyond ----
// int8_tile.hip: 64 tokens x 64 or 128 weight rows; Shared: two groups of waves share K; Short: two stages
enum class Int8Tile { k64Shared, k64, k64Short, k128Shared, k128 };
struct Int8Route {
  int blocks;                        // int8_wide.hip: tiles of 64 blocks tokens (2 to 4) x 256 weight rows; 0: `tile`
  Int8Tile tile;
};
Int8Route int8_route(int T, int N, int K, int device_cus);

}  // namespace mm
