// Plain host C++; 64 bits, so that the largest sizes do not overflow.
#include "attention_plan.h"

#include <algorithm>

namespace mm {

SplitPlan plan_splits(int sequences, int kv_heads, int group, int max_len, int window, int device_cus) {
  // a window that starts inside a block of 64 positions reaches over one more of them
  const int64_t span = std::max<int64_t>(1, window > 0 && window < max_len ? (int64_t)window + 63 : max_len);
  const int64_t blocks = (span + 63) / 64, tiles = (group + kHeadTile - 1) / kHeadTile;
  const int64_t units = std::max<int64_t>(1, (int64_t)sequences * kv_heads * tiles), wanted = 16 * (int64_t)device_cus;
  const int64_t most = kMaxSplit / 64;
  int64_t each = std::min(most, std::max<int64_t>(blocks * units / wanted, 8));      // blocks of a part
  each = std::min(each, blocks);
  return {(int)(each * 64), (int)((blocks + each - 1) / each)};
}

// Few workgroups: waiting until what they hand over has arrived costs each of them less than a second launch costs the call.
bool joins_inside(int sequences, int kv_heads, int group, const SplitPlan& p, int device_cus) {
  const int64_t units = (int64_t)sequences * kv_heads * ((group + kHeadTile - 1) / kHeadTile);
  return p.parts <= 32 && units <= kCounters && units * p.parts <= 3 * (int64_t)device_cus;
}

}  // namespace mm
