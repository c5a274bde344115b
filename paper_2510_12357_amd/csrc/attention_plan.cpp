// Plain host C++; 64 bits, so that the largest sizes do not overflow.
#include "attention_plan.h"

#include <algorithm>

namespace mm {

// slots: workgroups that the device runs at once.  As many have the line's blocks in equal shares, whatever the sequences' lengths are, so that all end together;
// fewer where their shares would be below the least.
AttentionPlan plan_attention(int sequences, int kv_heads, int group, int max_len, int window, int slots) {
  const int64_t units = (int64_t)sequences * kv_heads * ((group + kHeadTile - 1) / kHeadTile);
  // a window that starts inside a block reaches over one more of them
  const int64_t span = window > 0 && window < max_len ? (int64_t)window + kSpan - 1 : max_len;
  const int64_t blocks = (span + kSpan - 1) / kSpan, total = units * (blocks + kSetup);
  AttentionPlan p;
  p.fits = (double)units * (double)(blocks + kSetup) < (double)(1 << 30);
  p.workgroups = (int)std::clamp<int64_t>((total + kLeastBlocks - 1) / kLeastBlocks, 1, std::min(slots, kMostWorkgroups));
  p.split = blocks > 1;
  p.few_parts = std::min((blocks + kLeastBlocks - 1) / kLeastBlocks, p.workgroups / std::max<int64_t>(units, 1)) <= 16;
  return p;
}

}  // namespace mm
