// Plain host C++; 64 bits, so that the largest sizes do not overflow.
#include "attention_plan.h"

#include <algorithm>

namespace mm {

// slots: workgroups of four waves that the device runs at once.  As many have equal shares, whatever the sequences' lengths are, so that all end together.  Where the work is
// too little for that, a workgroup has one unit or a part of one: what a second one in a row would wait for costs more
// (us, shares / aligned: 4 sequences of up to 2000 on 8 key heads of 64 channels 16.5 / 9.9, 33 on a window of 1000 with 71 heads 19.5 / 17.0, 8 of up to 4096
// 21.7 / 21.3; not where units in parts take two rounds, 30 of up to 2000 28.9 / 34.4).  Parts of 4 blocks as long as there is a CU for each (4 sequences of up to 2000: 2 us
// more with 8).
// Many units of up to 8 blocks go one to a wave, which begins and ends each by itself, workgroups being waves (us, shares of four waves / one wave a unit: 128 sequences
// of up to 300 28.4 / 24.0, of up to 64 14.4 / 10.4, 214 of up to 3 26.3 / 12.0, 216 of up to 155 with 24 heads to a key head 35.6 / 21.9, 256 of up to 512 58.3 / 54.4; not
// units of more blocks, whose four waves read neighbouring rows: 128 of up to 1000 51.9 / 58.7, 64 of up to 8192 178 / 185).  Beyond two rounds of waves,
// one for units of one block, the waves have shares (one wave a unit / shares of one wave: 512 sequences of up to 200 56.9 / 58.2, 1000 115 / 103, 600 of up to 60 42.1 / 33.3,
// 2000 of up to 30 215 / 77, but 214 of up to 3 12.0 / 16.8).
AttentionPlan plan_attention(int sequences, int kv_heads, int group, int max_len, int window, int slots, int device_cus) {
  const int64_t units = (int64_t)sequences * kv_heads * ((group + kHeadTile - 1) / kHeadTile);
  // a window that starts inside a block reaches over one more of them
  const int64_t span = window > 0 && window < max_len ? (int64_t)window + kSpan - 1 : max_len;
  const int64_t blocks = std::max<int64_t>(1, (span + kSpan - 1) / kSpan);
  auto parts = [&](int64_t align) { return (blocks + align - 1) / align; };
  AttentionPlan p;
  const bool waves_alone = parts(8) == 1 && units > slots;
  p.waves = waves_alone ? 1 : kMostWaves;
  slots *= kMostWaves / p.waves;
  if (waves_alone) p.align = units <= (blocks > 1 ? 2 : 1) * (int64_t)slots ? 8 : 0;
  else p.align = units * parts(4) <= device_cus ? 4 : units * parts(8) <= slots ? 8 : 0;
  p.fits = (double)units * (double)(blocks + std::max(kSetup, p.align)) < (double)(1 << 30);
  if (!p.fits) return p;
  p.workgroups = p.align ? (int)std::max<int64_t>(1, units * parts(p.align)) : std::min(slots, kMostWorkgroups);
  p.split = p.align ? parts(p.align) > 1 : true;
  p.few_parts = (p.align ? parts(p.align) : p.workgroups / units) <= 16;
  return p;
}

}  // namespace mm
