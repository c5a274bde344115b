// Plain host C++; 64 bits, so that the largest sizes do not overflow.
#include "attention_plan.h"

#include <algorithm>

namespace mm {

// slots: workgroups of four waves that the device runs at once.  As many have equal shares, whatever the sequences' lengths are, so that all end together.  Where the work is
// too little for that, a workgroup has one unit or a part of one: what a second one in a row would wait for costs more
// (us, shares / aligned: 4 sequences of up to 2000 on 8 key heads of 64 channels 16.8 / 10.2, 33 on a window of 1000 with 71 heads 20.1 / 17.7, 8 of up to 4096 in
// 8 bits 17.8 / 17.3, in bf16 22.1 / 22.1; not where units in parts take two rounds, 30 of up to 2000 29.7 / 35.1).  Parts of 4 blocks as long as there is a CU for each
// (4 sequences of up to 2000: 1.6 us more with 8).  Both counts are of the bound of the lengths: of ragged ones up to half of the parts have nothing, and CUs that wait.
// Many units of up to 8 blocks go one to a wave, which begins and ends each by itself, workgroups being waves (us, shares of four waves / one wave a unit: 128 sequences
// of up to 300 29.6 / 21.9, of up to 64 15.2 / 11.0, 214 of up to 3 26.9 / 12.2, 216 of up to 155 with 24 heads to a key head 36.3 / 21.9, 256 of up to 512 59.3 / 55.0; not
// units of more blocks, whose four waves read neighbouring rows: 128 of up to 1000 52.8 / 59.6, 64 of up to 8192 179 / 186).  Beyond two rounds of waves,
// one for units of one block, the waves have shares (one wave a unit / shares of one wave: 512 sequences of up to 200 56.7 / 57.5, 1000 117 / 104, 600 of up to 60 43.9 / 34.6,
// 2000 of up to 30 221 / 77, but 214 of up to 3 12.2 / 17.2).
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
