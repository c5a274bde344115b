// Reads commands, one a line, and answers with the library's rules (csrc/attention_plan.h, attention_plan.cpp).
//   page SHIFT N_PAGES POS ENTRY...     -> page of a position, or -1
//   seen LENGTH MAX_LEN WINDOW TABLE_LEN SHIFT            -> first end bad blocks
//   plan SEQUENCES KV_HEADS GROUP MAX_LEN WINDOW SLOTS CUS -> fits workgroups align split few_parts waves
//   line WORKGROUPS ALIGN LEAST UNITS BLOCKS...           -> for every segment: workgroup sequence unit block blocks first-workgroup parts, ended by a -1
//   shift PAGE_SIZE
#include <algorithm>
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>
#include <vector>

#include "attention_plan.h"

int main() {
  for (std::string line; std::getline(std::cin, line);) {
    std::istringstream in(line);
    std::string what;
    in >> what;
    if (what == "page") {
      int shift, pages;
      long long pos;
      in >> shift >> pages >> pos;
      std::vector<int32_t> row;
      for (int e; in >> e;) row.push_back(e);
      std::printf("%d\n", mm::page_of(row.data(), (int)row.size(), pages, shift, pos));
    } else if (what == "seen") {
      int v[5];
      for (int& x : v) in >> x;
      const mm::Seen s = mm::seen_by(v[0], v[1], v[2], v[3], v[4]);
      std::printf("%d %d %d %d\n", s.first, s.end, (int)s.bad, mm::blocks_of(s));
    } else if (what == "plan") {
      int v[7];
      for (int& x : v) in >> x;
      const mm::AttentionPlan p = mm::plan_attention(v[0], v[1], v[2], v[3], v[4], v[5], v[6]);
      if (p.fits) std::printf("1 %d %d %d %d %d\n", p.workgroups, p.align, (int)p.split, (int)p.few_parts, p.waves);
      else std::printf("0\n");
    } else if (what == "line") {                             // the walk of every workgroup, as the kernel takes it
      int workgroups, align, least, units, total = 0;
      in >> workgroups >> align >> least >> units;
      std::vector<int> n;
      for (int x; in >> x;) { n.push_back(x); total += mm::line_places(x, align) * units; }
      const int each = mm::places_each(total, workgroups, align, least);
      for (int w = 0; w < workgroups; ++w) {
        int cursor = (int)std::min<long long>(total, (long long)w * each);
        const int finish = std::min(total, cursor + each);
        if (cursor >= finish) continue;
        int b = 0, line = 0;
        while (cursor >= line + mm::line_places(n[b], align) * units) line += mm::line_places(n[b++], align) * units;
        while (true) {
          const mm::Segment s = mm::segment_at(line, n[b], align, cursor, finish, each);
          if (s.blocks) std::printf("%d %d %d %d %d %d %d ", w, b, s.unit, s.block, s.blocks, s.workgroup, s.parts);
          cursor += s.length;
          if (cursor >= finish) break;
          if (cursor >= line + mm::line_places(n[b], align) * units) {
            line += mm::line_places(n[b], align) * units;
            do ++b; while (n[b] == 0);
          }
        }
      }
      std::printf("-1\n");
    } else {
      int n;
      in >> n;
      std::printf("%d\n", mm::page_shift(n));
    }
  }
}
