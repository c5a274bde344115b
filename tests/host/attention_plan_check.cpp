// Reads commands, one a line, and answers with the library's rules (csrc/attention_plan.h, attention_plan.cpp).
//   page SHIFT N_PAGES POS ENTRY...     -> page of a position, or -1
//   seen LENGTH MAX_LEN WINDOW TABLE_LEN SHIFT SPLIT PART -> first end bad begin end
//   plan SEQUENCES KV_HEADS GROUP MAX_LEN WINDOW CUS      -> split parts
//   shift PAGE_SIZE
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
      int v[7];
      for (int& x : v) in >> x;
      const mm::Seen s = mm::seen_by(v[0], v[1], v[2], v[3], v[4]);
      const mm::Part p = mm::part_of(s, v[5], v[6]);
      std::printf("%d %d %d %d %d\n", s.first, s.end, (int)s.bad, p.begin, p.end);
    } else if (what == "plan") {
      int v[6];
      for (int& x : v) in >> x;
      const mm::SplitPlan p = mm::plan_splits(v[0], v[1], v[2], v[3], v[4], v[5]);
      std::printf("%d %d\n", p.split, p.parts);
    } else {
      int n;
      in >> n;
      std::printf("%d\n", mm::page_shift(n));
    }
  }
}
