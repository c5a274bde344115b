// Where a position of a paged cache lies, what one new token sees of it, and how its attention is split over workgroups: plain C++ (no HIP
// include), from integers alone, so that pages, windows and splits can be checked without a GPU.  The kernels use the same functions.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define MM_BOTH __host__ __device__ __forceinline__
#else
#define MM_BOTH inline
#endif

namespace mm {

constexpr int kMinPage = 4;              // four neighbouring positions that start at a multiple of four are in one page
constexpr int kSpan = 64;                // positions of the blocks that work is counted in
constexpr int kMaxPiece = 4096;          // positions whose pages' numbers a workgroup has in LDS at once
constexpr int kHeadTile = 16;            // query heads of a workgroup, the columns of a matrix instruction

// log2 of the page size; -1 where it is none of 4, 8, 16 ..
MM_BOTH int page_shift(int page_size) {
  if (page_size < kMinPage || (page_size & (page_size - 1))) return -1;
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}

// The page of a position, or -1: a number outside the cache, a position before the sequence or behind the table's row.
MM_BOTH int page_of(const int32_t* table_row, int table_len, int n_pages, int shift, int64_t pos) {
  if (pos < 0 || (pos >> shift) >= table_len) return -1;
  const int p = table_row[pos >> shift];
  return p >= 0 && p < n_pages ? p : -1;
}

// Positions [first, end) that a sequence's new token sees; `bad`: its length is negative, above the call's bound or behind the table.
struct Seen { int first, end; bool bad; };
MM_BOTH Seen seen_by(int length, int max_len, int window, int table_len, int shift) {
  const bool bad = length < 0 || length > max_len || (int64_t)length > ((int64_t)table_len << shift);
  if (bad || length == 0) return {0, 0, bad};
  return {window > 0 && length > window ? length - window : 0, length, false};
}

// Its blocks, of which the first one may begin before what is seen.
MM_BOTH int blocks_of(const Seen& v) { return (int)(((int64_t)v.end - v.first / kSpan * kSpan + kSpan - 1) / kSpan); }

// All work of a call is a line of blocks: sequence by sequence, of each its units (a tile of query heads on a key head), of each unit its own blocks.  Workgroup w has the
// places [w each, (w + 1) each) of the line, a row of segments, each of one unit.  A unit whose own blocks lie in several workgroups has its parts joined.
// align 0: equal shares of the whole line, on which kSetup places in front of each unit stand for what it takes to begin and end one.  Else shares are of `align`
// places, and so is what units are rounded up to: a workgroup has one unit.
// (128 sequences of up to 1000 on 8 key heads, with 4, 2 or 1 places to begin and end a unit: 52.7, 54.3 and 63.8 us.)
constexpr int kSetup = 4;
MM_BOTH int unit_places(int n, int align) { return align ? (n + align - 1) / align * align : n + kSetup; }
MM_BOTH int line_places(int n, int align) { return n > 0 ? unit_places(n, align) : 0; }
MM_BOTH int places_each(int total, int workgroups, int align, int least) {
  if (align) return align;
  const int n = (int)(((int64_t)total + workgroups - 1) / workgroups);
  return n > least ? n : least;
}
struct Segment {
  int unit;                              // of the sequence
  int length;                            // places of the line
  int block, blocks;                     // of the unit's own, from where on, and how many
  int workgroup, parts;                  // that has the unit's first block, and how many have any
};
// The segment at place `at` of the line for a workgroup whose share ends at `end`; the sequence begins at `line` and has n > 0 blocks a unit.
MM_BOTH Segment segment_at(int line, int n, int align, int at, int end, int each) {
  Segment s;
  const int places = unit_places(n, align);
  s.unit = (at - line) / places;
  const int begin = line + s.unit * places, own = begin + (align ? 0 : kSetup), behind = own + n;
  const int stop = begin + places < end ? begin + places : end, last = behind < stop ? behind : stop, start = at > own ? at : own;
  s.length = stop - at;
  s.block = start - own;
  s.blocks = last > start ? last - start : 0;
  s.workgroup = own / each;
  s.parts = (behind - 1) / each - s.workgroup + 1;
  return s;
}

// What the host knows of a call.
constexpr int kLeast = 8;                // places of a workgroup
constexpr int kMostWorkgroups = 4096;
constexpr int kMostWaves = 4;
struct AttentionPlan {
  bool fits;                             // the line's length in 31 bits
  int workgroups, waves, align;          // waves of a workgroup: kMostWaves, or 1
  bool split;                            // a unit may lie in several workgroups
  bool few_parts;                        // units are expected to lie in so few that the last one to end joins them; else a second kernel
};
AttentionPlan plan_attention(int sequences, int kv_heads, int group, int max_len, int window, int slots, int device_cus);

}  // namespace mm
