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
constexpr int kMaxSplit = 4096;          // positions of a workgroup: its pages' numbers stay in LDS
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

// Part s of what a token sees, in positions: parts are `split` long (a multiple of 64) and start at multiples of 64.
struct Part { int begin, end; };
MM_BOTH Part part_of(const Seen& v, int split, int s) {
  const int64_t base = v.first / 64 * 64, b = base + (int64_t)s * split, e = b + split;
  return {(int)(b < v.end ? b : v.end), (int)(e < v.end ? e : v.end)};
}

// How many parts a sequence has.
MM_BOTH int parts_of(const Seen& v, int split) {
  const int64_t n = (int64_t)v.end - v.first / 64 * 64;
  return (int)((n + split - 1) / split);
}

// The split of a call: positions of a part and how many there are at most.
struct SplitPlan { int split, parts; };
constexpr int kCounters = 16384;         // of workgroups' ends, one per sequence, key head and head tile
bool joins_inside(int sequences, int kv_heads, int group, const SplitPlan& p, int device_cus);
SplitPlan plan_splits(int sequences, int kv_heads, int group, int max_len, int window, int device_cus);

}  // namespace mm
