// How a wave walks the page list of an item's keys [begin, end), 64 entries at a time, a lane each: plain C++, used by the
// kernels and tested on the CPU.
#pragma once

#include <stdint.h>

namespace maaso {

// `bad` has a bit for each of 64 entries that is no page of the pool.  A lane's entry as the wave keeps it: from the first bad
// one on 0, a page of every pool, for the step that the item's keys end in may have a second page behind their end.
constexpr int32_t kept_entry(int32_t page, uint64_t bad, uint32_t lane) { return bad & (~0ull >> (63u - lane)) ? 0 : page; }

// Where the keys end for the first bad entry among the 64 from page0 on.
constexpr uint32_t end_before(uint32_t page0, uint32_t first_bad, uint32_t page_log2, uint32_t begin) {
  const uint32_t stop = (page0 + first_bad) << page_log2;
  return stop < begin ? begin : stop;
}

// Whether a step of 32 keys from page `page_at` on needs entries other than the 64 from entry0 on: it reads that page's and,
// with pages of 16, the next one's.  (It may begin a page before the item.)
constexpr bool beyond_entries(uint32_t page_at, uint32_t entry0) { return page_at - entry0 >= 63u; }
constexpr uint32_t second_entry(uint32_t at, uint32_t page_log2) { return page_log2 < 5u ? at + 1u : at; }

// Whether a page of the list holds keys of the item: others' entries have not been looked at, and are taken as 0.
constexpr bool page_of_item(uint32_t page, uint32_t begin, uint32_t end, uint32_t page_log2) {
  return page >= begin >> page_log2 && page <= (end - 1u) >> page_log2;
}

// A tile's step takes entries by eight keys, a wave's key rows by the page of the first eight of its rows, which may lie
// before the item in the item's first page.
constexpr bool eight_of_item(uint32_t key8, uint32_t begin, uint32_t end) { return key8 < end && (key8 | 15u) >= begin; }

}  // namespace maaso
