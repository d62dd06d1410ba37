"""The walk over an item's page list (page_walk.hpp), compiled for the CPU with a wave as 64 lanes of a loop: no page is read
but the item's own good ones and page 0, whatever entry is bad, and a key of the item is read from its page."""
import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2509_06362_amd" / "csrc"

WALK = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "page_walk.hpp"
using namespace maaso;

constexpr int32_t kPages = 1000;
struct Item {
  std::vector<int32_t> list;
  uint32_t begin, end, log2;
  int32_t entries[64];
  uint32_t entry0;
};

static void fail(const Item& it, uint32_t at, int32_t page, int line) {
  std::printf("line %d: keys [%u, %u), pages of %u, at %u page %d\n", line, it.begin, it.end, 1u << it.log2, at, page);
  std::exit(1);
}

// held_end(): the list's entries 64 at a time, the end before the first bad one.
static void walk(Item& it) {
  const uint32_t first = it.begin >> it.log2, last = (it.end - 1u) >> it.log2;
  it.entry0 = first;
  for (uint32_t page0 = first; page0 <= last; page0 += 64u) {
    int32_t page[64];
    uint64_t bad = 0;
    for (uint32_t lane = 0; lane < 64u; ++lane) {
      page[lane] = page0 + lane <= last ? it.list.at(page0 + lane) : 0;
      if (page[lane] < 0 || page[lane] >= kPages) bad |= 1ull << lane;
    }
    if (page0 == first) for (uint32_t lane = 0; lane < 64u; ++lane) it.entries[lane] = kept_entry(page[lane], bad, lane);
    if (bad) {
      it.end = end_before(page0, (uint32_t)__builtin_ctzll(bad), it.log2, it.begin);
      return;
    }
  }
}

static int32_t own(const Item& it, uint32_t key) { return it.list.at(key >> it.log2); }

// StreamTile::ask() for every step of 32 keys that one of `split` waves takes.
static void steps(Item it, uint32_t split, uint32_t wave) {
  for (uint32_t base = (it.begin & ~31u) + 32u * wave; base < it.end; base += 32u * split) {
    const uint32_t page_at = base >> it.log2;
    if (beyond_entries(page_at, it.entry0)) {
      it.entry0 = page_at;
      for (uint32_t lane = 0; lane < 64u; ++lane)
        it.entries[lane] = page_of_item(page_at + lane, it.begin, it.end, it.log2) ? it.list.at(page_at + lane) : 0;
    }
    const uint32_t at = page_at - it.entry0, two = second_entry(at, it.log2);
    if (at >= 64u || two >= 64u) fail(it, base, -1, __LINE__);
    const int32_t pages[2] = {it.entries[at], it.entries[two]};
    for (uint32_t key = base; key < base + 32u; ++key) {
      const int32_t page = pages[(key - base) / 16u];
      if (page < 0 || page >= kPages) fail(it, key, page, __LINE__);
      if (key >= it.begin && key < it.end && page != own(it, key)) fail(it, key, page, __LINE__);
    }
  }
}

// The tiles' steps of `keys` keys: entries by eight keys, the first step's from the walk, the others' from the list.
static void tiles(const Item& it, uint32_t keys, uint32_t wave_rows) {
  const uint32_t first = it.begin & ~(keys - 1u);
  for (uint32_t base = first; base < it.end; base += keys) {
    int32_t ids[8];
    for (uint32_t c = 0; c < keys / 8u; ++c) {
      const uint32_t key8 = base + 8u * c, nth = (key8 >> it.log2) - (it.begin >> it.log2);
      ids[c] = !eight_of_item(key8, it.begin, it.end) ? 0 : base == first ? it.entries[nth & 63u] : it.list.at(key8 >> it.log2);
      if (ids[c] < 0 || ids[c] >= kPages) fail(it, key8, ids[c], __LINE__);
      for (uint32_t key = key8; key < key8 + 8u; ++key)
        if (key >= it.begin && key < it.end && ids[c] != own(it, key)) fail(it, key, ids[c], __LINE__);
    }
    for (uint32_t row0 = 0; row0 < keys; row0 += wave_rows)
      for (uint32_t key = base + row0; key < base + row0 + wave_rows; ++key)
        if (key >= it.begin && key < it.end && ids[row0 / 8u] != own(it, key)) fail(it, key, ids[row0 / 8u], __LINE__);
  }
}

int main() {
  long items = 0;
  for (uint32_t log2 = 4; log2 <= 7; ++log2)
    for (uint32_t n = 1; n <= 140; n += n < 8 ? 1 : n < 60 ? 19 : 31 + n % 3)
      for (int32_t where = -1; where < (int32_t)n; ++where)
        for (int32_t entry : {-1, kPages}) {
          if (where < 0 && entry != -1) continue;
          for (uint32_t skip : {0u, 1u, 16u, 31u, 48u, 64u, 250u, 1024u, 1100u})
            for (uint32_t left : {0u, 1u, 15u, 16u}) {
              if (left + 1u + skip > n << log2) continue;
              Item it{{}, skip, (n << log2) - left, log2, {}, 0};
              for (uint32_t k = 0; k < n; ++k) it.list.push_back((int32_t)((k * 37u + 5u) % kPages));
              if (where >= 0) it.list[(size_t)where] = entry;
              // (what lies before the item's first page is never looked at)
              for (uint32_t k = 0; k < skip >> log2; ++k) it.list[k] = -7;
              walk(it);
              ++items;
              if (it.begin >= it.end) continue;
              for (uint32_t wave = 0; wave < 4; ++wave) steps(it, 4, wave);
              steps(it, 1, 0);
              tiles(it, 64, 16);
              tiles(it, 32, 8);
            }
        }
  std::printf("%ld\n", items);
  return 0;
}
"""


def test_only_good_pages_are_read(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(WALK)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Wextra", "-Werror", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout
    assert int(run.stdout) > 30_000
