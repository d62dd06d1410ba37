// Which of the products' kernels a call takes: plain C++, used by the host side and tested on the CPU.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace maaso {

// Which tiles.  What a form takes is its rounds (tiles over the tiles that the card has places for; the last of several is not full) by what a
// round takes: us to begin and to end it, and us for each step of 128 bytes; and no less than the weights take from memory, where they are more than
// its cache holds beside the rest.  Ragged groups end in a tile of which half is empty, on the average.
struct Form {
  uint32_t rows, cols, places;  // of a tile; tiles of a compute unit
  float round, step, rate;      // us, us, bytes a us
};
// Fitted to (us of 64 x 64; 128 x 128 in four stages, one to a unit; in two, two to a unit; 256 x 256): 8 bits, 2048 to 4096 channels, 256 rows 8.1,
// 14.6, 16.3, 29.0; 512 rows 10.8, 15.4, 16.8, 29.3; 1024 rows 18.4, 16.4, 17.7, 30.0; 2048 rows 33.5, 29.3, 22.6, 31.7; 4096 rows of 4096 to 4096 113, 92, 71,
// 63; 512 rows of 8192 to 8192 in 16 bits 126, 84, 122, 199; 8 ragged experts of 16 bits, 2048 to 8192: 512 rows 69, 78, 85, 82; 1500 rows 127, 107, 99, 132; 3000
// rows 219, 181, 163, 136.  Where the choice is not the fastest it was at most 17 % slower in these and the like (1024 ragged rows 96 for 83).
constexpr Form kForms[] = {{64, 64, 1, 4.0f, 0.26f, 5.0e6f},
                           {64, 64, 2, 2.5f, 0.37f, 5.0e6f},
                           {128, 128, 1, 6.0f, 0.61f, 5.0e6f},
                           {128, 128, 2, 9.0f, 0.95f, 4.3e6f},
                           {256, 256, 1, 13.0f, 1.5f, 3.6e6f}};
constexpr uint64_t kManyWeights = 96u << 20;  // bytes

struct ProductShape {
  uint32_t n_rows, n_experts, channels, in_bytes;
  bool ragged;  // rows in groups by starts
};
constexpr uint64_t weights_of(const ProductShape& a) { return (uint64_t)a.n_experts * a.channels * a.in_bytes; }

inline uint32_t best_form(const ProductShape& a, uint32_t n_cu) {
  const uint64_t weights = weights_of(a);
  const float steps = (float)((a.in_bytes + 127u) / 128u), experts = (float)std::min(a.n_experts, a.n_rows);
  uint32_t best = 0;
  float least = 0.0f;
  for (uint32_t f = 0; f < sizeof(kForms) / sizeof(kForms[0]); ++f) {
    const Form& form = kForms[f];
    const float whole = (float)a.n_rows / (float)form.rows, down = a.ragged ? std::max(whole + 0.5f * experts, experts) : std::ceil(whole);
    const float full = down * (float)((a.channels + form.cols - 1u) / form.cols) / (float)(form.places * n_cu), rounds = full <= 1.0f ? 1.0f : full + 0.25f;
    const float work = rounds * (form.round + steps * form.step), memory = weights >= kManyWeights ? (float)weights / form.rate : 0.0f;
    const float us = std::max(work, memory) + 0.25f * std::min(work, memory);
    if (f == 0 || us < least) {
      least = us;
      best = f;
    }
  }
  return best;
}

enum ProductForm { kStream, kTiles64, kTiles128Four, kTiles128Two, kTiles256 };  // (in how many stages)

// Few rows go through waves that hold their operands in registers only: up to 16 of one matrix or of an expert where its weights are no more than 32
// MiB, which many small blocks bring sooner (8 bits, 8 MiB, 16 rows 4.7 us for 7.3 in tiles; 32 MiB 11.4 and 11.3), and up to 4 whatever the weights, for
// rows beside the last are read again by each block (64 experts of 2.3 MiB, a row each 30.6 us for 35.7, 6 rows 37.8 and 36.3; 8 experts of 32 MiB, 8 rows
// 63.4 and 58.6).
inline ProductForm product_form(const ProductShape& a, uint32_t n_cu) {
  const uint64_t rows = (a.n_rows + a.n_experts - 1u) / a.n_experts;
  if (rows <= 4u || (rows <= 16u && weights_of(a) <= (32u << 20))) return kStream;
  constexpr ProductForm kOf[] = {kTiles64, kTiles64, kTiles128Four, kTiles128Two, kTiles256};
  return kOf[best_form(a, n_cu)];
}

// Of 96 MiB of weights or more the tiles begin at unlike steps: 64 rows of 67 MB (of 16 bits) 14.1 us either way, of 100 MB 26.1 to 23.8, of 134 MB 36.8 to
// 26.2; of 32 MiB (8 bits, in the cache) 11.1 to 12.0.
constexpr bool begins_unlike(const ProductShape& a) { return weights_of(a) >= kManyWeights; }

}  // namespace maaso
