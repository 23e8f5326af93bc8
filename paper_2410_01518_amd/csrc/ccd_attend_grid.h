// Sizes of the grids of ccd_paged_attend: plain host arithmetic.
#pragma once
#include <stdint.h>

namespace ccd {

constexpr int64_t kMostWorkgroups = ((int64_t)1 << 24) - 1;      // of 256 threads: a launch has less than 2^32

// Blocks of `rows` rows that the sequences of a call can fill, those with more than `few` rows alone: T new tokens of G rows each, among at most B
// sequences.  Such a sequence has few / G + 1 tokens or more, and its last block up to rows - 1 rows less than a whole one.
inline int64_t most_blocks(int64_t B, int64_t T, int64_t G, int64_t rows, int64_t few) {
  const int64_t sequences = T / (few / G + 1) < B ? T / (few / G + 1) : B;
  const int64_t blocks = (T * G + sequences * (rows - 1)) / rows;
  return blocks < 1 ? 1 : blocks;
}

// stretches of every block that one launch holds beside `others` workgroups; one at least
inline int64_t most_parts(int64_t workgroups, int64_t others) {
  const int64_t parts = (kMostWorkgroups - others) / workgroups;
  return parts < 1 ? 1 : parts;
}

}  // namespace ccd
