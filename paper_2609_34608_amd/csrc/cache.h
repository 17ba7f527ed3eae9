// Where the tokens of a paged cache lie.  Host arithmetic too, so that a CPU test can ask.
#pragma once

#include <stdint.h>

#ifdef __HIP__
#define WAM_HD __host__ __device__ inline
#else
#define WAM_HD inline
#endif

namespace wam {

// Page of token t of a sequence whose row of the table is `row` (of `width` entries;
// pages of 2^shift tokens, a pool of `pages`), or -1 where it has none.
WAM_HD int page_of(const int32_t* row, int width, int shift, int pages, int t) {
  if (t < 0 || (t >> shift) >= width) return -1;
  const int e = row[t >> shift];
  return (uint32_t)e < (uint32_t)pages ? e : -1;
}

// Tokens that the table of a sequence of this length reaches.
WAM_HD int tokens_held(int length, int width, int shift) {
  const int64_t room = (int64_t)width << shift;
  return length < 0 ? 0 : length > room ? (int)room : length;
}

// How many of the first tokens row t of `rows` sees, of `held` tokens of a sequence of
// this length: all, or, causal, those up to its own, the last rows being the sequence's
// last tokens.
WAM_HD int tokens_seen(int held, int length, bool causal, int rows, int t) {
  if (t >= rows) return 0;
  if (!causal) return held;
  const int64_t n = (int64_t)length - rows + t + 1;
  return n < 0 ? 0 : n > held ? held : (int)n;
}

}  // namespace wam
