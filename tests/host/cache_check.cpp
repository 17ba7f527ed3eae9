// Answers where a paged cache's tokens lie and what a row sees, with the library's own
// header (host arithmetic): lines on standard input,
//   page WIDTH SHIFT PAGES T e0 e1 ...   -> page of token T (-1: none)
//   held LENGTH WIDTH SHIFT              -> tokens held
//   seen HELD LENGTH CAUSAL ROWS T       -> tokens that row T sees
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "cache.h"

int main() {
  char line[4096];
  while (std::fgets(line, sizeof(line), stdin)) {
    std::vector<long> v;
    char* at = line + 4;
    for (char* end;; at = end) {
      const long x = std::strtol(at, &end, 10);
      if (end == at) break;
      v.push_back(x);
    }
    if (!std::strncmp(line, "page", 4)) {
      std::vector<int32_t> row(v.begin() + 4, v.end());  // exactly `width` entries: a read past them is out of bounds
      if ((long)row.size() != v[0]) return 1;
      std::printf("%d\n", wam::page_of(row.data(), (int)v[0], (int)v[1], (int)v[2], (int)v[3]));
    } else if (!std::strncmp(line, "held", 4)) {
      std::printf("%d\n", wam::tokens_held((int)v[0], (int)v[1], (int)v[2]));
    } else {
      std::printf("%d\n", wam::tokens_seen((int)v[0], (int)v[1], v[2] != 0, (int)v[3], (int)v[4]));
    }
  }
  return 0;
}
