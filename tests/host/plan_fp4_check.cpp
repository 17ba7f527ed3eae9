// Answers which tile a product of 4-bit blocks takes: lines "blocks M N K" (blocks 1: 4-bit
// results) on standard input, "BMxBN" per line on standard output; "tables" lists every
// tile.  The library's own planner header, host arithmetic only.
#include <cstdio>
#include <cstring>

#include "plan.h"

using namespace wam;

int main() {
  char line[256];
  while (std::fgets(line, sizeof(line), stdin)) {
    if (!std::strncmp(line, "tables", 6)) {
      for (const auto& t : kFp4Cfgs) std::printf("%dx%d ", t.bm, t.bn);
      std::printf("\n");
      continue;
    }
    int blocks, M, N, K;
    if (std::sscanf(line, "%d %d %d %d", &blocks, &M, &N, &K) != 4) return 1;
    const TileCfg& t = kFp4Cfgs[plan_fp4(kFp4Cfgs, M, N, K, blocks != 0)];
    std::printf("%dx%d\n", t.bm, t.bn);
  }
  return 0;
}
