// Answers which tile a product of e4m3 matrices takes: lines "exact M N K" (exact 0
// or 1) on standard input, "BMxBN" per line on standard output; "tables" lists every
// tile of both tables.  The library's own planner header, host arithmetic only.
#include <cstdio>
#include <cstring>

#include "plan.h"

using namespace wam;

template <int NC>
static const TileCfg& choice(const TileCfg (&c)[NC], int M, int N, int K) {
  return c[plan_fp8(c, M, N, K)];
}

int main() {
  char line[256];
  while (std::fgets(line, sizeof(line), stdin)) {
    if (!std::strncmp(line, "tables", 6)) {
      for (const auto& t : kFp8Cfgs) std::printf("0:%dx%d ", t.bm, t.bn);
      for (const auto& t : kFp8ExactCfgs) std::printf("1:%dx%d ", t.bm, t.bn);
      std::printf("\n");
      continue;
    }
    int exact, M, N, K;
    if (std::sscanf(line, "%d %d %d %d", &exact, &M, &N, &K) != 4) return 1;
    const TileCfg& t = exact ? choice(kFp8ExactCfgs, M, N, K) : choice(kFp8Cfgs, M, N, K);
    std::printf("%d:%dx%d\n", exact, t.bm, t.bn);
  }
  return 0;
}
