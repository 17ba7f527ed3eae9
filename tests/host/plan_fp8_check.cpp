// Answers which tile a product of e4m3 matrices takes: lines "form M N K" (form 0:
// bf16 result, 1: float32, 2: QKV, 3: 8-bit blocks) on standard input, "BMxBN" per line on standard output; "tables" lists every
// tile of both tables.  The library's own planner header, host arithmetic only.
#include <cstdio>
#include <cstring>

#include "plan.h"

using namespace wam;

template <int NC>
static const TileCfg& choice(const TileCfg (&c)[NC], int M, int N, int K, Fp8Result r) {
  return c[plan_fp8(c, M, N, K, r)];
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
    int form, M, N, K;
    if (std::sscanf(line, "%d %d %d %d", &form, &M, &N, &K) != 4) return 1;
    const TileCfg& t = form == 1 ? choice(kFp8ExactCfgs, M, N, K, FP8_PLAIN)
                                 : choice(kFp8Cfgs, M, N, K, form == 2 ? FP8_QKV : form == 3 ? FP8_BLOCKS : FP8_PLAIN);
    std::printf("%d:%dx%d\n", form, t.bm, t.bn);
  }
  return 0;
}
