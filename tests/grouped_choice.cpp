// grouped_tile of csrc/t3_choice.h for the tests.
#include "t3_choice.h"

extern "C" void grouped_tile(int wgrad, int kn, int64_t M, int64_t N, int64_t K, int64_t groups, int cus, int wide_ok, int32_t *out) {
  const t3k::Choice c = t3k::grouped_tile(wgrad, kn, M, N, K, groups, cus, wide_ok);
  out[0] = c.kernel == t3k::kWideTile;
  out[1] = c.tile.m;
  out[2] = c.tile.n;
  out[3] = t3k::quarters_of(c.tile);
}

extern "C" int grouped_wide_fits(int kn, int64_t K, int64_t lda, int64_t ldb, int64_t ldc) { return t3k::grouped_wide_fits(kn, K, lda, ldb, ldc); }
