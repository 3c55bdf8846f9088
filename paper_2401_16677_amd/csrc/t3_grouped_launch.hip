// Launches of the products by group.
#include "t3_small.h"
#include "t3_launch.h"

namespace t3k {
namespace {

template <int BM, int MODE, int BKN, int AKM, int I8>
t3_status launch_tiles(const Plan &q, hipStream_t s) {
  // (a launch has less than 2^32 lanes: 2^23 workgroups at a time, `begin` the first one's grid position)
  constexpr int32_t kPart = 1 << 23;
  if (q.total_blocks > kPart) {
    Plan part = q;
    for (int32_t at = 0; at < q.total_blocks; at += kPart) {
      part.begin = at;
      part.total_blocks = q.total_blocks - at < kPart ? q.total_blocks - at : kPart;
      const t3_status st = launch(small_tile_kernel<BM, BM, 4, 2, MODE, BKN, AKM, false, I8>, dim3((unsigned)part.total_blocks), dim3(256), s, part);
      if (st != T3_OK) return st;
    }
    return T3_OK;
  }
  const dim3 grid((unsigned)q.total_blocks), block(256);
  // (the plan by one vector request while all workgroups are on the chip at once: see small_tile_kernel)
  if (q.total_blocks <= q.resident * (BM == 32 ? 2 : 1)) return launch(small_tile_kernel<BM, BM, 4, 2, MODE, BKN, AKM, true, I8>, grid, block, s, q);
  return launch(small_tile_kernel<BM, BM, 4, 2, MODE, BKN, AKM, false, I8>, grid, block, s, q);
}
template <int MODE, int BKN, int AKM, int I8>
t3_status launch_small(const Plan &q, int32_t tm, int32_t tn, hipStream_t s) {
  if (tm == 64 && tn == 64) return launch_tiles<64, MODE, BKN, AKM, I8>(q, s);
  return tm == 32 && tn == 32 ? launch_tiles<32, MODE, BKN, AKM, I8>(q, s) : T3_ERR_UNSUPPORTED;
}

}  // namespace

t3_status launch_small_grouped(const Plan &q, int32_t tm, int32_t tn, bool b_kn, hipStream_t s) {
  return b_kn ? launch_small<kModeGrouped, 1, 0, 0>(q, tm, tn, s) : launch_small<kModeGrouped, 0, 0, 0>(q, tm, tn, s);
}
t3_status launch_small_grouped_i8(const Plan &q, int32_t tm, int32_t tn, hipStream_t s) {
  return launch_small<kModeGrouped, 0, 0, 1>(q, tm, tn, s);
}
t3_status launch_small_wgrad(const Plan &q, int32_t tm, int32_t tn, bool add, hipStream_t s) {
  return add ? launch_small<kModeWgradAdd, 1, 1, 0>(q, tm, tn, s) : launch_small<kModeWgrad, 1, 1, 0>(q, tm, tn, s);
}

}  // namespace t3k
