// Launches of the small-tile kernel on operands in 8 bits, A and B K-contiguous.
#include "t3_small.h"
#include "t3_launch.h"

namespace t3k {
namespace {

template <int BM, int BN, int MODE>
t3_status launch_small(const Plan &q, hipStream_t s) {
  const dim3 grid((unsigned)q.total_blocks), block(256);
  // (the plan by one vector request while all workgroups are on the chip at once: see small_tile_kernel)
  if (q.total_blocks <= q.resident * (BM == 32 ? 2 : 1)) return launch(small_tile_kernel<BM, BN, 4, 2, MODE, 0, 0, true, 1>, grid, block, s, q);
  return launch(small_tile_kernel<BM, BN, 4, 2, MODE, 0, 0, false, 1>, grid, block, s, q);
}

}  // namespace

t3_status launch_small_fused_i8(const Plan &q, int32_t tm, int32_t tn, hipStream_t s) {
  if (tm == 64 && tn == 64) return launch_small<64, 64, kModeFused>(q, s);
  return tm == 32 && tn == 32 ? launch_small<32, 32, kModeFused>(q, s) : T3_ERR_UNSUPPORTED;
}
t3_status launch_small_gemm_i8(const Plan &q, int32_t tm, int32_t tn, hipStream_t s) {
  if (tm == 64 && tn == 64) return launch_small<64, 64, kModeGemm>(q, s);
  return tm == 32 && tn == 32 ? launch_small<32, 32, kModeGemm>(q, s) : T3_ERR_UNSUPPORTED;
}

}  // namespace t3k
