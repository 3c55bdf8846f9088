// Host side of the C ABI declared in include/t3.h: argument validation, the launch plan
// (ring order, tile grid, XCD grouping, release granularity) and the kernel launches.
#include "t3.h"

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>
#include <stdio.h>

#include <atomic>
#include <mutex>

#include "t3_aux.h"
#include "t3_choice.h"
#include "t3_groups.h"
#include "t3_launch.h"
#include "t3_quant.h"

namespace t3k {
thread_local int32_t last_hip_error = 0;
}

namespace {

using t3k::ceil_div;
using t3k::launch;
using t3k::TileShape;

// preference order of t3_default_tile
constexpr TileShape kTileShapes[] = {{256, 256}, {256, 128}, {128, 256}, {128, 128}};
constexpr int kNumTileShapes = sizeof(kTileShapes) / sizeof(kTileShapes[0]);
constexpr int kDefaultCus = 256;       // compute units of an MI355X (host-only plan queries assume it)
constexpr int kMaxDevices = 64;
constexpr int kReleaseAgents = 32;     // release workgroups per chunk (t3_release_chunks)
constexpr int64_t kMaxCopyBlocks = 1 << 20;   // workgroups of t3_ag_step; more rows are walked
constexpr int kReduceWordsBlocks = 1024;   // workgroups up to which the reduction takes its plan by a vector request
constexpr int kNtMinK = 3072;          // K from which result stores take the streaming hint
constexpr int64_t kMemorySideCacheBytes = 256ll << 20;
// What the launch plan needs to know of the device it launches on, read from the runtime once
// per device (hardware attributes only; they never change while the process lives).
struct DeviceFacts {
  int cus;     // compute units: persistent workgroups are sized to them
  int xcds;    // accelerator dies the dispatcher deals workgroups to, round-robin
};
std::mutex g_facts_mutex;
DeviceFacts g_facts[kMaxDevices];
bool g_facts_known[kMaxDevices];

// Facts of the current device; T3_ERR_HIP if the runtime cannot tell.
t3_status device_facts(DeviceFacts *out) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess && (dev < 0 || dev >= kMaxDevices)) e = hipErrorInvalidDevice;
  if (e == hipSuccess) {
    std::lock_guard<std::mutex> lock(g_facts_mutex);
    if (!g_facts_known[dev]) {
      DeviceFacts f{0, 0};
      e = hipDeviceGetAttribute(&f.cus, hipDeviceAttributeMultiprocessorCount, dev);
      if (e == hipSuccess && hipDeviceGetAttribute(&f.xcds, hipDeviceAttributeNumberOfXccs, dev) != hipSuccess) {
        (void)hipGetLastError();
        f.xcds = 1;                // unknown: plan without XCD grouping
      }
      if (e == hipSuccess && f.cus < 1) e = hipErrorInvalidDevice;
      if (e == hipSuccess) {
        g_facts[dev] = f;
        g_facts_known[dev] = true;
      }
    }
    if (e == hipSuccess) *out = g_facts[dev];
  }
  if (e != hipSuccess) {
    t3k::last_hip_error = (int32_t)e;
    return T3_ERR_HIP;
  }
  return T3_OK;
}

// Where tile kernels record their timelines (t3_timeline), for the launches of every thread.
std::atomic<uint64_t *> g_timeline{nullptr};
std::atomic<int64_t> g_timeline_wgs{0};

void set_timeline(t3k::Plan &q) {
  q.timeline = g_timeline.load();
  const int64_t wgs = g_timeline_wgs.load();
  q.timeline_wgs = (int32_t)(wgs > (1ll << 30) ? (1ll << 30) : wgs);
}

// Tracker state for t3_gemm_rs_fused_static, the entry point for callers that cannot allocate:
// one array per device (each GPU the library runs on holds its own copy at its own address
// until the process ends).  Host code never uses the array's name as an address: the device
// address is looked up once per device and kept.
constexpr int kStaticMaxTp = T3_STATIC_MAX_TP;
constexpr int kStaticTrackWords = 2 * (3 * kStaticMaxTp + 2) + 2 + t3k::kTailSlots;
static __device__ __align__(256) uint32_t scratch[kStaticTrackWords];
uint32_t *g_scratch_ptr[kMaxDevices];

// Device address of the current device's `scratch`; T3_ERR_HIP if the runtime cannot tell.
t3_status static_track(uint32_t **out) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess && (dev < 0 || dev >= kMaxDevices)) e = hipErrorInvalidDevice;
  if (e == hipSuccess) {
    std::lock_guard<std::mutex> lock(g_facts_mutex);
    if (!g_scratch_ptr[dev]) {
      void *ptr = nullptr;
      e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));   // the current device's copy
      if (e == hipSuccess && !ptr) e = hipErrorInvalidSymbol;
      if (e == hipSuccess) g_scratch_ptr[dev] = static_cast<uint32_t *>(ptr);
    }
    if (e == hipSuccess) *out = g_scratch_ptr[dev];
  }
  if (e != hipSuccess) {
    t3k::last_hip_error = (int32_t)e;
    return T3_ERR_HIP;
  }
  return T3_OK;
}

// Flags of the tiles a balanced tail splits, for t3_gemm, which is given no tracker state to
// keep them in: a few sets of flag words per device.  Two launches may share a set only one
// after the other (the second half of a tile clears the flag the first half raised), so behind
// every launch an event is recorded, and a launch that takes a set whose last user may still be
// running is made to wait for that event first: a launch on the same stream would have waited
// anyway, launches on more streams than there are sets get serialised.  A launch whose stream is
// being captured runs without a balanced tail (a replayed graph would use the set while this
// bookkeeping knows nothing of it).
constexpr int kGemmTailSets = 8;
static __device__ __align__(256) uint32_t gemm_tail_flags[kGemmTailSets * t3k::kTailSlots];
struct GemmTail {
  uint32_t *base = nullptr;              // device address of the current device's gemm_tail_flags
  hipEvent_t done[kGemmTailSets] = {};   // recorded behind the last launch that used the set
  hipStream_t stream[kGemmTailSets] = {};
  bool used[kGemmTailSets] = {};
  unsigned next = 0;
};
GemmTail g_gemm_tail[kMaxDevices];

// Launches the plain GEMM `q` (balanced tail wanted) on stream s with a set of flags, or without
// a balanced tail if no set can be had.  The whole sequence runs under the lock, so that the
// event of a set always belongs to its last launch.
template <typename LaunchFn>
t3_status launch_with_gemm_tail(t3k::Plan &q, hipStream_t s, LaunchFn launch_fn) {
  auto plain = [&]() {
    (void)hipGetLastError();
    q.tail_r = q.tail_q = 0;
    q.tail_flags = nullptr;
    return launch_fn(q);
  };
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  int dev = 0;
  if (hipStreamIsCapturing(s, &cap) != hipSuccess || cap != hipStreamCaptureStatusNone ||
      hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices)
    return plain();
  std::lock_guard<std::mutex> lock(g_facts_mutex);
  GemmTail &g = g_gemm_tail[dev];
  if (!g.base) {
    void *ptr = nullptr;
    if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(gemm_tail_flags)) != hipSuccess || !ptr) return plain();
    g.base = static_cast<uint32_t *>(ptr);
  }
  // the set this stream used last, else the next in turn
  int set = -1;
  for (int i = 0; i < kGemmTailSets; ++i)
    if (g.used[i] && g.stream[i] == s) set = i;
  if (set < 0) set = (int)(g.next++ % kGemmTailSets);
  if (!g.used[set]) {
    if (hipEventCreateWithFlags(&g.done[set], hipEventDisableTiming) != hipSuccess) return plain();
  } else if (hipStreamWaitEvent(s, g.done[set], 0) != hipSuccess) {
    return plain();
  }
  g.used[set] = true;
  g.stream[set] = s;
  q.tail_flags = g.base + set * t3k::kTailSlots;
  const t3_status st = launch_fn(q);
  // (a launch that failed used nothing; a record that fails leaves the older record in place)
  if (st == T3_OK && hipEventRecord(g.done[set], s) != hipSuccess) (void)hipGetLastError();
  return st;
}

// T3_STAGGER="groups,window_ns" from the environment, read once per process.
struct StaggerEnv {
  bool set = false, off = false;
  int groups = 0, window_ns = 0;
};
const StaggerEnv &stagger_env() {
  static const StaggerEnv env = [] {
    StaggerEnv v;
    if (const char *e = getenv("T3_STAGGER")) {
      int eg = 0, ens = 0;
      const int n = sscanf(e, "%d,%d", &eg, &ens);
      if (n == 2 && eg > 1 && ens > 0) {
        v.set = true;
        v.groups = eg;
        v.window_ns = ens;
      } else if (n >= 1 && eg == 0) {
        v.set = v.off = true;
      }
    }
    return v;
  }();
  return env;
}

t3_status check_shape(const t3_problem *p) {
  if (!p) return T3_ERR_NULL;
  if (p->M < 0 || p->N < 0 || p->K < 0 || p->tp < 1 || p->rank < 0 || p->rank >= p->tp)
    return T3_ERR_BAD_SHAPE;
  if (p->N % p->tp != 0) return T3_ERR_BAD_SHAPE;
  return T3_OK;
}

bool tile_supported(int32_t tm, int32_t tn) {
  for (int i = 0; i < kNumTileShapes; ++i)
    if (kTileShapes[i].m == tm && kTileShapes[i].n == tn) return true;
  return false;
}

void default_tile(const t3_problem *p, int cus, int32_t *tm, int32_t *tn) {
  // The TRACKED tile of a caller who names none (workgroup tiles are workgroup_tile's).  A caller
  // sizes counters by it, so the rule stays as it is: cheapest shape by (work padded up to whole
  // tiles) x (cost per product relative to 256 x 256) x (how far the tiles fall short of filling `cus`
  // compute units), 128 x 256 counted in pairs.
  static const double kSlower[kNumTileShapes] = {1.0, 1.21, 1.0, 1.28};
  const int64_t W = p->N / p->tp;
  double best = -1.0;
  *tm = 128;
  *tn = 128;
  for (int i = 0; i < kNumTileShapes; ++i) {
    const int64_t Mt = ceil_div(p->M, kTileShapes[i].m), Wt = ceil_div(W, kTileShapes[i].n);
    const int64_t T = Mt * Wt * p->tp;
    if (T == 0) continue;
    const bool paired = kTileShapes[i].m == 128 && kTileShapes[i].n == 256 && Mt > 1;
    const int64_t rows = paired ? ceil_div(p->M, 256) * 256 : Mt * kTileShapes[i].m;
    const int64_t groups = paired ? ceil_div(Mt, 2) * Wt * p->tp : T;     // workgroup tiles
    const double padded = (double)rows * (double)(Wt * kTileShapes[i].n) / ((double)p->M * (double)W);
    const double score = padded * kSlower[i] * (groups < cus ? (double)cus / (double)groups : 1.0);
    if (best < 0 || score < best) {
      best = score;
      *tm = kTileShapes[i].m;
      *tn = kTileShapes[i].n;
    }
  }
}

t3_status resolve_tile(const t3_problem *p, int32_t *tm, int32_t *tn) {
  if (p->tile_m == 0 && p->tile_n == 0) {
    default_tile(p, kDefaultCus, tm, tn);
    return T3_OK;
  }
  if (!tile_supported(p->tile_m, p->tile_n)) return T3_ERR_BAD_TILE;
  *tm = p->tile_m;
  *tn = p->tile_n;
  return T3_OK;
}

// the kernels test the same flag bits under their own names
static_assert(T3_FLAG_STEP0_STORE_ONLY == t3k::kFlagStep0StoreOnly &&
                  T3_FLAG_FWD_DIRECT == t3k::kFlagFwdDirect &&
                  T3_FLAG_TWO_WRITERS == t3k::kFlagTwoWriters && T3_FLAG_FWD_BF16 == t3k::kFlagFwdBf16,
              "flag bits of the header and of the kernels");
static_assert(sizeof(t3_problem) == 104, "layout documented in the header");
static_assert(T3_TIMELINE_ITEMS == t3k::kTimelineItems, "timeline layout of the header and of the kernels");

inline bool aligned16(const void *q) { return (reinterpret_cast<uintptr_t>(q) & 15u) == 0; }

enum Need { kNeedAB = 1, kNeedR = 2, kNeedC = 4, kNeedFwd = 8, kNeedTrack = 16,
            kNeedTwoWriters = 32 /* the call exists only in two-writer mode */ };

// The flag words of a balanced tail in tracker state: behind the two banks, gen and error.
inline uint32_t *tail_flags_in(uint32_t *track, int32_t tp) { return track + 2 * (3 * (int64_t)tp + 2) + 2; }

// Validates everything and fills the plan.  *empty is set when there is nothing to launch.
t3_status make_plan(const t3_problem *p, t3k::Call call, int need, const void *A, const void *B, const float *C,
                    float *R, void *fwd, uint32_t *track, t3k::Plan *plan, int32_t *tm,
                    int32_t *tn, bool *empty, bool i8 = false) {
  t3_status st = check_shape(p);
  if (st != T3_OK) return st;
  st = resolve_tile(p, tm, tn);
  if (st != T3_OK) return st;
  const bool fused_like = (need & kNeedTrack) != 0;
  const bool direct = fused_like && (p->flags & T3_FLAG_FWD_DIRECT);
  const bool two_writers = fused_like && (p->flags & T3_FLAG_TWO_WRITERS);
  // (in 8 bits an array without elements needs no address)
  const bool some = !i8 || (p->M && p->N);
  if ((need & kNeedAB) && some && (!i8 || p->K) && (!A || !B)) return T3_ERR_NULL;
  if ((need & kNeedR) && some && !R) return T3_ERR_NULL;
  if ((need & kNeedC) && some && !C) return T3_ERR_NULL;
  if ((need & kNeedTrack) && !track) return T3_ERR_NULL;
  if ((need & kNeedFwd) && some && p->tp > 1 && !fwd && !(two_writers && (need & kNeedAB)))
    return T3_ERR_NULL;                         // (the fused call releases nothing with two writers)
  if (p->flags & ~(T3_FLAG_STEP0_STORE_ONLY | T3_FLAG_FWD_DIRECT | T3_FLAG_TWO_WRITERS |
                   T3_FLAG_FWD_BF16))
    return T3_ERR_UNSUPPORTED;
  if (two_writers && direct) return T3_ERR_UNSUPPORTED;   // both writers must target R
  if ((need & kNeedTwoWriters) && !two_writers) return T3_ERR_UNSUPPORTED;
  // split-K: several workgroups add into one tile, so it needs the atomic updates of two-writer
  // mode, and every part needs at least one full K-slab of 64
  const int32_t split_k = p->split_k > 1 ? p->split_k : 1;
  if (p->split_k < 0) return T3_ERR_BAD_SHAPE;
  if (split_k > 1 && fused_like && (!two_writers || split_k > p->K / 64 || split_k > 64))
    return T3_ERR_UNSUPPORTED;
  // the unfused reduction kernel has no second writer to wait for
  if (two_writers && (need & kNeedC) && (need & kNeedFwd) && !(need & kNeedTwoWriters))
    return T3_ERR_UNSUPPORTED;

  const int64_t W = p->N / p->tp;
  if (need & kNeedAB) {
    if (p->b_layout != T3_B_NK && p->b_layout != T3_B_KN) return T3_ERR_BAD_SHAPE;
    if (p->a_layout != T3_A_MK && p->a_layout != T3_A_KM) return T3_ERR_BAD_SHAPE;
    if (p->reserved != 0) return T3_ERR_BAD_SHAPE;
    const bool kn = p->b_layout == T3_B_KN, km = p->a_layout == T3_A_KM;
    if (p->lda < (km ? p->M : p->K) || p->ldb < (kn ? p->N : p->K)) return T3_ERR_BAD_SHAPE;
    if (p->K % 8 || p->lda % 8 || p->ldb % 8 || !aligned16(A) || !aligned16(B)) return T3_ERR_ALIGN;
    // A stored K x M: 16-byte pieces run along M, and whole K-slabs of 64 only
    if (km && p->M % 8) return T3_ERR_ALIGN;
    if (km && p->K % 64) return T3_ERR_UNSUPPORTED;
    // B stored K x N: 16-byte pieces run along N, so chunks must be cut on multiples of 8
    // columns, and the transposed operand path takes whole K-slabs of 64 only
    if (kn && W % 8) return T3_ERR_ALIGN;
    if (kn && p->K % 64) return T3_ERR_UNSUPPORTED;
    // kernels address A and B with 32-bit element offsets
    if ((int64_t)(km ? p->K : p->M) * p->lda >= (1ll << 31) ||
        (int64_t)(kn ? p->K : p->N) * p->ldb >= (1ll << 31))
      return T3_ERR_UNSUPPORTED;
  }
  // kernels address R, C and a forward slot with 32-bit byte offsets
  if (need & kNeedR) {
    if (p->ldr < p->N) return T3_ERR_BAD_SHAPE;
    if (p->ldr % 4 || W % 4 || !aligned16(R)) return T3_ERR_ALIGN;
    if ((int64_t)p->M * p->ldr * 4 >= (1ll << 32)) return T3_ERR_UNSUPPORTED;
  }
  if (need & kNeedC) {
    if (p->ldc < p->N) return T3_ERR_BAD_SHAPE;
    if (p->ldc % 4 || W % 4 || !aligned16(C)) return T3_ERR_ALIGN;
    if ((int64_t)p->M * p->ldc * 4 >= (1ll << 32)) return T3_ERR_UNSUPPORTED;
  }
  if ((need & kNeedFwd) && fwd && !aligned16(fwd)) return T3_ERR_ALIGN;
  // bfloat16 forward slots move 8 elements per 16-byte access
  if ((need & kNeedFwd) && fused_like && (p->flags & T3_FLAG_FWD_BF16) && W % 8) return T3_ERR_ALIGN;

  // (the last refusals, before the device is asked anything: tracked tiles, which the issue order, the tile
  // range and the tracker's thresholds are counted in, fit 31 bits, with split-K in as many parts too; the workgroup tiles
  // of arrays below 4 GiB always do)
  const int64_t T_t = ceil_div(p->M, *tm) * ceil_div(W, *tn) * p->tp;
  if (T_t >= (1ll << 31)) return T3_ERR_UNSUPPORTED;
  if (two_writers && T_t * split_k >= (1ll << 31)) return T3_ERR_UNSUPPORTED;
  if ((need & kNeedTwoWriters) && (need & kNeedC) && p->upstream_agents < 0) return T3_ERR_BAD_SHAPE;

  DeviceFacts dev{kDefaultCus, t3k::kNumXcd};
  if (T_t) {                                     // (nothing is launched otherwise: no device needed)
    st = device_facts(&dev);
    if (st != T3_OK) return st;
  }
  const t3k::LaunchShape shape = t3k::launch_shape(p, call, {*tm, *tn}, dev.cus, i8);
  *tm = shape.tile.m;
  *tn = shape.tile.n;
  const int64_t Mt = shape.Mt, Wt = shape.Wt, tpc = shape.tpc;
  *empty = shape.begin >= shape.limit;           // (no tiles, or an empty range of them)

  t3k::Plan &q = *plan;
  q = t3k::Plan{};                               // (callers give memory with an earlier call's plan in it, and not every kernel has every field set)
  q.A = static_cast<const uint16_t *>(A);
  q.B = static_cast<const uint16_t *>(B);
  q.C = C;
  q.R = R;
  q.fwd = static_cast<float *>(fwd);     // (bfloat16 under T3_FLAG_FWD_BF16)
  q.track = track;
  q.lda = p->lda;
  q.ldb = p->ldb;
  q.ldr = p->ldr;
  q.ldc = p->ldc;
  q.limit = shape.limit;
  q.begin = shape.begin;
  q.M = p->M;
  q.N = p->N;
  q.K = p->K;
  q.P = p->tp;
  q.rank = p->rank;
  q.W = (int32_t)W;
  q.own = (p->rank + p->tp - 1) % p->tp;
  q.Mt = (int32_t)Mt;
  q.Wt = (int32_t)Wt;
  q.tpc = (int32_t)tpc;
  q.tile_m = *tm;
  q.tile_n = *tn;
  q.tracked = (int32_t)shape.tracked_tpc;
  q.flags = fused_like ? p->flags : 0u;

  const t3k::XcdBlocks blocks = t3k::xcd_blocks(p, shape, dev.xcds);
  q.xcd_nbm = blocks.by_rows;
  q.xcd_bmk = blocks.rows;
  q.xcd_bnk = blocks.columns;
  const int64_t range_steps = tpc > 0 ? ceil_div(q.limit, tpc) - q.begin / tpc : 0;

  // (an empty problem has no tiles to divide by)
  q.by_tpc = t3k::fast_div((uint32_t)(tpc > 0 ? tpc : 1));
  q.by_column = t3k::fast_div((uint32_t)(tpc == 0 ? 1 : (q.xcd_nbm ? q.xcd_bmk : Mt)));

  const int64_t resident = shape.resident;
  q.stage0 = (int32_t)shape.stage0;
  q.total_blocks = (int32_t)shape.total_blocks;
  // Start-up phase offsets (see stagger_start); T3_STAGGER="groups,window_ns" overrides them ("0" turns them off).
  {
    t3k::StartOffsets o = t3k::start_offsets(p, call, shape);
    const StaggerEnv &env = stagger_env();
    if (env.set) o = env.off ? t3k::StartOffsets{0, 0.0} : t3k::StartOffsets{env.groups, (double)env.window_ns};
    if (o.groups > 1 && o.window_ns >= 100.0) {
      q.stagger_groups = o.groups;
      q.stagger_ticks = (int32_t)(o.window_ns / 10.0 / o.groups);   // 100 MHz ticks between consecutive groups
      q.stagger_blocks = (int32_t)resident;
    }
  }
  q.expected_done = (int32_t)(q.limit - q.begin);
  // updates expected per element (Sec. 4.2.1): with two writers the launches of both count in
  // one bank, which closes when the tiles of both have been counted
  q.upd_first = q.upd_rest = 1;
  q.split_k = 1;
  if (two_writers) {
    q.split_k = split_k;                        // local updates per element = parts of K (Sec. 7.7)
    const bool step0 = (p->flags & T3_FLAG_STEP0_STORE_ONLY) != 0;
    q.upd_rest = split_k + 1;
    q.upd_first = split_k + (step0 ? 0 : 1);
    const int64_t up_begin = (step0 && q.begin < tpc) ? (tpc < q.limit ? tpc : q.limit) : q.begin;
    q.expected_done = (int32_t)((q.limit - q.begin) * split_k + (q.limit - up_begin));
  }
  // K walks start at a different slab on every XCD (see the kernels' `koff`)
  q.k_groups = dev.xcds > 1 ? dev.xcds : 0;
  q.by_groups = t3k::fast_div((uint32_t)(q.k_groups > 1 ? q.k_groups : 1));
  q.resident = (int32_t)resident;
  // Results leave the XCD's L2 at once (streaming hint) where that L2 is better spent on slabs
  // of A and B: long K loops, or an output that the memory-side cache cannot hold anyway.
  // The plain GEMM of 16384 x 3072 x 1536 and the reduction that reads C next: 275 us with the hint, 257
  // without.  (The wide-tile kernel streams fused results always: 4096 x 12288 x 1536 166 us with, 174
  // without; gemm_tile_kernel loses 6 % there with it, and gains 3 % where K or the output is large.)
  q.nt_out = (!two_writers &&
              (p->K >= kNtMinK || 4ll * p->M * p->N > kMemorySideCacheBytes)) ? 1 : 0;
  set_timeline(q);
  q.wide = shape.kernel == t3k::kWideTile;
  if (q.wide) {
    q.order = t3k::tile_order(p, call, shape, t3k::xcd_rows(p, call, shape, blocks));
    q.granule = (p->flags & T3_FLAG_FWD_BF16) && fused_like ? 32 : 16;
    q.overlap = t3k::column_overlap(p, call, shape.tile, Wt);
  }
  q.col_align = q.wide ? t3k::column_align(p, call, shape.tile, Wt) : 0;
  q.tail_r = (int32_t)shape.tail_r;
  q.tail_q = (int32_t)shape.tail_q;
  q.tail_flags = track ? tail_flags_in(track, p->tp) : nullptr;   // (t3_gemm brings its own)
  // Counting.  Groups pay where many tiles finish together; up to 32 ring steps x 8 groups, 16 x 16
  // or 8 x 32 fit the words.
  q.whole_chunks = !two_writers && tpc > 0 && q.begin % tpc == 0 && q.limit % tpc == 0;
  q.sub_groups = 1;
  q.sub_shift = 0;
  if (q.whole_chunks && track && !q.tail_r && range_steps <= 32 && tpc >= 24) {
    q.sub_groups = 8;
    for (int g = 16; g <= 32 && tpc >= 8 * g && range_steps * g <= t3k::kTailSlots; g *= 2) {
      q.sub_groups = g;
      ++q.sub_shift;
    }
  }
  return T3_OK;
}

inline unsigned grid_size(const t3k::Plan &q) { return (unsigned)q.total_blocks; }

t3_status launch_gemm(int mode, const t3k::Plan &q, int32_t tm, int32_t tn, bool b_kn, bool a_km, hipStream_t s) {
  using namespace t3k;
  if (q.wide) {
    if (mode == kModeFused && q.overlap)
      return a_km ? (b_kn ? launch_wide_overlap_km_kn(q, tm, tn, s) : launch_wide_overlap_km(q, tm, tn, s))
                  : (b_kn ? launch_wide_overlap_kn(q, tm, tn, s) : launch_wide_overlap(q, tm, tn, s));
    if (mode == kModeFused)
      return a_km ? (b_kn ? launch_wide_fused_km_kn(q, tm, tn, s) : launch_wide_fused_km(q, tm, tn, s))
                  : (b_kn ? launch_wide_fused_kn(q, tm, tn, s) : launch_wide_fused(q, tm, tn, s));
    Plan g = q;
    g.ldr = q.ldc;                      // C through R
    return a_km ? (b_kn ? launch_wide_gemm_km_kn(g, tm, tn, s) : launch_wide_gemm_km(g, tm, tn, s))
                : (b_kn ? launch_wide_gemm_kn(g, tm, tn, s) : launch_wide_gemm_nk(g, tm, tn, s));
  }
  if (tm < 128)
    return mode == kModeFused ? launch_small_fused(q, tm, tn, b_kn, a_km, s) : launch_small_gemm(q, tm, tn, b_kn, a_km, s);
  if (mode == kModeFused)
    return a_km ? (b_kn ? launch_fused_km_kn(q, tm, tn, s) : launch_fused_km(q, tm, tn, s))
                : (b_kn ? launch_fused_kn(q, tm, tn, s) : launch_fused(q, tm, tn, s));
  return a_km ? (b_kn ? launch_gemm_km_kn(q, tm, tn, s) : launch_gemm_km(q, tm, tn, s))
              : (b_kn ? launch_gemm_kn(q, tm, tn, s) : launch_gemm_nk(q, tm, tn, s));
}

// ---- products in 8 bits
constexpr int32_t kMaxK8 = 131056;     // (K of 131072 times -128 -128 is 2^31)
constexpr int64_t kFarLd = 1ll << 32;  // leading dimensions from which products with a number of rows might not be 64-bit numbers
constexpr int64_t kFarStride = 1ll << 48;
inline bool aligned4(const void *q) { return (reinterpret_cast<uintptr_t>(q) & 3u) == 0; }

// What a call in 8 bits has to check beside make_plan, and the problem as make_plan takes it: A and B in pairs of int8, which are where
// a bf16 would be.
t3_status pairs_of(const t3_problem *p, bool fused, const float *scale_a, const float *scale_b, t3_problem *pairs) {
  t3_status st = check_shape(p);
  if (st != T3_OK) return st;
  if (p->M && p->N && (!scale_a || !scale_b)) return T3_ERR_NULL;
  int32_t tm, tn;
  st = resolve_tile(p, &tm, &tn);
  if (st != T3_OK) return st;
  if ((p->a_layout != T3_A_MK && p->a_layout != T3_A_KM) || (p->b_layout != T3_B_NK && p->b_layout != T3_B_KN)) return T3_ERR_BAD_SHAPE;
  if (p->a_layout != T3_A_MK || p->b_layout != T3_B_NK) return T3_ERR_UNSUPPORTED;
  if (fused && ((p->flags & T3_FLAG_TWO_WRITERS) || p->split_k > 1)) return T3_ERR_UNSUPPORTED;
  if (p->lda < p->K || p->ldb < p->K) return T3_ERR_BAD_SHAPE;
  if (p->K % 16 || p->lda % 16 || p->ldb % 16 || !aligned4(scale_a) || !aligned4(scale_b)) return T3_ERR_ALIGN;
  if (p->K > kMaxK8 || p->lda >= kFarLd || p->ldb >= kFarLd) return T3_ERR_UNSUPPORTED;
  // ranges of whole ring steps (a range that cuts one is in tracked tiles, which the kernels here do not work in)
  const int64_t tpc = ceil_div(p->M, tm) * ceil_div(p->N / p->tp, tn), T = tpc * p->tp;
  const int64_t limit = p->tile_limit < 0 || p->tile_limit > T ? T : p->tile_limit, begin = p->tile_begin < 0 ? 0 : p->tile_begin;
  if (tpc && begin < limit && (begin % tpc || limit % tpc)) return T3_ERR_UNSUPPORTED;
  *pairs = *p;
  pairs->K /= 2;
  pairs->lda /= 2;
  pairs->ldb /= 2;
  return T3_OK;
}

// ---- products by group
// The sizes of a grouped product's operands, and what has to hold for them.  size: bytes of an element of A and of B (of dC, in the
// gradient of the weights, whose result is fp32 in B's place).
t3_status check_grouped(const t3_grouped *g, bool wgrad, int size) {
  if (!g) return T3_ERR_NULL;
  if (g->rows < 0 || g->groups < 1 || g->N < 0 || g->K < 0) return T3_ERR_BAD_SHAPE;
  if (g->b_layout != T3_B_NK && g->b_layout != T3_B_KN) return T3_ERR_BAD_SHAPE;
  const bool kn = g->b_layout == T3_B_KN;
  const int64_t b_rows = kn ? g->K : g->N, b_cols = kn ? g->N : g->K;
  if (g->lda < g->K || g->ldb < b_cols || g->ldc < g->N || g->stride_b < 0) return T3_ERR_BAD_SHAPE;
  if (wgrad && g->groups > 1 && b_rows && g->ldb < kFarLd && g->stride_b < (b_rows - 1) * g->ldb + b_cols) return T3_ERR_BAD_SHAPE;
  if (g->flags & ~(wgrad ? T3_GROUPED_ACCUMULATE : 0u)) return T3_ERR_UNSUPPORTED;
  if (g->groups > T3_MAX_GROUPS || (size == 1 && (kn || g->K > kMaxK8))) return T3_ERR_UNSUPPORTED;
  if (g->lda >= kFarLd || g->ldb >= kFarLd || g->ldc >= kFarLd || g->stride_b >= kFarStride) return T3_ERR_UNSUPPORTED;
  const int per = 16 / size;                     // elements of 16 bytes
  if (g->K % per || g->lda % per) return T3_ERR_ALIGN;
  if (wgrad) {
    if (g->N % 8 || g->ldc % 8 || g->ldb % 4 || g->stride_b % 4) return T3_ERR_ALIGN;
  } else {
    if (g->ldb % per || g->stride_b % per || g->N % 4 || g->ldc % 4 || (kn && g->N % 8)) return T3_ERR_ALIGN;
  }
  // 32-bit offsets in the kernels: A and a group's B (and dC) below 2^32 bytes and 2^31 elements of 2 bytes, fp32 results below 2^32 bytes
  // (B's in the gradient of a group)
  if (g->rows * g->lda >= (1ll << 32) / size || g->rows * g->ldc >= (wgrad ? 1ll << 31 : 1ll << 30) || b_rows * g->ldb >= (wgrad ? 1ll << 30 : (1ll << 32) / size))
    return T3_ERR_UNSUPPORTED;
  // (so tiles, 32 x 32 the smallest, are less than 2^31: at most 256 gradients of 2^22, or 2^27 of a result's)
  return T3_OK;
}

// What the launches of products by group have in common: how grid positions fall to the workgroups, and whether results leave the caches.
// bytes: of operands and result.  Results stream where all of it is more than the memory-side cache holds.  In us, kept and streamed, and with a reader
// of the result right behind (to bfloat16), which is what counts; operands in memory: 4096 rows of 8 groups x 5120 x 1280, 199 MB, 87 and 85, with the reader
// 106 and 108; 8192 of 16 x 5120 x 1280, 398 MB, 157 and 151, 196 and 193; 16384 of 8 x 8192 x 1024, 705 MB, 317 and 321, 463 and 451; 16384 of 16 x 6144 x 2048,
// 872 MB, 408 and 400, 505 and 490; gradients of weights: 4096 of 8 x 2560 x 1280, 136 MB, 59 and 45, 82 and 82; 8190 of 16 x 5120 x 1280, 524 MB, 171 and
// 163, 287 and 268; 16384 of 32 x 4096 x 2048, 1275 MB, 409 and 381, 697 and 651.  On one set of operands again and again 2 to 3 us more than kept, with the
// reader, up to 199 MB, and 1 to 6 % less from 398 MB on.
void plan_rounds(t3k::Plan &q, const t3k::Choice &c, const DeviceFacts &dev, int64_t most_tiles, int64_t bytes) {
  q.tile_m = c.tile.m;
  q.tile_n = c.tile.n;
  q.wide = c.kernel == t3k::kWideTile;
  q.Wt = (int32_t)ceil_div(q.N, c.tile.n);
  q.resident = dev.cus * (c.tile.m == 128 && c.tile.n == 128 ? 2 : 1);
  q.cut = t3k::quarters_of(c.tile) && most_tiles > q.resident ? t3k::kCutLeave : t3k::kCutNone;
  q.order.round = (uint32_t)q.resident;
  q.order.by_round = t3k::fast_div(q.order.round);
  q.total_blocks = (int32_t)((most_tiles + 7) / 8 * 8);
  q.k_groups = dev.xcds > 1 ? dev.xcds : 0;
  q.by_groups = t3k::fast_div((uint32_t)(q.k_groups > 1 ? q.k_groups : 1));
  q.nt_out = bytes > kMemorySideCacheBytes ? 1 : 0;
  set_timeline(q);
}

// The launch, and behind it the one of a last round's tiles in quarters (which has nothing to do if that round is fuller, or if there is none).
t3_status launch_rounds(t3k::Plan &q, t3_status (*launch_fn)(const t3k::Plan &, int32_t, int32_t, hipStream_t), hipStream_t s) {
  const t3_status st = launch_fn(q, q.tile_m, q.tile_n, s);
  if (st != T3_OK || q.cut != t3k::kCutLeave) return st;
  q.cut = t3k::kCutQuarters;
  q.total_blocks = q.resident *= 2;              // (two workgroups of 128 x 128 to a compute unit)
  return launch_fn(q, 128, 128, s);
}

static_assert(T3_MAX_GROUPS == t3k::kMaxGroups, "groups of the header and of the kernels");

t3_status grouped_product(const t3_grouped *g, bool i8, const int32_t *offsets, const void *A, const float *scale_a, const void *B,
                          const float *scale_b, float *C, void *stream) {
  t3_status st = check_grouped(g, false, i8 ? 1 : 2);
  if (st != T3_OK) return st;
  // (arrays without elements need no address, nor do those that nothing is read of: a rank that got no rows has none)
  const bool some = g->rows && g->N;
  if (!offsets || (some && (!C || (i8 && (!scale_a || !scale_b)))) || (some && g->K && (!A || !B))) return T3_ERR_NULL;
  if (!aligned4(offsets) || !aligned16(A) || !aligned16(B) || !aligned16(C) || (i8 && (!aligned4(scale_a) || !aligned4(scale_b)))) return T3_ERR_ALIGN;
  if (!some) return T3_OK;
  const int per = i8 ? 2 : 1;
  t3k::Plan q{};
  q.A = static_cast<const uint16_t *>(A);
  q.B = static_cast<const uint16_t *>(B);
  q.R = C;
  q.lda = g->lda / per;
  q.ldb = g->ldb / per;
  q.ldr = q.ldc = g->ldc;
  q.M = q.rows = g->rows;
  q.N = q.W = g->N;
  q.K = g->K / per;
  q.P = 1;
  q.split_k = 1;
  q.scale_a = scale_a;
  q.scale_b = scale_b;
  q.offsets = offsets;
  q.stride_b = g->stride_b / per;
  q.groups = g->groups;
  const bool kn = g->b_layout == T3_B_KN;
  DeviceFacts dev;
  st = device_facts(&dev);
  if (st != T3_OK) return st;
  const bool wide_ok = t3k::grouped_wide_fits(kn, q.K, q.lda, q.ldb, q.ldc);
  const t3k::Choice c = t3k::grouped_tile(false, kn, g->rows, g->N, q.K, g->groups, dev.cus, wide_ok);
  const int32_t tm = c.tile.m, tn = c.tile.n;
  // rows of tiles: every group may end with a tile of its own that is not full, and has no more tiles than rows
  plan_rounds(q, c, dev, (ceil_div(g->rows, tm) + (g->rows < g->groups ? g->rows : g->groups)) * ceil_div(g->N, tn),
              2ll * q.rows * q.K + 2ll * q.groups * q.N * q.K + 4ll * q.rows * q.N);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (q.wide) return launch_rounds(q, i8 ? t3k::launch_wide_grouped_i8 : (kn ? t3k::launch_wide_grouped_kn : t3k::launch_wide_grouped_nk), s);
  return i8 ? t3k::launch_small_grouped_i8(q, tm, tn, s) : t3k::launch_small_grouped(q, tm, tn, kn, s);
}

}  // namespace

extern "C" {

const char *t3_status_string(t3_status s) {
  switch (s) {
    case T3_OK: return "ok";
    case T3_ERR_NULL: return "null pointer";
    case T3_ERR_BAD_SHAPE: return "bad shape";
    case T3_ERR_BAD_TILE: return "unsupported tile shape";
    case T3_ERR_ALIGN: return "misaligned pointer or leading dimension";
    case T3_ERR_UNSUPPORTED: return "unsupported request";
    case T3_ERR_HIP: return "HIP runtime error";
  }
  return "unknown status";
}

int32_t t3_last_hip_error(void) { return t3k::last_hip_error; }

t3_status t3_chunk_order(int32_t tp, int32_t rank, int32_t *order, int32_t *own) {
  if (!order || !own) return T3_ERR_NULL;
  if (tp < 1 || rank < 0 || rank >= tp) return T3_ERR_BAD_SHAPE;
  for (int32_t s = 0; s < tp; ++s) order[s] = (rank + s) % tp;
  *own = (rank + tp - 1) % tp;
  return T3_OK;
}

t3_status t3_default_tile(const t3_problem *p, int32_t *tile_m, int32_t *tile_n) {
  if (!tile_m || !tile_n) return T3_ERR_NULL;
  const t3_status st = check_shape(p);
  if (st != T3_OK) return st;
  default_tile(p, kDefaultCus, tile_m, tile_n);
  return T3_OK;
}

t3_status t3_tiles_per_chunk(const t3_problem *p, int64_t *tpc) {
  if (!tpc) return T3_ERR_NULL;
  t3_status st = check_shape(p);
  if (st != T3_OK) return st;
  int32_t tm, tn;
  st = resolve_tile(p, &tm, &tn);
  if (st != T3_OK) return st;
  *tpc = ceil_div(p->M, tm) * ceil_div(p->N / p->tp, tn);
  return T3_OK;
}

t3_status t3_tile_of(const t3_problem *p, int64_t t, int32_t *s, int32_t *c, int32_t *mi,
                     int32_t *nj) {
  if (!s || !c || !mi || !nj) return T3_ERR_NULL;
  int64_t tpc;
  const t3_status st = t3_tiles_per_chunk(p, &tpc);
  if (st != T3_OK) return st;
  if (t < 0 || t >= tpc * p->tp) return T3_ERR_BAD_SHAPE;
  int32_t tm, tn;
  resolve_tile(p, &tm, &tn);
  const int64_t Mt = ceil_div(p->M, tm);
  const int64_t q = t % tpc;
  *s = (int32_t)(t / tpc);
  *c = (p->rank + *s) % p->tp;
  *mi = (int32_t)(q % Mt);
  *nj = (int32_t)(q / Mt);
  return T3_OK;
}

int64_t t3_track_words(int32_t tp) { return tp < 1 ? 0 : 2 * (3ll * tp + 2) + 2 + t3k::kTailSlots; }

t3_status t3_track_reset(int32_t tp, uint32_t *track, void *stream) {
  if (!track) return T3_ERR_NULL;
  if (tp < 1 || tp > (1 << 20)) return T3_ERR_BAD_SHAPE;
  return launch(t3k::track_reset_kernel, dim3(1), dim3(256), static_cast<hipStream_t>(stream), track,
                (int)tp);
}

t3_status t3_gemm_rs_fused(const t3_problem *p, const void *A, const void *B, float *R,
                           void *fwd, uint32_t *track, void *stream) {
  t3k::Plan q;
  int32_t tm, tn;
  bool empty = false;
  const t3_status st = make_plan(p, t3k::kCallFused, kNeedAB | kNeedR | kNeedFwd | kNeedTrack, A, B, nullptr, R,
                                 fwd, track, &q, &tm, &tn, &empty);
  if (st != T3_OK) return st;
  if (empty) return T3_OK;
  return launch_gemm(t3k::kModeFused, q, tm, tn, p->b_layout == T3_B_KN, p->a_layout == T3_A_KM,
                                      static_cast<hipStream_t>(stream));
}

t3_status t3_gemm_rs_fused_static(const t3_problem *p, const void *A, const void *B, float *R,
                                  void *fwd, uint32_t *track_copy, void *stream) {
  if (!p) return T3_ERR_NULL;
  if (p->tp > kStaticMaxTp) return T3_ERR_UNSUPPORTED;   // the static tracker state holds no more
  if (p->flags & T3_FLAG_TWO_WRITERS) return T3_ERR_UNSUPPORTED;   // needs a tracker that outlives the call
  // validate everything first (a non-null stand-in for the tracker pointer: nothing reads it)
  t3k::Plan q;
  int32_t tm, tn;
  bool empty = false;
  uint32_t stand_in = 0;
  t3_status st = make_plan(p, t3k::kCallFused, kNeedAB | kNeedR | kNeedFwd | kNeedTrack, A, B, nullptr, R, fwd,
                           &stand_in, &q, &tm, &tn, &empty);
  if (st != T3_OK) return st;
  uint32_t *track = nullptr;
  st = static_track(&track);
  if (st != T3_OK) return st;
  q.track = track;
  q.tail_flags = tail_flags_in(track, p->tp);
  hipStream_t s = static_cast<hipStream_t>(stream);
  // the array keeps the last call's contents: every call starts from a cleared tracker
  st = launch(t3k::track_reset_kernel, dim3(1), dim3(256), s, track, (int)p->tp);
  if (st != T3_OK) return st;
  if (!empty) {
    st = launch_gemm(t3k::kModeFused, q, tm, tn, p->b_layout == T3_B_KN, p->a_layout == T3_A_KM, s);
    if (st != T3_OK) return st;
  }
  if (track_copy)
    st = launch(t3k::track_copy_kernel, dim3(1), dim3(256), s, (const uint32_t *)track, track_copy,
                (int)t3_track_words(p->tp));
  return st;
}

t3_status t3_gemm(const t3_problem *p, const void *A, const void *B, float *C, void *stream) {
  // (flags and split_k are ignored: make_plan sees no tracker for this call)
  t3k::Plan q;
  int32_t tm, tn;
  bool empty = false;
  const t3_status st = make_plan(p, t3k::kCallGemm, kNeedAB | kNeedC, A, B, C, nullptr, nullptr, nullptr, &q,
                                 &tm, &tn, &empty);
  if (st != T3_OK) return st;
  if (empty) return T3_OK;
  q.R = C;   // the GEMM kernel's output pointer, addressed with ldc
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool b_kn = p->b_layout == T3_B_KN, a_km = p->a_layout == T3_A_KM;
  auto go = [&](const t3k::Plan &plan) { return launch_gemm(t3k::kModeGemm, plan, tm, tn, b_kn, a_km, s); };
  return q.tail_r ? launch_with_gemm_tail(q, s, go) : go(q);
}

t3_status t3_quant_rows(int32_t rows, int32_t cols, int32_t x_type, const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale,
                        void *stream) {
  if (rows < 0 || cols < 0 || (x_type != T3_TYPE_BF16 && x_type != T3_TYPE_F32) || ldx < cols || ldq < cols) return T3_ERR_BAD_SHAPE;
  if (rows && (!scale || (cols && (!x || !q)))) return T3_ERR_NULL;
  const bool f32 = x_type == T3_TYPE_F32;
  if (cols % 8 || ldx % (f32 ? 4 : 8) || ldq % 8 || !aligned16(x) || (reinterpret_cast<uintptr_t>(q) & 7u) || !aligned4(scale)) return T3_ERR_ALIGN;
  if (ldx >= kFarLd || ldq >= kFarLd) return T3_ERR_UNSUPPORTED;
  if (!rows) return T3_OK;
  // a wavefront per row of up to four pieces a lane, else a workgroup; as many pieces as the row has
  const bool wave = cols <= 8 * 64 * 4;
  const int64_t held = ceil_div(cols, 8 * (wave ? 64 : 256));
  auto pick = [&](auto type) {
    constexpr bool kF32 = decltype(type)::value;
    if (wave) return held <= 1 ? t3k::quant_rows_kernel<64, 1, kF32> : (held <= 2 ? t3k::quant_rows_kernel<64, 2, kF32> : t3k::quant_rows_kernel<64, 4, kF32>);
    return held <= 2 ? t3k::quant_rows_kernel<256, 2, kF32> : (held <= 4 ? t3k::quant_rows_kernel<256, 4, kF32> : t3k::quant_rows_kernel<256, t3k::kQuantPieces, kF32>);
  };
  auto kernel = f32 ? pick(std::true_type{}) : pick(std::false_type{});
  // (a launch has less than 2^32 lanes: 2^23 workgroups at a time)
  const int64_t part = (wave ? 4ll : 1ll) << 23;
  for (int64_t at = 0; at < rows; at += part) {
    const int32_t here = (int32_t)(rows - at < part ? rows - at : part);
    const t3_status st = launch(kernel, dim3((unsigned)(wave ? ceil_div(here, 4) : here)), dim3(256), static_cast<hipStream_t>(stream),
                                static_cast<const void *>(static_cast<const char *>(x) + at * ldx * (f32 ? 4 : 2)), ldx, q + at * ldq, ldq, scale + at, here, cols);
    if (st != T3_OK) return st;
  }
  return T3_OK;
}

t3_status t3_gemm_i8(const t3_problem *p, const int8_t *A, const float *scale_a, const int8_t *B, const float *scale_b, float *C,
                     void *stream) {
  t3_problem pairs;
  t3_status st = pairs_of(p, false, scale_a, scale_b, &pairs);
  if (st != T3_OK) return st;
  t3k::Plan q;
  int32_t tm, tn;
  bool empty = false;
  st = make_plan(&pairs, t3k::kCallGemm, kNeedAB | kNeedC, A, B, C, nullptr, nullptr, nullptr, &q, &tm, &tn, &empty, true);
  if (st != T3_OK || empty) return st;
  q.R = C;
  q.scale_a = scale_a;
  q.scale_b = scale_b;
  hipStream_t s = static_cast<hipStream_t>(stream);
  q.ldr = q.ldc;                                 // (C through R)
  auto go = [&](const t3k::Plan &plan) { return plan.wide ? t3k::launch_wide_gemm_i8(plan, tm, tn, s) : t3k::launch_small_gemm_i8(plan, tm, tn, s); };
  return q.tail_r ? launch_with_gemm_tail(q, s, go) : go(q);
}

t3_status t3_gemm_rs_fused_i8(const t3_problem *p, const int8_t *A, const float *scale_a, const int8_t *B, const float *scale_b, float *R,
                              void *fwd, uint32_t *track, void *stream) {
  t3_problem pairs;
  t3_status st = pairs_of(p, true, scale_a, scale_b, &pairs);
  if (st != T3_OK) return st;
  t3k::Plan q;
  int32_t tm, tn;
  bool empty = false;
  st = make_plan(&pairs, t3k::kCallFused, kNeedAB | kNeedR | kNeedFwd | kNeedTrack, A, B, nullptr, R, fwd, track, &q, &tm, &tn, &empty, true);
  if (st != T3_OK || empty) return st;
  q.scale_a = scale_a;
  q.scale_b = scale_b;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!q.wide) return t3k::launch_small_fused_i8(q, tm, tn, s);
  return q.overlap ? t3k::launch_wide_overlap_i8(q, tm, tn, s) : t3k::launch_wide_fused_i8(q, tm, tn, s);
}

t3_status t3_gemm_grouped(const t3_grouped *g, const int32_t *offsets, const void *A, const void *B, float *C, void *stream) {
  return grouped_product(g, false, offsets, A, nullptr, B, nullptr, C, stream);
}

t3_status t3_gemm_grouped_i8(const t3_grouped *g, const int32_t *offsets, const int8_t *A, const float *scale_a, const int8_t *B,
                             const float *scale_b, float *C, void *stream) {
  return grouped_product(g, true, offsets, A, scale_a, B, scale_b, C, stream);
}

t3_status t3_gemm_grouped_wgrad(const t3_grouped *g, const int32_t *offsets, const void *A, const void *dC, float *dB, void *stream) {
  t3_status st = check_grouped(g, true, 2);
  if (st != T3_OK) return st;
  const bool some = g->N && g->K;                // (no rows: gradients of zeros, made of no A and no dC)
  if (!offsets || (some && !dB) || (some && g->rows && (!A || !dC))) return T3_ERR_NULL;
  if (!aligned4(offsets) || !aligned16(A) || !aligned16(dC) || !aligned16(dB)) return T3_ERR_ALIGN;
  if (!some) return T3_OK;
  const bool kn = g->b_layout == T3_B_KN;        // the result's rows are the columns of: A (else dC)
  t3k::Plan q{};
  q.A = static_cast<const uint16_t *>(kn ? A : dC);
  q.B = static_cast<const uint16_t *>(kn ? dC : A);
  q.R = dB;
  q.lda = kn ? g->lda : g->ldc;
  q.ldb = kn ? g->ldc : g->lda;
  q.ldr = q.ldc = g->ldb;
  q.M = kn ? g->K : g->N;
  q.N = q.W = kn ? g->N : g->K;
  q.rows = g->rows;
  q.P = 1;
  q.split_k = 1;
  q.offsets = offsets;
  q.stride_b = g->stride_b;
  q.groups = g->groups;
  const bool wide_ok = t3k::wgrad_wide_fits(g->rows, q.lda, q.ldb, q.ldc);
  if (!wide_ok && ceil_div(q.M, 64) * ceil_div(q.N, 64) * g->groups >= 1 << 24) return T3_ERR_UNSUPPORTED;
  DeviceFacts dev;
  st = device_facts(&dev);
  if (st != T3_OK) return st;
  const t3k::Choice c = t3k::grouped_tile(true, true, q.M, q.N, g->rows, g->groups, dev.cus, wide_ok);
  const int32_t tm = c.tile.m, tn = c.tile.n;
  q.Mt = (int32_t)ceil_div(q.M, tm);
  q.tpc = q.Mt * (int32_t)ceil_div(q.N, tn);
  q.by_tpc = t3k::fast_div((uint32_t)q.tpc);
  const int64_t tiles = (int64_t)q.tpc * g->groups;
  plan_rounds(q, c, dev, tiles, 2ll * q.rows * (q.M + q.N) + 4ll * q.groups * q.M * q.N);
  hipStream_t s = static_cast<hipStream_t>(stream);
  // (the host knows these tiles: where no last round is to be cut, no second launch.  In us, with and without: 16384 rows of 32 groups x 2048 x 1024 134 and 131.5,
  // 4000 of 64 x 1024 x 768 48 and 46.4)
  const int64_t last = tiles % q.resident;
  if (!last || 2 * last > q.resident) q.cut = t3k::kCutNone;
  const bool add = g->flags & T3_GROUPED_ACCUMULATE;
  if (q.wide) return launch_rounds(q, add ? t3k::launch_wide_wgrad_add : t3k::launch_wide_wgrad, s);
  return t3k::launch_small_wgrad(q, tm, tn, add, s);
}

t3_status t3_rs_reduce(const t3_problem *p, const float *C, float *R, void *fwd,
                       uint32_t *track, void *stream) {
  t3k::Plan q;
  int32_t tm, tn;
  bool empty = false;
  const t3_status st = make_plan(p, t3k::kCallReduce, kNeedC | kNeedR | kNeedFwd | kNeedTrack, nullptr, nullptr, C,
                                 R, fwd, track, &q, &tm, &tn, &empty);
  if (st != T3_OK) return st;
  if (empty) return T3_OK;
  const int64_t W = p->N / p->tp, elements = (int64_t)(tm < p->M ? tm : p->M) * (tn < W ? tn : W);
  const bool one = elements <= 4 * t3k::kReduceBatch * t3k::kReduceThreads;
  auto kernel = q.total_blocks <= kReduceWordsBlocks ? (one ? t3k::reduce_tile_kernel<true, true> : t3k::reduce_tile_kernel<false, true>)
                                                     : (one ? t3k::reduce_tile_kernel<true, false> : t3k::reduce_tile_kernel<false, false>);
  return launch(kernel, dim3(grid_size(q)), dim3(t3k::kThreads),
                static_cast<hipStream_t>(stream), q);
}

t3_status t3_upstream_update(const t3_problem *p, const float *incoming, float *R,
                             uint32_t *track, void *stream) {
  t3k::Plan q;
  int32_t tm, tn;
  bool empty = false;
  const t3_status st = make_plan(p, t3k::kCallOther, kNeedC | kNeedR | kNeedTrack | kNeedTwoWriters, nullptr, nullptr,
                                 incoming, R, nullptr, track, &q, &tm, &tn, &empty);
  if (st != T3_OK) return st;
  if (empty) return T3_OK;
  unsigned blocks = grid_size(q);
  if (p->upstream_agents > 0 && (unsigned)p->upstream_agents < blocks)
    blocks = (unsigned)p->upstream_agents;     // the rest of the positions are walked in a loop
  const dim3 grid(blocks), block(t3k::kThreads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (tm == 256 && tn == 256)
    return launch(t3k::upstream_update_kernel<256, 256>, grid, block, s, q);
  else if (tm == 256 && tn == 128)
    return launch(t3k::upstream_update_kernel<256, 128>, grid, block, s, q);
  else if (tm == 128 && tn == 256)
    return launch(t3k::upstream_update_kernel<128, 256>, grid, block, s, q);
  return launch(t3k::upstream_update_kernel<128, 128>, grid, block, s, q);
}

t3_status t3_release_chunks(const t3_problem *p, const float *R, void *fwd,
                            const uint32_t *track, void *stream) {
  t3k::Plan q;
  int32_t tm, tn;
  bool empty = false;
  const t3_status st = make_plan(p, t3k::kCallOther, kNeedR | kNeedFwd | kNeedTrack | kNeedTwoWriters, nullptr,
                                 nullptr, nullptr, const_cast<float *>(R), fwd,
                                 const_cast<uint32_t *>(track), &q, &tm, &tn, &empty);
  if (st != T3_OK) return st;
  if (p->tp < 2 || p->M == 0 || p->N == 0) return T3_OK;
  q.agents = kReleaseAgents;
  q.rows_per_agent = (int32_t)ceil_div(p->M, q.agents);
  return launch(t3k::release_ready_kernel, dim3((unsigned)(q.agents * (p->tp - 1))),
                dim3(t3k::kThreads), static_cast<hipStream_t>(stream), q);
}

t3_status t3_timeline(uint64_t *stamps, int64_t words) {
  if (stamps && words < 0) return T3_ERR_BAD_SHAPE;
  if (stamps && (reinterpret_cast<uintptr_t>(stamps) & 7u)) return T3_ERR_ALIGN;
  // (the count first when switching off, the pointer first when switching on: a launch planned
  // in between records nothing rather than out of bounds)
  if (!stamps) {
    g_timeline.store(nullptr);
    g_timeline_wgs.store(0);
    return T3_OK;
  }
  g_timeline_wgs.store(0);
  g_timeline.store(stamps);
  g_timeline_wgs.store(words / (4 * T3_TIMELINE_ITEMS));
  return T3_OK;
}

t3_status t3_ag_step(const t3_problem *p, int32_t step, const float *upstream_R, int64_t ld_up,
                     float *R, void *stream) {
  const t3_status st = check_shape(p);
  if (st != T3_OK) return st;
  if (step < 0 || step >= p->tp - 1) return T3_ERR_BAD_SHAPE;
  if (!upstream_R || !R) return T3_ERR_NULL;
  const int64_t W = p->N / p->tp;
  if (p->ldr < p->N || ld_up < p->N) return T3_ERR_BAD_SHAPE;
  if (p->ldr % 4 || ld_up % 4 || W % 4 || !aligned16(R) || !aligned16(upstream_R)) return T3_ERR_ALIGN;
  if (p->M == 0 || W == 0) return T3_OK;
  const int64_t c = (p->rank + step) % p->tp;    // what the upstream neighbour owned, or got a step ago
  DeviceFacts dev;
  const t3_status known = device_facts(&dev);
  if (known != T3_OK) return known;
  const t3k::CopyShape shape = t3k::copy_shape(p->M, W, dev.cus);
  auto kernel = t3k::ag_copy_kernel<256, 8, 8>;
  if (shape.team == 256 && shape.batch == 1) kernel = t3k::ag_copy_kernel<256, 1, 1>;
  if (shape.team == 64 && shape.batch == 8)
    kernel = shape.in_flight == 8 ? t3k::ag_copy_kernel<64, 8, 8> : (shape.in_flight == 2 ? t3k::ag_copy_kernel<64, 8, 2> : t3k::ag_copy_kernel<64, 8, 1>);
  if (shape.team == 64 && shape.batch == 4) kernel = shape.in_flight == 4 ? t3k::ag_copy_kernel<64, 4, 4> : t3k::ag_copy_kernel<64, 4, 1>;
  if (shape.team == 16) kernel = t3k::ag_copy_kernel<16, 4, 4>;
  if (shape.team == 4) kernel = t3k::ag_copy_kernel<4, 4, 4>;
  const int64_t blocks = shape.workgroups < kMaxCopyBlocks ? shape.workgroups : kMaxCopyBlocks;
  return launch(kernel, dim3((unsigned)blocks), dim3(t3k::kThreads), static_cast<hipStream_t>(stream),
                upstream_R + c * W, ld_up, R + c * W, (int64_t)p->ldr, (int32_t)p->M, (int32_t)W, blocks * (t3k::kThreads / shape.team));
}

}  // extern "C"
