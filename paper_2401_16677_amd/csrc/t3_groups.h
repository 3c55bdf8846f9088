// Rows sorted by group: which rows, and which tile, of which group a workgroup has.
//
// The groups' sizes are known on the device alone (offsets, written by whatever routed the rows), so a workgroup
// finds its tile itself: a lane per group has where the group's rows end and how many rows of tiles there are up to
// and with it, by two scans over the lanes; the group of tile t is the number of groups that end before t.  One request
// and about sixty instructions at the start of a workgroup; after that a tile is a comparison and a few reads of lanes away.  (A launch whose tiles are all on the
// chip at once is a chain of latencies, of which this is one: 2 rows of 8 groups x 4096 x 1024 take 5.1 us, 3.3 at the rate of a copy.)
//
// Offsets are taken as they should be: below 0 as 0, past the rows as their number, below the one before as that one.
// So no group has a row outside of A, no row is in two groups, and there are at most rows / BM + groups rows of tiles.
#pragma once

#include "t3_device.h"

namespace t3k {

constexpr int kMaxGroups = 256;

struct GroupTile {
  int group, row0, rows;               // the group, its first row, how many it has
  int mi, nj;                          // row and column of the tile in the group (of the result, if its rows are not the group's)
};

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t old, uint32_t v) {      // (lanes without a source, and rows not in the mask: old)
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, ROWS, 0xf, false);
}
// Inclusive scans over the 64 lanes: shifts inside rows of 16 lanes, then the rows' last lanes on to the rows behind.
template <typename Op>
__device__ __forceinline__ uint32_t lane_scan(uint32_t v, Op op) {        // (0 is neutral)
  v = op(v, dpp<0x111, 0xf>(0u, v));
  v = op(v, dpp<0x112, 0xf>(0u, v));
  v = op(v, dpp<0x114, 0xf>(0u, v));
  v = op(v, dpp<0x118, 0xf>(0u, v));
  v = op(v, dpp<0x142, 0xa>(0u, v));
  return op(v, dpp<0x143, 0xc>(0u, v));
}

struct GroupRows {
  static constexpr int kSets = kMaxGroups / 64;
  uint32_t end[kSets], tiles[kSets];   // lane l of set r, group 64 r + l: behind its last row; rows of tiles up to and with it
  uint32_t first, all_tiles;           // first row of the first group; rows of tiles of all groups
  bool sorted = false;                 // contractions over rows: the groups are taken in the order of by_length
  uint32_t by_length = 0;

  // bm: rows of a tile
  __device__ __forceinline__ void load(const Plan &p, int lane, uint32_t bm) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p.offsets, (uint32_t)(p.groups + 1) * 4u);
    auto offset = [&](int i) {                   // (past the array's end 0: no rows)
      return (uint32_t)min(max((int)__builtin_amdgcn_raw_buffer_load_b32(r, i * 4, 0, 0), 0), p.rows);
    };
    uint32_t v[kSets];
    const uint32_t v0 = offset(0);
#pragma unroll
    for (int s = 0; s < kSets; ++s) v[s] = s == 0 || p.groups > 64 * s ? offset(64 * s + lane + 1) : 0u;
    first = __builtin_amdgcn_readfirstlane(v0);
    uint32_t before = first, count = 0u;
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      end[s] = before;
      tiles[s] = count;
      if (s == 0 || p.groups > 64 * s) {
        const uint32_t e = lane_scan(max(v[s], before), [](uint32_t a, uint32_t b) { return max(a, b); });
        const uint32_t rows = e - dpp<0x138, 0xf>(before, e);               // (the lane before's; lane 0: the set before's last)
        const uint32_t t = lane_scan((rows + bm - 1) / bm, [](uint32_t a, uint32_t b) { return a + b; }) + count;
        end[s] = e;
        tiles[s] = t;
        before = __builtin_amdgcn_readlane(e, 63);
        count = __builtin_amdgcn_readlane(t, 63);
      }
    }
    all_tiles = count;
  }
  // Contractions over a group's rows: the groups by length, the longest first, where there is more than a round of tiles, so that those of a round take about as
  // long as one another and the last ones are short.  Lane r then has the r-th group: it is behind as many as have a larger key.  (In us, in the order
  // that the groups are in, shortest first and longest first: 8190 rows of 16 groups x 5120 x 1280 177, 190 and 165; 16384 of 32 x 2048 x 1024 132, 120 and 122; 16000 of
  // 8 x 2560 x 2560 226, 245 and 212.  More than 64 groups are left as they are: their tiles are short ones.)
  __device__ __forceinline__ void longest_first(const Plan &p, int lane) {
    sorted = p.groups <= 64 && (uint32_t)p.tpc * (uint32_t)p.groups > p.order.round;
    if (!sorted) return;
    const uint32_t rows = end[0] - dpp<0x138, 0xf>(first, end[0]);
    const uint32_t key = min(rows, (1u << 26) - 1) << 6 | (uint32_t)(63 - lane);       // (no two alike; behind the last group no rows)
    uint32_t before = 0u;
    for (int g = 0; g < p.groups; g += 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) before += __builtin_amdgcn_readlane(key, g + i) > key ? 1u : 0u;
    }
    by_length = (uint32_t)__builtin_amdgcn_ds_permute((int)(lane < p.groups ? before : (uint32_t)lane) * 4, lane);
  }
  __device__ __forceinline__ static uint32_t of(const uint32_t (&a)[kSets], int g) {
    uint32_t v = __builtin_amdgcn_readlane(a[0], g & 63);
#pragma unroll
    for (int s = 1; s < kSets; ++s)
      if (g >> 6 == s) v = __builtin_amdgcn_readlane(a[s], g & 63);
    return v;
  }
  __device__ __forceinline__ void rows_of(int g, GroupTile &t) const {
    t.group = g;
    t.row0 = (int)(g ? of(end, g - 1) : first);
    t.rows = (int)of(end, g) - t.row0;
  }
  // Grid position b of n tiles.  Workgroups are dealt round-robin to the 8 XCDs: of every round of positions each XCD gets a run of
  // neighbouring tiles, as long as the others' up to one.
  __device__ __forceinline__ static bool place(const Plan &p, uint32_t b, uint32_t n, uint32_t &at) {
    const uint32_t base = div_by(b, p.order.by_round) * p.order.round, j = b - base, x = j & 7;
    if (base >= n) return false;
    const uint32_t here = min(n - base, p.order.round), odd = here & 7;
    at = base + (here >> 3) * x + min(odd, x) + (j >> 3);
    return (j >> 3) < (here >> 3) + (x < odd ? 1u : 0u);
  }
  // Tile q of a group's Mt x Wt: columns four at a time, row by row, so that a run of tiles shares both rows and columns.
  __device__ __forceinline__ static void in_group(uint32_t q, uint32_t Mt, uint32_t Wt, GroupTile &t) {
    const uint32_t band = q / (4u * Mt), in = q - band * 4u * Mt, width = min(4u, Wt - 4u * band), row = in / width;
    t.mi = (int)row;
    t.nj = (int)(4u * band + in - row * width);
  }
  // Tiles of products whose rows are grouped, and of products whose contraction runs over a group's rows (tpc for every group)
  template <bool ROWS>
  __device__ __forceinline__ uint32_t count(const Plan &p) const { return ROWS ? all_tiles * (uint32_t)p.Wt : (uint32_t)p.groups * (uint32_t)p.tpc; }
  // How many of n tiles the first launch does where the last round's may be cut: the others are at most half a round.
  __device__ __forceinline__ static uint32_t uncut(const Plan &p, uint32_t n) {
    const uint32_t round = p.order.round, left = n - div_by(n, p.order.by_round) * round;
    return n > round && 2u * left <= round ? n - left : n;
  }
  template <bool ROWS>
  __device__ __forceinline__ void tile(const Plan &p, uint32_t at, GroupTile &t) const {
    if (ROWS) tile_at(p, at, t);
    else tile_of_all(p, at, t);
  }
  // The tile at grid position b; false: behind the last one.
  template <bool ROWS>
  __device__ __forceinline__ bool tile_of_position(const Plan &p, uint32_t b, GroupTile &t) const {
    const uint32_t n = count<ROWS>(p);
    uint32_t at;
    if (!place(p, b, p.cut == kCutLeave ? uncut(p, n) : n, at)) return false;
    tile<ROWS>(p, at, t);
    return true;
  }
  __device__ __forceinline__ void tile_at(const Plan &p, uint32_t at, GroupTile &t) const {
    int g = 0;
#pragma unroll
    for (int s = 0; s < kSets; ++s) g += __builtin_popcountll(__ballot(tiles[s] * (uint32_t)p.Wt <= at));
    rows_of(g, t);
    const uint32_t before = g ? of(tiles, g - 1) : 0u, Mt = of(tiles, g) - before, q = at - before * (uint32_t)p.Wt;
    in_group(q, Mt, (uint32_t)p.Wt, t);
  }
  __device__ __forceinline__ void tile_of_all(const Plan &p, uint32_t at, GroupTile &t) const {
    const uint32_t g = div_by(at, p.by_tpc);
    rows_of((int)(sorted ? __builtin_amdgcn_readlane(by_length, g & 63) : g), t);
    in_group(at - g * (uint32_t)p.tpc, (uint32_t)p.Mt, (uint32_t)p.Wt, t);
  }
};

}  // namespace t3k
