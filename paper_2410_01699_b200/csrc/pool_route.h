// How sjd_pool_attention shares its units out: arithmetic of the host alone.
#pragma once

#include <cstdint>

#include "sjd.h"

namespace sjd {

constexpr int kTile = 128;           // keys
constexpr int kMaxEntries = 512;     // (sequence, tile of rows) pairs of a call whose tiles are cut into equal ranges
constexpr int kUnitCost = 3;        // what a unit's begin and end take, in tiles (41 calls of windows of up to 64 rows: with 1 7 % slower, 2 2.6, 4 0.5, 5 1.3)
constexpr int kWholeTiles = 4;      // units of up to so many tiles are not cut where they are few

// Whether the tiles of all units are cut into equal ranges; else a CTA takes a unit.  A CTA per unit where units are short and few (the
// joining launch costs more than it could win: 2 us), or where the CTAs would have to look at too many positions to find equal ranges
// (a long sequence is then one CTA's per kv head: 512 tokens, one of them behind 100,000 positions, 32 heads on 8, 179 us, 513 of them 990).
// Places on the line of tiles are counted in 32 bits, and the rows of a window may stand at any positions, so that a unit can have all tiles of
// its table, with a sliding window too.
inline bool pool_equal_ranges(int64_t entries, int64_t kv_heads, int64_t positions, int64_t pages_per_seq, int64_t window, int64_t sliding,
                              int64_t sinks, int64_t sms) {
  const int64_t table = (pages_per_seq * SJD_KV_PAGE + kTile - 1) / kTile, units = entries * kv_heads;
  int64_t usual = table;   // tiles of a unit whose rows follow one another
  if (sliding > 0) {
    const int64_t in = (sliding + window + kTile - 2) / kTile + 1 + (sinks + kTile - 1) / kTile;
    usual = usual < in ? usual : in;
  }
  return entries <= kMaxEntries && positions <= 8192 && (usual > kWholeTiles || units > 2 * sms) && units * (table + kUnitCost) < 1 << 30;
}

}  // namespace sjd
