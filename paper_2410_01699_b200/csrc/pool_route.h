// How sjd_pool_attention shares its units out, and when sjd_pool_attention_shared leaves a call to it: arithmetic of the host alone.
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

// Whether each sequence is attended for itself where some may share pages.  rows: of a sequence for one kv head; alone: as many groups as sequences, so
// that none can.  A call for shared pages begins with a plan and ends with a joining launch, 27 to 45 us for any lengths; the kernel that takes each
// sequence for itself begins with 10 to 15, and then a tile of 16, 32 or 64 rows takes a CTA 0.75, 1.25 or 2 us.  Where the tables could not keep it
// busy for more than 24 us, it is faster whatever is shared (54 calls of 2 to 32 sequences, 208 to 2128 positions: 43 are its own by this
// rule, 5 to 30 us faster each; of the others it would be faster in three, by up to 5).  Sequences that are alone meet tiles of 128 rows in the other kernel, 1.8 us for up to 128 of them: up to 64 rows
// this one is faster (16 sequences of 4096 positions, 32 heads: 16 rows 97 us against 241, 32 rows 144 and 211, 64 rows 229 and 226, 128 rows 428 and 243).
// All of these had tables as wide as their longest sequence.  The width is what the host knows, and a short call of a pool with wide tables is not left to the other kernel by it: two
// tokens of 217 positions take 9.7 us with tables of 4 pages, and 19.3 with tables of 16,384, where that would take 12.2.
inline bool pool_each_for_itself(int64_t batch, int64_t window, int64_t kv_heads, int64_t rows, int64_t pages_per_seq, bool alone, int64_t sms) {
  const int64_t tile = rows <= 16 ? 16 : rows <= 32 ? 32 : 64, quarters = rows <= 16 ? 3 : rows <= 32 ? 5 : 8;   // (quarters of a us)
  const int64_t entries = batch * ((rows + tile - 1) / tile), table = (pages_per_seq * SJD_KV_PAGE + kTile - 1) / kTile;
  if (entries > kMaxEntries || batch * window > 8192) return false;   // (its keys would not be cut evenly)
  return (alone && rows <= 64) || entries * kv_heads * (table + kUnitCost) * quarters <= 96 * sms;
}

}  // namespace sjd
