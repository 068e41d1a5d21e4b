// How the attention over a paged cache is cut into shares of equal work: arithmetic that the host can check.
//
// A request's new tokens are taken in tiles of `tokens` of them, once for each of `parts` groups of heads.  An item
// (request, part, tile) costs what it reads, its keys, and `fixed` keys' worth beside.  All items in a row
// are one line of units; a workgroup takes `share` units of it, which may begin and end within
// an item.  Nothing but the lengths, which only the GPU knows, decides: a single long request is split along its
// keys, many short ones are dealt out whole.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define OCC_PLAN __host__ __device__ __forceinline__
#else
#define OCC_PLAN inline
#endif

namespace occ {

struct AttnCut {
  int tokens;   // of a tile
  int parts;    // groups of heads
  int fixed;    // keys' worth of an item's beginning and end
  int block;    // keys that a share is a multiple of
  int window;   // 0: none
  int causal;
};

struct AttnSeq {
  int first;  // its first row of q
  int fresh;  // its rows
  int len;    // its keys
};

// Request i of starts and lens, whatever these hold: rows within [0, rows], keys within [0, most].
OCC_PLAN AttnSeq attn_seq(int start, int end, int len, int rows, int most) {
  const int a = start < 0 ? 0 : start > rows ? rows : start;
  const int b = end < a ? a : end > rows ? rows : end;
  return AttnSeq{a, b - a, len < 0 ? 0 : len > most ? most : len};
}

OCC_PLAN int attn_tiles(const AttnCut &c, const AttnSeq &s) { return (s.fresh + c.tokens - 1) / c.tokens; }

// Keys [first, last) that some token of tile m sees.
OCC_PLAN int attn_last_key(const AttnCut &c, const AttnSeq &s, int m) {
  if (!c.causal) return s.len;
  const int64_t token = (int64_t)(m + 1) * c.tokens < s.fresh ? (int64_t)(m + 1) * c.tokens : s.fresh;
  const int64_t end = (int64_t)s.len - s.fresh + token;
  return end < 0 ? 0 : (int)end;
}
OCC_PLAN int attn_first_key(const AttnCut &c, const AttnSeq &s, int m) {
  if (c.window == 0) return 0;
  const int64_t at = (int64_t)s.len - s.fresh + (int64_t)m * c.tokens - c.window + 1;
  const int last = attn_last_key(c, s, m);
  return at < 0 ? 0 : at > last ? last : (int)at;
}

// Sum over j < n of max(0, a + j step).
OCC_PLAN int64_t attn_ramp(int64_t n, int64_t a, int64_t step) {
  const int64_t skip = a < 0 ? (-a + step - 1) / step : 0;
  if (n <= skip) return 0;
  const int64_t count = n - skip;
  return count * (a + skip * step) + step * (count * (count - 1) / 2);
}

// Units of a request's tiles before tile m (of one part).
OCC_PLAN int64_t attn_units_before(const AttnCut &c, const AttnSeq &s, int m) {
  const int64_t base = (int64_t)s.len - s.fresh;
  int64_t keys;
  if (c.causal) {
    keys = attn_ramp(m, base + c.tokens, c.tokens);
    // the last tile may have fewer tokens
    const int64_t over = base + (int64_t)m * c.tokens;
    if (m > 0 && (int64_t)m * c.tokens > s.fresh) keys -= (over > 0 ? over : 0) - s.len;
  } else {
    keys = (int64_t)m * s.len;
  }
  if (c.window) keys -= attn_ramp(m, base - c.window + 1, c.tokens);
  return keys + (int64_t)m * c.fixed;
}

OCC_PLAN int64_t attn_units(const AttnCut &c, const AttnSeq &s) {
  return c.parts * attn_units_before(c, s, attn_tiles(c, s));
}

// The tile that unit x of a part of a request lies in.
OCC_PLAN int attn_tile_at(const AttnCut &c, const AttnSeq &s, int64_t x) {
  int lo = 0, hi = attn_tiles(c, s) - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (attn_units_before(c, s, mid) <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// An item on the line: units [at, at + fixed + keys), of which block b (keys first + b block ...) belongs to
// the share that unit at + fixed + b block lies in.
struct AttnItem {
  int64_t at;
  int keys;
};

// Blocks of the item before unit x.
OCC_PLAN int attn_blocks_before(const AttnCut &c, const AttnItem &it, int64_t x) {
  int64_t k = x - it.at - c.fixed;
  k = k < 0 ? 0 : k > it.keys ? it.keys : k;
  return ((int)k + c.block - 1) / c.block;
}

// Who computes an item's blocks: shares [from, to), each of them some (a share is no shorter than a block); without
// keys none does, and share `from` has the item's rows to write.
struct AttnOwners {
  int from, to;
};
OCC_PLAN AttnOwners attn_owners(const AttnCut &c, const AttnItem &it, int64_t share) {
  if (it.keys == 0) return AttnOwners{(int)(it.at / share), (int)(it.at / share)};
  const int64_t last = (int64_t)(it.keys - 1) / c.block * c.block;
  return AttnOwners{(int)((it.at + c.fixed) / share), (int)((it.at + c.fixed + last) / share) + 1};
}

}  // namespace occ
