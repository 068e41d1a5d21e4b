// How the attention over a paged cache is cut into shares of equal work: arithmetic that the host can check.
//
// A request's new tokens are taken in tiles of `tokens` of them, once for each of `parts` groups of heads.  An item
// (request, part, tile) costs what it reads, its keys, and `fixed` keys' worth beside.  Nothing but the lengths, which only
// the GPU knows, decides who does what:
//  * The line.  All items in a row are one line of units; a workgroup takes a share of it, which may begin and end within an
//    item.  Shares are equal, whatever the lengths; an item that several have a part of is joined.
//  * Few items (attn_even): each item goes to as many workgroups as it is long for, in equal parts, and a workgroup has
//    one part and no more.
#pragma once

#include "divider.h"

#define OCC_PLAN OCC_DIVIDE

namespace occ {

struct AttnCut {
  int tokens;   // of a tile
  int parts;    // groups of heads
  int fixed;    // keys' worth of an item's beginning and end
  int block;    // keys that are computed at once, a power of two
  int window;   // 0: none
  int causal;
  int flat;     // all tiles of a request count as its longest: no sums over tiles
  Divider by_tokens;
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

// Numbers of rows go up to 2^31 - 1: nothing is added to one before it is divided.
OCC_PLAN int attn_tiles(const AttnCut &c, const AttnSeq &s) { return s.fresh == 0 ? 0 : c.by_tokens(s.fresh - 1) + 1; }

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

// Token t of tile m: whether there is one, which of the request's, and the keys [lo, hi) that it sees.
struct AttnRow {
  int token, lo, hi;
  bool valid;
};
OCC_PLAN AttnRow attn_row(const AttnCut &c, const AttnSeq &s, int m, int t) {
  const int before = m * c.tokens;
  AttnRow r{0, 0, 0, t < s.fresh - before};
  const int pos = s.len - s.fresh + before + t;  // negative where a request has more rows than keys
  r.token = r.valid ? before + t : 0;
  r.hi = !r.valid ? 0 : !c.causal ? s.len : pos < 0 ? 0 : pos + 1 < s.len ? pos + 1 : s.len;
  r.lo = c.window != 0 && pos >= c.window ? pos - c.window + 1 : 0;
  return r;
}
// Keys [lo, hi) that all of its tokens t0 .. t1 - 1 see, as far as these exist.
struct AttnKeys {
  int lo, hi;
};
OCC_PLAN AttnKeys attn_all_see(const AttnCut &c, const AttnSeq &s, int m, int t0, int t1) {
  const int left = s.fresh - m * c.tokens;
  return AttnKeys{attn_row(c, s, m, (t1 < left ? t1 : left) - 1).lo, t0 < left ? attn_row(c, s, m, t0).hi : s.len};
}

// Sum over j < n of max(0, a + j tokens).
OCC_PLAN int64_t attn_ramp(const AttnCut &c, int n, int64_t a) {
  const int64_t step = c.tokens;
  if (n <= 0 || a + (n - 1) * step <= 0) return 0;
  // here -a < (n - 1) step, at most a request's rows
  const int skip = a < 0 ? c.by_tokens((int)(-a - 1)) + 1 : 0;
  const int64_t count = n - skip;
  return count * (a + skip * step) + step * (count * (count - 1) / 2);
}

// Keys that a tile has at most.
OCC_PLAN int attn_most_keys(const AttnCut &c, const AttnSeq &s) {
  // without causality the last key of all is every tile's last
  const int64_t seen = (int64_t)c.window + (c.causal ? c.tokens : s.fresh) - 1;
  return c.window && seen < s.len ? (int)seen : s.len;
}

// Units of a request's tiles before tile m (of one part).
OCC_PLAN int64_t attn_units_before(const AttnCut &c, const AttnSeq &s, int m) {
  if (c.flat) return (int64_t)m * (attn_most_keys(c, s) + c.fixed);
  const int64_t base = (int64_t)s.len - s.fresh;
  int64_t keys;
  if (c.causal) {
    keys = attn_ramp(c, m, base + c.tokens);
    // the last tile may have fewer tokens
    const int64_t over = base + (int64_t)m * c.tokens;
    if (m > 0 && (int64_t)m * c.tokens > s.fresh) keys -= (over > 0 ? over : 0) - s.len;
  } else {
    keys = (int64_t)m * s.len;
  }
  if (c.window) keys -= attn_ramp(c, m, base - c.window + 1);
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

// An item on the line: units [at, at + fixed + keys) and, flat, some behind them, of which block b (keys first + b block ...) belongs to
// the share that unit at + fixed + b block lies in.
struct AttnItem {
  int64_t at;
  int keys;
};

// Blocks of the item before unit x.
OCC_PLAN int attn_blocks_before(const AttnCut &c, const AttnItem &it, int64_t x) {
  int64_t k = x - it.at - c.fixed;
  k = k < 0 ? 0 : k > it.keys ? it.keys : k;
  return (int)((k + c.block - 1) / c.block);
}

// The share that a unit lies in, below 2^53 units and 2^31 shares: a product in binary64 is off by less than one of them.
struct AttnShare {
  int64_t units;
  double per_unit;
  OCC_PLAN int operator()(int64_t x) const {
    int q = (int)((double)x * per_unit);
    const int64_t left = x - q * units;
    if (left < 0) --q;
    if (left >= units) ++q;
    return q;
  }
};
// `total` units in at most `shares` of them, of `least` units or more.
OCC_PLAN AttnShare attn_share(int64_t total, int shares, int least) {
  // rounded up, or one more
  int64_t units = (int64_t)((double)total / shares) + 1;
  if (units < least) units = least;
  return AttnShare{units, 1.0 / (double)units};
}

// Who computes an item's blocks: shares [from, to), each of them some (a share is no shorter than a block); without
// keys none does, and share `from` has the item's rows to write.
struct AttnOwners {
  int from, to;
};
OCC_PLAN AttnOwners attn_owners(const AttnCut &c, const AttnItem &it, const AttnShare &share) {
  if (it.keys == 0) return AttnOwners{share(it.at), share(it.at)};
  const int64_t last = (int64_t)(it.keys - 1) / c.block * c.block;
  return AttnOwners{share(it.at + c.fixed), share(it.at + c.fixed + last) + 1};
}

// Few items: parts of an item of at most `most` keys where a part has `units` of them, and whether that is better than
// the line with `items` items of `total` units: if every part has a workgroup, and the longest is not so much longer
// than a share that a second piece (and one more joining) would be cheaper, `spare` keys' worth.
OCC_PLAN int attn_even_units(int64_t total, int64_t items, int shares, int least, int spare) {
  if (items >= shares) return 0;
  const double even = (double)total / (double)(shares - (int)items) + 1;  // the parts are less than `shares`
  if (even > (double)total / shares + spare || even > 1e9) return 0;
  return (int)even + 1 < least ? least : (int)even + 1;
}
OCC_PLAN int attn_even_parts(int most, int units) { return most <= units ? 1 : (int)((uint32_t)(most - 1) / (uint32_t)units) + 1; }
// Blocks of an item before part j of k: the first parts have one more; if there are fewer blocks than parts, one each.
OCC_PLAN int attn_even_blocks(int blocks, int k, int j) {
  const int each = (int)((uint32_t)blocks / (uint32_t)k), more = blocks - each * k;
  return j * each + (j < more ? j : more);
}

}  // namespace occ
