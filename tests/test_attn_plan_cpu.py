"""How the paged attention is cut (csrc/attn_plan.h): every block of every item computed once, by the share that
owns it, its partial results in places of their own; and csrc/divider.h."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_09200_amd", "csrc")

PLAN = r"""
#include "attn_plan.h"
#include <algorithm>
#include <map>
#include <random>
#include <set>
#include <stdio.h>
#include <vector>

using namespace occ;

static long bad, items_seen, split, evened;

static void line(const AttnCut &c, const std::vector<AttnSeq> &seqs, int workgroups, int min_share) {
  // the items as the definition has them
  struct Placed { int64_t at; int keys, units; };
  std::vector<Placed> items;
  int64_t at = 0;
  for (const AttnSeq &s : seqs) {
    const int tiles = attn_tiles(c, s);
    if (attn_units(c, s) < 0) ++bad;
    for (int part = 0; part < c.parts; ++part) {
      int64_t before = 0;
      for (int m = 0; m < tiles; ++m) {
        int first = 1 << 30, last = 0;
        for (int t = m * c.tokens; t < std::min((m + 1) * c.tokens, s.fresh); ++t) {
          const int64_t pos = (int64_t)s.len - s.fresh + t;
          const int64_t hi = c.causal ? std::min<int64_t>(pos + 1, s.len) : s.len, lo = c.window ? std::max<int64_t>(0, pos - c.window + 1) : 0;
          if (hi > lo) first = std::min<int64_t>(first, lo), last = std::max<int64_t>(last, hi);
        }
        const int a = attn_first_key(c, s, m), b = attn_last_key(c, s, m);
        if (a < 0 || b < a || b > s.len) ++bad;
        if (last > 0 && (a > first || b < last || b != last)) ++bad;
        if (attn_units_before(c, s, m) != before) ++bad;
        const int units = c.fixed + (c.flat ? attn_most_keys(c, s) : b - a);
        if (b - a > attn_most_keys(c, s)) ++bad;
        if (attn_tile_at(c, s, before) != m || attn_tile_at(c, s, before + units - 1) != m) ++bad;
        items.push_back({at, b - a, units});
        at += units;
        before += units;
      }
      if (attn_units_before(c, s, tiles) != before) ++bad;
    }
  }
  const int64_t total = at;
  const AttnShare cutter = attn_share(total, workgroups, min_share);
  const int64_t share = cutter.units;
  if (share * workgroups < total || share < min_share) ++bad;
  if (share > min_share && (share - 2) * workgroups > total) ++bad;
  std::set<int> counters;
  std::set<std::pair<int, int>> slots;
  for (const Placed &placed : items) {
    const AttnItem it{placed.at, placed.keys};
    ++items_seen;
    const AttnOwners o = attn_owners(c, it, cutter);
    const int blocks = (it.keys + c.block - 1) / c.block;
    int next = 0;
    const int64_t end = it.at + placed.units;
    for (int w = (int)(it.at / share); w * share < end; ++w) {
      const int b0 = attn_blocks_before(c, it, w * share), b1 = attn_blocks_before(c, it, std::min((w + 1) * share, total));
      if (b0 != next) ++bad;
      next = b1;
      const bool owns = it.keys > 0 && w >= o.from && w < o.to;
      if ((b0 < b1) != owns) ++bad;
      if (owns && o.to - o.from > 1 && !slots.insert({w, it.at >= w * share}).second) ++bad;
      if (w >= workgroups) ++bad;
    }
    if (next != blocks) ++bad;
    if (it.keys == 0 && (o.from != o.to || o.from != it.at / share)) ++bad;
    if (o.to - o.from > 1) {
      ++split;
      if (!counters.insert(o.from).second) ++bad;
    }
  }
}

// Items of these blocks in even parts: every block once, by parts that a joining workgroup finds in order.
static void even(const std::vector<int> &keys, int shares, int least, int spare) {
  int64_t total = 0;
  for (int k : keys) total += k;
  const int units = attn_even_units(total, keys.size(), shares, least, spare);
  if (units == 0) return;
  ++evened;
  if (units < least) ++bad;
  int64_t parts = 0;
  for (int most : keys) {
    const int k = attn_even_parts(most, units);
    if (k < 1 || (int64_t)k * units < most) ++bad;
    parts += k;
    for (int n : {most, most / 2, most / 100, 1, 0}) {   // a tile may have fewer keys than its request's longest
      const int blocks = (n + 31) / 32;
      int have = 0;
      if (attn_even_blocks(blocks, k, 0) != 0 || attn_even_blocks(blocks, k, k) != blocks) ++bad;
      for (int j = 0; j < k; ++j) {
        const int b0 = attn_even_blocks(blocks, k, j), b1 = attn_even_blocks(blocks, k, j + 1);
        if (b1 < b0) ++bad;
        if (b1 > b0 && have++ != j) ++bad;   // the parts that have any come first
      }
      if (have != std::min(blocks, k)) ++bad;
    }
  }
  if (parts > shares) ++bad;
}

int main() {
  std::mt19937 g(1);
  auto pick = [&](std::vector<int> v) { return v[g() % v.size()]; };
  for (int n = 0; n < 3000; ++n) {
    AttnCut c;
    c.tokens = pick({1, 2, 4, 16, 18, 128});
    c.by_tokens = Divider(c.tokens);
    c.parts = pick({1, 2, 8});
    c.block = pick({32, 64});
    c.fixed = pick({0, 1, 32, 64, 300, 512, 2000}) + (n % 2 ? 32 : 1);
    c.window = pick({0, 0, 1, 5, 100, 1 << 30});
    c.causal = pick({1, 1, 0});
    c.flat = pick({0, 1});
    std::vector<AttnSeq> seqs;
    const int count = pick({1, 3, 9});
    for (int i = 0; i < count; ++i) {
      AttnSeq s{0, pick({0, 1, 1, 3, 40, 300}), pick({0, 1, 31, 64, 257, 1000})};
      if (pick({0, 1, 2})) s.len += s.fresh;  // else fewer keys than tokens, as no program has it
      seqs.push_back(s);
    }
    line(c, seqs, pick({1, 2, 7, 256, 512}), pick({64, 256, 256}));
  }
  for (int n = 0; n < 20000; ++n) {
    std::vector<int> keys(pick({1, 2, 8, 40, 100, 200, 255, 256, 300}));
    const int most = pick({1, 100, 700, 5000, 130000, 2000000000});
    for (int &k : keys) k = pick({0, 1, 2}) ? g() % most + 1 : 0;
    even(keys, pick({256, 256, 304, 8}), pick({128, 256}), pick({0, 512}));
  }
  // sizes near the limits: no sum leaves 64 bits, no key 31
  AttnCut c{2, 8, 32, 32, 0, 1, 0, Divider(2)};
  const AttnSeq big{0, 1 << 24, 2147418112};
  if (attn_units(c, big) <= 0 || attn_last_key(c, big, attn_tiles(c, big) - 1) != big.len) ++bad;
  c.window = 1 << 30;
  if (attn_units(c, big) <= 0 || attn_first_key(c, big, 0) != big.len - big.fresh - c.window + 1) ++bad;
  const AttnSeq s = attn_seq(-5, 2000000000, -7, 100, 1000), e = attn_seq(50, 20, 5000, 100, 1000);
  if (s.first != 0 || s.fresh != 100 || s.len != 0 || e.first != 50 || e.fresh != 0 || e.len != 1000) ++bad;
  // shares of far units
  for (int n = 0; n < 2000000; ++n) {
    const int64_t total = ((int64_t)g() << 20 | g() >> 12) >> pick({0, 3, 10, 20, 30, 40});
    const AttnShare by = attn_share(total, pick({1, 7, 256, 512}), pick({32, 256}));
    const int64_t x = total == 0 ? 0 : (((int64_t)g() << 31 | g()) % total) / pick({1, 1, 1000});
    const int64_t y = x / by.units * by.units;   // the first of its share
    if (by(x) != x / by.units || by(y) != y / by.units || (y > 0 && by(y - 1) != (y - 1) / by.units)) ++bad;
  }
  printf("bad %ld items %ld split %ld\n", bad, items_seen, split);
  return bad != 0 || split < 1000 || evened < 1000;
}
"""

DIVIDE = r"""
#include "divider.h"
#include <stdio.h>

int main() {
  long bad = 0;
  const int ds[] = {1, 2, 3, 5, 7, 16, 24, 48, 63, 64, 65, 640, 65535, 65536, 1000003, 2147483647};
  for (int d : ds) {
    const occ::Divider by(d);
    for (long n = 0; n < 2147483648L; n += n < 200000 ? 1 : 999983) {
      bad += by((int)n) != (int)n / d;
    }
    for (long m = 1; m * d <= 2147483647L && m < 100000; m += 7)
      for (long n = m * d - 1; n <= m * d + 1 && n <= 2147483647L; ++n) bad += by((int)n) != (int)(n / d);
    bad += by(2147483647) != 2147483647 / d;
  }
  printf("%ld\n", bad);
  return bad != 0;
}
"""


def run(tmp_path, text):
    src = tmp_path / "t.cpp"
    src.write_text(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-I", CSRC, str(src), "-o", str(tmp_path / "t")], check=True)
    r = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "runtime error" not in r.stderr, r.stdout + r.stderr


def test_every_block_is_computed_once(tmp_path):
    run(tmp_path, PLAN)


def test_division(tmp_path):
    run(tmp_path, DIVIDE)
