"""The paged attention's plan (csrc/attn_plan.h) at the ends of what occ.h allows: 2^31 - 1 rows of one request, windows
and lengths next to 2^31.  Its numbers against the definition in 128 bits, with the host's check for overflow on."""
from test_attn_plan_cpu import run

LIMITS = r"""
#include "attn_plan.h"
#include <algorithm>
#include <random>
#include <stdio.h>
#include <vector>

using namespace occ;
typedef __int128 i128;

static long bad, seen;
static void check(bool ok, const char *what, const AttnCut &c, const AttnSeq &s, int64_t m) {
  ++seen;
  if (ok) return;
  if (++bad < 20) printf("%s: tokens %d window %d causal %d fresh %d len %d, %ld\n", what, c.tokens, c.window, c.causal, s.fresh, s.len, (long)m);
}

static i128 clampi(i128 v, i128 lo, i128 hi) { return v < lo ? lo : v > hi ? hi : v; }
static i128 ceil_div(i128 a, i128 b) { return a <= 0 ? 0 : (a + b - 1) / b; }

// Sum over j < n of max(0, a + j step).
static i128 ramp(i128 n, i128 a, i128 step) {
  const i128 skip = clampi(ceil_div(-a, step), 0, n), count = n - skip;
  return count * (a + skip * step) + step * (count * (count - 1) / 2);
}

static void sequence(const AttnCut &c, const AttnSeq &s) {
  const i128 tiles = ceil_div(s.fresh, c.tokens), base = (i128)s.len - s.fresh;
  check(attn_tiles(c, s) == (int64_t)tiles, "tiles", c, s, 0);
  std::vector<int64_t> some = {0, 1, 2, (int64_t)tiles / 2, (int64_t)tiles - 2, (int64_t)tiles - 1};
  for (int64_t m : some) {
    if (m < 0 || m >= tiles) continue;
    const i128 t0 = (i128)m * c.tokens, t1 = std::min<i128>(t0 + c.tokens, s.fresh);
    const i128 last = c.causal ? clampi(base + t1, 0, s.len) : s.len;
    const i128 first = c.window ? clampi(base + t0 - c.window + 1, 0, last) : 0;
    check(attn_last_key(c, s, (int)m) == last, "last key", c, s, m);
    check(attn_first_key(c, s, (int)m) == first, "first key", c, s, m);
    if (!c.flat) {
      // keys of the m tiles before this one, all of them whole
      i128 units = c.causal ? ramp(m, base + c.tokens, c.tokens) : (i128)m * s.len;
      if (c.window) units -= ramp(m, base - c.window + 1, c.tokens);
      check(attn_units_before(c, s, (int)m) == (int64_t)(units + (i128)m * c.fixed), "units", c, s, m);
    }
    for (int t : {0, 1, c.tokens / 2, c.tokens - 1}) {
      const AttnRow r = attn_row(c, s, (int)m, t);
      const i128 token = t0 + t, pos = base + token;
      check(r.valid == (token < s.fresh), "valid", c, s, m);
      const i128 hi = !r.valid ? 0 : c.causal ? clampi(pos + 1, 0, s.len) : s.len, lo = c.window ? std::max<i128>(0, pos - c.window + 1) : 0;
      check(!r.valid || (r.token == token && r.hi == hi && r.lo == lo), "row", c, s, m);
      check(r.hi >= 0 && r.lo >= 0 && (r.valid || r.hi == 0), "no keys", c, s, m);
      for (int u : {t, c.tokens - 1}) {
        // keys that all of tokens t .. u see
        const AttnKeys all = attn_all_see(c, s, (int)m, t, u + 1);
        const i128 until = std::min<i128>(t0 + u + 1, s.fresh);
        if (token >= s.fresh) {  // rows that nobody writes leave no key out
          check(all.hi == s.len, "none", c, s, m);
          continue;
        }
        check(all.hi == hi && all.lo == (c.window ? std::max<i128>(0, base + until - c.window) : 0), "all", c, s, m);
      }
    }
  }
}

int main() {
  std::mt19937 g(3);
  auto pick = [&](std::vector<int> v) { return v[g() % v.size()]; };
  const int most = 2147483647, keys = 2147418112;
  for (int n = 0; n < 200000; ++n) {
    AttnCut c{};
    c.tokens = pick({1, 2, 16, 37, 64, 128, 256});
    c.by_tokens = Divider(c.tokens);
    c.parts = 1, c.fixed = pick({256, 384, 512}), c.block = 64, c.causal = g() & 1, c.flat = g() & 1;
    c.window = g() & 1 ? 0 : pick({1, 2, 1000, 65536, keys / 2, keys - 262144, keys - 2, keys - 1});
    AttnSeq s{};
    s.fresh = pick({1, 2, 255, 256, 1 << 18, 1 << 19, most - 65536, most - 65535, most - 256, most - 255, most - 254, most - 1, most});
    if (g() & 1) s.fresh -= g() % std::min(s.fresh, 300);
    s.len = pick({0, 1, 2, 63, 64, 65, 1000, 1 << 18, 1 << 19, keys - 65536, keys - 1, keys});
    // (rows + requests) * keys < 2^50
    if ((double)s.fresh * s.len >= 0x1p50) continue;
    sequence(c, s);
  }
  printf("bad %ld of %ld\n", bad, seen);
  return bad != 0 || seen < 100000;
}
"""


def test_numbers_of_31_bits(tmp_path):
    run(tmp_path, LIMITS)
