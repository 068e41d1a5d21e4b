// How the rows of occ_rope are dealt out among workgroups: arithmetic that the host can check.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace occ {

struct RopeGrid {
  int tokens;   // of a workgroup
  int threads;
  int x, y;     // workgroups; those of one x share its tokens' items
};

// `rows` tokens of `per_token` items on a chip of `cus`.
//   A token a workgroup, an item or two a thread, where there are plenty of tokens (several tokens where they have few items),
// dealt out among workgroups where there are few.  HIP takes fewer than 2^32 threads in a dimension: with more, workgroups have
// two tokens.
inline RopeGrid rope_grid(int rows, int per_token, int cus) {
  constexpr int kThreads = 256;
  RopeGrid g;
  g.tokens = rows >= 16 * cus ? std::max(1, kThreads / per_token) : 1;
  g.threads = rows >= cus && g.tokens == 1 ? std::min(512, (per_token + 63) / 64 * 64) : kThreads;
  if ((int64_t)rows * g.threads >= (int64_t)1 << 32 && g.tokens == 1) g.tokens = 2, g.threads = kThreads;
  const int64_t items = (int64_t)g.tokens * per_token;
  const int passes = (int)((items + g.threads - 1) / g.threads);
  g.x = (rows + g.tokens - 1) / g.tokens;
  g.y = std::max(1, std::min({passes, 4 * cus / g.x, 64}));
  return g;
}

}  // namespace occ
