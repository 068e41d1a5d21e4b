"""The launches of occ_rope (csrc/rope_plan.h): every token has a workgroup, and a launch has fewer than 2^32 threads in a
dimension, which is what HIP takes, up to the documented 2^24 rows."""
import pytest
import torch

from test_attn_plan_cpu import run

GRID = r"""
#include "rope_plan.h"
#include <stdio.h>

int main() {
  long bad = 0, seen = 0;
  const int rows[] = {1, 2, 255, 256, 257, 4095, 4096, 4097, 100003, 1 << 22, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, (1 << 24) - 1, 1 << 24};
  const int items[] = {1, 2, 3, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 320, 321, 447, 448, 449, 511, 512, 513, 1000, 65536, 512 * 196608};
  for (int cus : {1, 64, 256, 304})
    for (int t : rows)
      for (int per : items) {
        const occ::RopeGrid g = occ::rope_grid(t, per, cus);
        ++seen;
        if (g.tokens < 1 || g.threads < 64 || g.threads > 512 || g.threads % 64 || g.x < 1 || g.y < 1 || g.y > 65535) ++bad;
        if ((int64_t)g.x * g.tokens < t || (int64_t)(g.x - 1) * g.tokens >= t) ++bad;
        if ((int64_t)g.x * g.threads >= (int64_t)1 << 32 || (int64_t)g.y * g.threads >= (int64_t)1 << 32) ++bad, printf("%d rows %d items\n", t, per);
        // (cos, sin) of all its tokens' pairs, at most 512 a token and 16 an item, fit into 64 KB of LDS
        if ((int64_t)g.tokens * 512 * 8 > 65536 && (int64_t)g.tokens * per * 16 * 8 > 65536) ++bad;
        if ((int64_t)g.tokens * per > 2147483647) ++bad;
      }
  printf("bad %ld of %ld\n", bad, seen);
  return bad != 0;
}
"""


def test_every_launch_fits(tmp_path):
    run(tmp_path, GRID)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,heads,D", [(1 << 23, 14, 66), (1 << 24, 5, 126)])
def test_many_rows(rows, heads, D):
    """2^32 threads and more if each token had a workgroup of its own (halves of odd length: an item is a pair): the bits of the
    same rows a few at a time."""
    from gpu_common import DEV
    from paper_2606_09200_amd import binding as occ
    q = torch.empty((rows, heads, D), dtype=torch.bfloat16, device=DEV)
    turns = occ.rope_turns(D // 2, device=DEV)
    positions = torch.arange(rows, dtype=torch.int32, device=DEV)
    some = [0, 1, 255, rows // 2 - 1, rows // 2, rows // 2 + 1, rows - 2, rows - 1]
    values = torch.randn((len(some), heads, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    q[some] = values
    want = occ.occ_rope(values.clone(), None, positions[some].contiguous(), turns)[0]
    occ.occ_rope(q, None, positions, turns)
    assert torch.equal(q[some], want)
