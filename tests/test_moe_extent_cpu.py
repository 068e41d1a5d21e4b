"""The byte ranges of the expert layer's weights and scales that its descriptors open, for every block of rows that a
task of either product can have: within the expert's bytes, so that the last expert's stay within the batch's."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_09200_amd", "csrc")

HARNESS = r"""
#include "moe_extent.h"
#include <stdio.h>
#include <vector>

using namespace occ;

static int bad;

// Tasks of `rbs` blocks of 16 rows, as many as `rows` need: every row is opened once, nothing past the matrix.
static void walk(int rows, int rbs, unsigned code_pitch, unsigned scale_pitch) {
  std::vector<int> seen(rows);
  const size_t codes = (size_t)rows * code_pitch, scales = (size_t)((rows + 15) / 16) * scale_pitch;
  for (int row0 = 0; row0 < rows; row0 += 16 * rbs)
    for (int b = 0; b < rbs; ++b) {
      const int r = moe_block_row(row0, b, rows);
      const MoeExtent w = moe_rows_extent(code_pitch, r, rows), s = moe_scales_extent(scale_pitch, r, rows);
      if ((w.bytes > 0 && w.at + w.bytes > codes) || w.bytes % code_pitch) ++bad;
      if (s.bytes > 0 && s.at + s.bytes > scales) ++bad;
      if ((w.bytes > 0) != (s.bytes > 0)) ++bad;
      if (w.bytes > 0 && (s.at != (size_t)(r / 16) * scale_pitch || s.bytes != scale_pitch)) ++bad;
      for (unsigned i = 0; i < w.bytes / code_pitch; ++i) ++seen[r + i];
    }
  for (int n : seen) bad += n != 1;
}

int main() {
  for (int rows = 8; rows <= 1064; rows += 8)
    for (int rbs = 1; rbs <= 8; rbs *= 2)
      for (unsigned pitch : {16u, 256u, 5008u}) walk(rows, rbs, pitch, 256u * (pitch / 256 + 1));
  walk(65536, 2, 131072, 32768);
  walk(65528, 8, 131072, 32768);
  // a block that starts at the matrix's end, the last scale tile being full: the tile there is the next expert's
  if (moe_scales_extent(256, 32, 32).bytes != 0 || moe_rows_extent(256, 32, 32).bytes != 0) ++bad;
  printf("%d\n", bad);
  return bad != 0;
}
"""


def test_descriptors_stay_within_an_experts_bytes(tmp_path):
    src = tmp_path / "extent.cpp"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(src), "-o", str(tmp_path / "extent")], check=True)
    r = subprocess.run([str(tmp_path / "extent")], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def test_the_kernels_open_no_other_ranges():
    text = open(os.path.join(CSRC, "moe.hip")).read()
    body = text[text.index("struct Rows16 {"):text.index("// Where chunk c of a row of a staged unit lies")]
    assert body.count("rsrc_of(") == 2 and "w.at, w.bytes" in body and "s.at, s.bytes" in body
    assert text.count("moe_block_row(") == 2
