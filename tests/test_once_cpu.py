"""csrc/once.h under the thread sanitizer (host code alone), and that the library's launchers keep to it."""
import glob
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_09200_amd", "csrc")

HARNESS = r"""
#include "once.h"
#include <stdio.h>
#include <thread>
#include <vector>

static occ::Once once[3], failing;
static int facts[3], calls[3], tries;   // plain: ordered by Once alone

int main() {
  std::vector<std::thread> threads;
  std::atomic<int> bad{0};
  for (int t = 0; t < 8; ++t)
    threads.emplace_back([&, t] {
      for (int i = 0; i < 300; ++i) {
        const int k = (t + i) % 3;
        if (!once[k].run([&] { facts[k] = 40 + k; ++calls[k]; return true; })) ++bad;
        if (facts[k] != 40 + k) ++bad;
        if (failing.run([&] { return ++tries >= 5; }) && tries != 5) ++bad;
      }
    });
  for (std::thread &t : threads) t.join();
  for (int k = 0; k < 3; ++k) bad += calls[k] != 1;
  printf("bad %d tries %d\n", bad.load(), tries);
  return bad != 0 || tries != 5;
}
"""


def test_once_under_the_thread_sanitizer(tmp_path):
    flags = ["-std=c++17", "-O1", "-g", "-pthread", "-fsanitize=thread"]
    probe = tmp_path / "probe.cpp"
    probe.write_text("int main() { return 0; }\n")
    if subprocess.run(["g++", *flags, str(probe), "-o", str(tmp_path / "probe")], capture_output=True).returncode or \
            subprocess.run([str(tmp_path / "probe")], capture_output=True).returncode:
        pytest.skip("no thread sanitizer here")
    src = tmp_path / "once.cpp"
    src.write_text(HARNESS)
    subprocess.run(["g++", *flags, "-Wall", "-I", CSRC, str(src), "-o", str(tmp_path / "once")], check=True)
    r = subprocess.run([str(tmp_path / "once")], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "WARNING" not in r.stderr, r.stdout + r.stderr


def test_launchers_keep_no_plain_flags():
    """A host-side static that calls change is a Once: two threads' first calls may come together."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        plain = re.findall(r"^\s+static (?:bool|int|float|double|char|void \*)\s*\w+(?:\[[^\]]*\])*\s*(?:=[^(]*)?;", open(path).read(), re.M)
        assert not plain, (path, plain)


def test_dynamic_lds_limits_do_not_depend_on_the_call():
    """The limit is the kernel's, for every host thread: one call's own size would lower what another is about to launch
    with.  Only device facts, constants and a kernel's own bytes may be in it."""
    asked = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip"))):
        for m in re.finditer(r"hipFuncAttributeMaxDynamicSharedMemorySize,\s*([^;]*?)\)\s*(?:==|!=) hipSuccess", open(path).read()):
            asked.append((os.path.basename(path), " ".join(m.group(1).split())))
    known = {"di->max_lds_per_wg", "p.max_lds_per_wg", "p.max_lds_per_wg - v->lds", "di.max_lds_per_wg - own",
             "kMaxTokens * kMaxExperts * 4", "lds"}   # lds: the wide norms' 2 x 64 KiB
    assert len(asked) >= 6 and {a for _, a in asked} <= known, asked
