"""What products ask of a device once (csrc/sp_known.h, plain C++), by threads that come at the same time."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2504_04104_amd", "csrc")
DRIVER = r"""
#include <stdio.h>
#include <thread>
#include <vector>
#include "sp_known.h"
KnownNumbers<4> g;
std::atomic<int> asked[4], wrong;
int main() {
  std::vector<std::thread> all;
  for (int t = 0; t < 8; ++t)
    all.emplace_back([] {
      for (int i = 0; i < 4000; ++i) {
        const int dev = i % 4;
        const int n = g.of(dev, [dev] { ++asked[dev]; return dev == 3 ? 0 : 100 + dev; });
        if (n != (dev == 3 ? 0 : 100 + dev)) ++wrong;
      }
    });
  for (auto& t : all) t.join();
  bool few = asked[3] == 8 * 1000;                 // not known: asked every time
  for (int d = 0; d < 3; ++d) few = few && asked[d] >= 1 && asked[d] <= 8;
  printf("%s\n", few && !wrong ? "right" : "wrong");
  return 0;
}
"""


def test_threads_learn_a_number_without_a_race(tmp_path):
    (tmp_path / "d.cpp").write_text(DRIVER)
    exe = str(tmp_path / "d")
    built = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=thread", "-I", CSRC, str(tmp_path / "d.cpp"), "-o", exe], capture_output=True, text=True)
    if built.returncode != 0 and "tsan" in built.stderr:
        pytest.skip("no thread sanitizer to link with")
    assert built.returncode == 0, built.stderr
    r = subprocess.run([exe], capture_output=True, text=True)
    if "unexpected memory mapping" in r.stderr:
        pytest.skip("the thread sanitizer does not run on this kernel")
    assert r.returncode == 0 and r.stdout == "right\n" and "data race" not in r.stderr, r.stderr[:2000]
