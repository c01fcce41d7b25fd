"""Which parts of a CTA get NaN after a given-up wait, run on the host from the kernels' own header: every part that one of its warps has not begun, in the
ring through which they are handed out, taken but not published, or still to come; none twice."""
import os
import shutil
import subprocess

import pytest

from paper_2608_23599_b200 import build as _build

HARNESS = r"""
#include <cstdio>
#include <random>
#include <vector>
#include "gkv_chunk.h"

struct Part {
  int tile;
};

int main() {
  std::mt19937 g(1);
  auto upto = [&](int n) { return static_cast<int>(g() % (n + 1)); };
  for (int i = 0; i < 200000; ++i) {
    const int parts = 1 + upto(9);
    const bool whole = upto(1);                       // the parts are taken one by one, and what was not taken another CTA has
    // `published` parts went through the ring, the last of them without a tile where there were no more; every warp has begun those that were put over
    const int published = upto(parts + 1);
    Part ring[3] = {{-7}, {-7}, {-7}};
    for (int n = 0; n < published; ++n) ring[n % 3] = {n < parts ? n : -1};
    const bool hand = published < parts && upto(1);
    int begun = parts;                                // by the slowest of the warps
    for (int w = 0; w < 11; ++w) begun = std::min(begun, std::max(0, published - 3) + upto(std::min(3, published)));
    std::vector<int> seen(parts, 0);
    int at = published;
    bool wrong = false;
    gkv::parts_left<3>(ring, published, hand, Part{published},
                       [&](Part& p) {
                         if (whole || ++at >= parts) return false;
                         p.tile = at;
                         return true;
                       },
                       [&](const Part& p) {
                         if (p.tile < 0 || p.tile >= parts || seen[p.tile]++) wrong = true;
                       });
    // where nothing is in hand, what was not published was not taken: of a range, only before the first part or behind the last
    const int taken = hand ? (whole ? published + 1 : parts) : std::min(published, parts);
    for (int n = 0; n < parts; ++n) wrong = wrong || (n >= begun && n < taken && !seen[n]) || (seen[n] && n >= taken) || (seen[n] && n < published - 3);
    if (wrong) {
      std::printf("case %d: parts %d published %d hand %d whole %d begun %d\n", i, parts, published, hand, whole, begun);
      return 1;
    }
  }
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_every_part_that_was_not_begun(tmp_path):
    src = tmp_path / "left.cpp"
    src.write_text(HARNESS)
    exe = str(tmp_path / "left")
    subprocess.run(["g++", "-O1", "-g", "-fsanitize=address,undefined", "-std=c++17", f"-I{_build.CSRC}", str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0, r.stdout + r.stderr
