"""Which pages the packing kernels walk, compiled and run on the host: their own bounds and their own loop, for words in the arrays that hold anything."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_13544_amd", "csrc")

# (built so that an int that overflows ends the program)
PROGRAM = r"""
#include <cstdio>
#include "bounds.h"
int main() {
  int first, end, max_pages, each;
  while (scanf("%d %d %d %d", &first, &end, &max_pages, &each) == 4) {
    const int lo = mtla::pages_inside(first, max_pages), hi = mtla::pages_inside(end, max_pages);
    int n = 0, least = max_pages, most = -1;
    for (int block = 0; block < each; ++block)  // the grid of a launch
      for (int page = lo + block; page < hi; page += each) {
        ++n;
        least = page < least ? page : least;
        most = page > most ? page : most;
      }
    printf("%d %d %d\n", n, least, most);
  }
  return 0;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_pages_that_a_launch_walks(tmp_path):
    (tmp_path / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-ftrapv", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    big, small = (1 << 31) - 1, -(1 << 31)
    words = [small, -7, -1, 0, 1, 3, 9, 10, 11, 1 << 20, big - 1, big]
    calls = [(f, e, mp, each) for f in words for e in words for mp in (1, 10) for each in (1, 2, 10) if each <= mp]
    calls += [(f, big, 1 << 27, 1 << 12) for f in (big, (1 << 27) - 1)]                 # the most pages that there can be, in a launch of many
    run = subprocess.run([str(tmp_path / "main")], input="\n".join("%d %d %d %d" % c for c in calls), check=True, capture_output=True, text=True)
    for (f, e, mp, _), line in zip(calls, run.stdout.splitlines()):
        n, least, most = map(int, line.split())
        want = range(min(max(f, 0), mp), min(max(e, 0), mp))
        assert n == len(want) and (n == 0 or (least, most) == (want[0], want[-1])), (f, e, mp)


def test_the_kernel_bounds_both_ends():
    # the kernel takes its pages through that function, and from nowhere else
    src = open(os.path.join(CSRC, "pages_pack.hip")).read()
    assert src.count("a.first[b]") == src.count("pages_inside(a.first ? a.first[b] : 0, a.pages.max_pages)") == 1
    assert src.count("a.end[b]") == src.count("pages_inside(a.end[b], a.pages.max_pages)") == 1
