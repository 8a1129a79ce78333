"""Bounds of the calls for packed pages, on the host: which pages the packing kernels walk (their own bounds and their own loop, for words in the arrays that
hold anything), and the sums that the page tables' launches keep in the workspace."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2505_13544_amd import binding as B

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


SUMS = r"""
#include "decode_schedule.h"
#include <initializer_list>
using namespace mtla;
int main() {
  for (int most = 1; most <= 65535; ++most) {
    const long long room = fit_scratch_bytes(most);
    if (room > most * 96LL * 4) return 1;   // a context's smallest query: one head, r = 64 and 32 RoPE columns
    for (int batch : {1, 64, 65, 1023, 1024, 1025, most - 1, most})
      if (batch >= 1 && batch <= most && (fit_groups(batch) * fit_group(batch) < batch || 16LL * (fit_groups(batch) + 1) > room)) return 2;
  }
  return 0;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_the_sums_of_the_page_tables_fit_where_they_lie(tmp_path):
    (tmp_path / "main.cpp").write_text(SUMS)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    subprocess.run([str(tmp_path / "main")], check=True)


def test_page_tables_refuse_a_workspace_that_is_not_aligned():
    ctx = B.Context(n_heads=8, d_head=64, r=256, d_rope=32, d_hyper=64, stride=2, max_batch=16, max_slots=640, dtype="bf16", page_slots=64, n_pages=40)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)
    pool = B.PagePool(ints(16, 10), ints(16), ints(16), ints(40), ints(4))
    for workspace in (1028, 1032, 1025):
        assert ctx.pages_fit_status(pool, None, 1024, None, 1, 0, 16, None, workspace) == B.MTLA_ERR_INVALID_ARG


CHUNKS = r"""
#include "bounds.h"
#include <climits>
#include <initializer_list>
int main() {
  for (int live : {0, 1, 31, 32, 33, 640, INT_MAX - 1, INT_MAX})
    for (int chunk : {32, 64, 96, 1024, 1 << 30, INT_MAX - 31})
      if (mtla::chunks_of(live, chunk) != (live + (long long)chunk - 1) / chunk) return 1;
  return 0;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_chunks_of_any_size(tmp_path):
    (tmp_path / "main.cpp").write_text(CHUNKS)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-ftrapv", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    subprocess.run([str(tmp_path / "main")], check=True)


@pytest.mark.parametrize("page_slots,n_pages", [(0, 0), (64, 40)])
@pytest.mark.parametrize("max_slots", [1, 64, 65, 640])
def test_workspace_for_a_chunk_that_holds_every_slot(max_slots, page_slots, n_pages):
    ctx = B.Context(n_heads=8, d_head=64, r=256, d_rope=32, d_hyper=64, stride=2, max_batch=16, max_slots=max_slots, dtype="bf16", page_slots=page_slots, n_pages=n_pages)
    sizes = []
    for chunk in (1024, 1 << 30, (1 << 31) - 32):
        ctx.set_decode_chunk(chunk)
        sizes.append(ctx.workspace_bytes())
    assert sizes[0] == sizes[1] == sizes[2]
