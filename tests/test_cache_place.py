"""Rows that a read of the cache looks up: whatever the block table and the ranges hold, the row that is loaded lies in the planes.  The rule
is compiled for the host; the kernel takes its addresses from it alone."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_01831_b200", "csrc")

CHECK = r"""
#include <climits>
#include <cstdio>
#include <initializer_list>
#include "cache_place.cuh"
int main() {
  long long bad = 0, dead = 0, alive = 0;
  for (int32_t nb : {1, 4, 8192, 1 << 20})
    for (int32_t heads : {1, 8, 128})
      for (int32_t bt : {1, 5, 16, 1024})
        for (int32_t max_blocks : {1, 3, 1 << 20}) {
          const int64_t rows = (int64_t)nb * heads * bt, capacity = (int64_t)max_blocks * bt;
          for (int64_t token : {(int64_t)INT32_MIN * 2, (int64_t)-1, (int64_t)0, (int64_t)bt - 1, capacity - 1, capacity, capacity + 7, (int64_t)INT32_MAX * 2})
            for (int32_t id : {INT32_MIN, -nb, -1, 0, nb - 1, nb, nb + 1, INT32_MAX}) {
              const bool in = lynx::in_table(token, max_blocks, bt), want = token >= 0 && token < capacity && id >= 0 && id < nb;
              const lynx::CacheRow r = lynx::cache_row(in, id, token - token / bt * bt, nb, heads, bt);
              const int64_t last = r.row + (int64_t)(heads - 1) * bt;                 // of the token's last head
              bad += in != (token >= 0 && token < capacity) || r.live != want || r.row < 0 || last >= rows;
              bad += want && r.row != (int64_t)id * heads * bt + token % bt;
              dead += !want;
              alive += want;
            }
        }
  std::printf("%lld %d", bad, dead > 1000 && alive > 100);
}
"""


def test_no_row_outside_the_planes(tmp_path):
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(CHECK)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout == "0 1"


@pytest.mark.parametrize("plane", ["anchor", "residual", "meta"])
def test_the_kernel_reads_at_that_row(plane):
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "cache_rows.cu")).read())
    body = code[code.index("cache_read_kernel("):code.index("inline bool aligned(")]
    assert re.findall(r"int64_t (\w+) = ([^;]*\bsrc\b[^;]*);", body) == [("s", "src.row + (int64_t)min(h0 + u, last - 1) * p.bt")]
    index = {"anchor": "s * 8 + l", "residual": "s * 8 + l", "meta": "s"}[plane]
    assert re.findall(rf"ld_dep\({plane} \+ ([^)]*)\)", body) == [index]
    assert re.findall(r"\bsrc = ([^;]*);", body) == ["{0, false}", "cache_row(true, ld_dep(p.table + (int64_t)b * p.max_blocks + i), token - i * p.bt, "
                                                     "p.num_blocks, p.heads, p.bt)"]
