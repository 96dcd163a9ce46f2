"""Rules of the paged calls that host code alone decides by, compiled by themselves."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_01701_amd", "csrc")

JOIN = r"""
#include <cstdio>
#include <initializer_list>
#include "t2v_paged.h"
int main() {
  for (long long rows : {1LL, 32LL, 33LL, 1536LL, (1LL << 31) - 1}) std::printf("%d ", t2v::paged_join_blocks(rows, 32, 4));
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_the_join_goes_by_the_rows_of_a_call(tmp_path):
    """A chunk of 512 tokens, three heads a key head, is joined alike in a cache of one sequence and in one with 255 idle ones beside it."""
    src, exe = tmp_path / "join.cpp", str(tmp_path / "join")
    src.write_text(JOIN)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(src), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    assert subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split() == ["1", "1", "4", "4", "4"]
