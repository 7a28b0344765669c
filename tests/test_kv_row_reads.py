"""What the kernels of the paged cache read of rows that may lie anywhere, from their own header compiled by g++: words with an element of the row and no
others, and of a cached row no more than its last 16 bytes.  A read of anything else may fall in no memory, so that it is looked for here and not on a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2410_05911_gb300", "csrc")
CUDA_INC = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
E = 16  # elements of a lane

HARNESS = r"""
#include "aecct_internal.h"
#include <cstdio>
int main() {
  for (int left = -300; left <= 256; ++left)
    for (int odd = 0; odd < 2; ++odd)
      for (int i = 0; i < 9; ++i) std::printf("w %d %d %d %d\n", left, odd, i, int(aecct::reads_new_word(left, i, odd, 16)));
  for (int left = -300; left <= 256; ++left)
    for (int size = 1; size <= 2; ++size)
      for (int follows = 0; follows < 2; ++follows) std::printf("c %d %d %d %d\n", left, size, follows, aecct::reads_cached(left, size, follows));
}
"""


@pytest.fixture(scope="module")
def reads(tmp_path_factory):
    if not os.path.isdir(CUDA_INC):
        pytest.skip("CUDA headers not found")
    d = tmp_path_factory.mktemp("kv_row_reads")
    src, exe = d / "harness.cpp", d / "harness"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{CUDA_INC}", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    lines = [line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()]
    return {(line[0], *map(int, line[1:4])): int(line[4]) for line in lines}


def test_words_with_an_element_of_a_new_row(reads):
    for left in range(-300, 257):
        for odd in (0, 1):
            # element e of the lane lies in word (e + odd) / 2
            want = {(e + odd) // 2 for e in range(min(left, E))}
            assert {i for i in range(9) if reads["w", left, odd, i]} == want, (left, odd)


def test_no_more_than_a_cached_rows_last_16_bytes(reads):
    for left in range(-300, 257):
        for size in (1, 2):
            assert reads["c", left, size, 0] == max(left, 0)
            n = reads["c", left, size, 1]
            assert n * size % 16 == 0 and (n == 0 if left <= 0 else 0 <= n - left < 16 // size), (left, size)
