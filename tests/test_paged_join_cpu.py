"""The range of parts that the joining kernel of the attention over a paged cache walks, for any number found in memory."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "swarm_paged.h"
int main() {
  const int lasts[] = {-2147483647 - 1, -2147483647, -148, -1, 0, 1, 2, 73, 146, 147, 148, 149, 1184, 1 << 20, 2147483646, 2147483647};
  for (int ctas = 1; ctas <= 148; ++ctas)
    for (int first = 0; first < ctas; ++first)
      for (int last : lasts) {
        const int n = swarm::parts_between(first, last, ctas);
        const bool steady = last >= first && last < ctas;                       // what a call whose lengths stay as they are finds
        if (n < 1 || first + n > ctas || (steady && first + n - 1 != last)) { std::printf("%d %d %d: %d\n", ctas, first, last, n); return 1; }
      }
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("nvcc") is None, reason="needs nvcc")
def test_parts_of_an_item_stay_inside_the_workspace(tmp_path):
    source, program = tmp_path / "parts.cu", tmp_path / "parts"
    source.write_text(PROGRAM)
    package = os.path.join(ROOT, "paper_1910_12308_b200")
    done = subprocess.run(["nvcc", "-std=c++17", "-arch=sm_100a", "-I", os.path.join(package, "csrc"), "-I", os.path.join(ROOT, "include"),
                           str(source), "-o", str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    done = subprocess.run([str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
