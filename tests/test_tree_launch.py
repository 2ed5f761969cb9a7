"""A tree's launch that no kernel serves is an error, not a call that computes nothing:
asked of the library's own launch function, which starts nothing then."""
import os
import subprocess

import pytest

from paper_2605_06675_amd import build

SOURCE = """
#include <cstdio>
#include "rq_block.h"

int main() {
  // 64 rows of 128 channels with a cap, a window or slopes
  for (int fmt : {RQ_INT8, RQ_E4M3})
    for (int bf16 = 0; bf16 < 2; ++bf16)
      for (int waves : {4, 8}) {
        float slope = 1.0f;
        rq::BlockTreeLaunch a{};
        a.c.B = a.c.H = a.G = a.splits = 1;
        a.c.D = 128;
        a.c.fmt = fmt;
        a.c.is_bf16 = bf16;
        a.n = a.group_rows = 64;
        a.waves = waves;
        a.cap = 1.0f;
        a.window = 3;
        a.slopes = &slope;
        std::printf("%d\\n", (int)rq::launch_tree_rows(a, nullptr));
      }
}
"""


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no compiler")
def test_a_launch_without_a_kernel_is_an_error(tmp_path):
    source, program = tmp_path / "ask.cpp", tmp_path / "ask"
    source.write_text(SOURCE)
    subprocess.run([build.HIPCC, "-std=c++17", "--offload-host-only", "-w", "-x", "hip", str(source), "-x", "none", build.OUT,
                    f"-I{build.CSRC}", f"-Wl,-rpath,{build.HERE}", "-o", str(program)], check=True)
    said = subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.split()
    assert said == ["1"] * 8                                  # hipErrorInvalidValue
