"""The parts of a verification's workspace, from the rule that its kernels use (csrc/verify_cut.h, compiled for the host): a
workspace for T rows of V logits is enough for every call of no more."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_13804_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "verify_cut.h"
// The most T * slices of the calls of up to T rows, for every T in turn, against the bound; and that the bound never falls.
int main(int, char** argv) {
  const int slots = std::atoi(argv[1]);
  const int Vs[] = {1, 2047, 2048, 2049, 4097, 20000, 32000, 51200, 51201, 65536, 65537, 102401, 152064, 1700000, 1 << 24};
  const int Bs[] = {1, 2, 7, 64, 255, 256};
  size_t below = 0;
  for (int V : Vs) {
    size_t most = 0, last = 0;
    for (int T = 0; T <= 5000; ++T) {
      for (int B : Bs)
        for (int drafted = 0; drafted < 2; ++drafted) {
          const sp::Cut c = sp::verify_cut(T, B, V, 6, drafted, false, slots);
          if (c.slices < 1 || c.slices > sp::kRowSlices) return std::printf("slices %d\n", c.slices), 1;
          most = std::max(most, (size_t)T * c.slices);
        }
      const size_t n = sp::verify_parts(T, V, slots);
      if (n < most) return std::printf("T %d V %d: %zu of %zu\n", T, V, n, most), 1;
      if (n < last) return std::printf("T %d V %d: falls\n", T, V), 1;
      last = n;
    }
    if (last < below) return std::printf("V %d: falls\n", V), 1;
    below = last;
  }
  for (int T : {1, 5, 100, 406, 700, 5000, 1 << 24}) {
    size_t last = 0;
    for (int V = 1; V < (1 << 24); V += V / 64 + 1) {
      const size_t n = sp::verify_parts(T, V, slots);
      if (n < last) return std::printf("T %d V %d: falls\n", T, V), 1;
      last = n;
    }
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("cut")
    (d / "main.cc").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, str(d / "main.cc"), "-o", str(d / "main")], check=True)
    return str(d / "main")


@pytest.mark.parametrize("slots", [4, 592, 608])
def test_a_workspace_is_enough_for_smaller_calls(program, slots):
    r = subprocess.run([program, str(slots)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
