"""AdamW's host side: what its step makes of a count of steps, and what optim.AdamW refuses to load (no GPU needed)."""
import os
import subprocess
from types import SimpleNamespace

import pytest
import torch

from paper_2309_15812_amd import build, optim

POWERS = r"""
#include <math.h>
#include <stdio.h>
#include "o1d_adam.h"
using namespace o1d::rows;
// Every count ends: the loop over its bits, and the count after the step.
int main() {
  for (int found : {-2147483647 - 1, -2147483647, -3, -2, -1, 0, 1, 2, 19, 1000, 65535, 0x3fffffff, 0x7ffffffe, 0x7fffffff}) {
    const int t = steps_taken(found) + 1;
    if (t < 1 || (found >= 0 && found < 0x7fffffff && t != found + 1) || (found < 0 && t != 1)) {
      printf("step %d after %d\n", t, found);
      return 1;
    }
    for (double b : {0., 0.5, 0.9, 0.999, 0.9999999}) {
      const double got = power(b, t), want = pow(b, (double)t);
      // (a squaring doubles the error that there is: 2 t roundings at most)
      if (!(fabs(got - want) <= want * 2. * t * 1.2e-16 + 1e-300)) {
        printf("%g^%d: %g for %g\n", b, t, got, want);
        return 1;
      }
    }
  }
  return 0;
}
"""


def test_counts_of_steps_end(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(POWERS)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC)))
    subprocess.run(["g++", "-O1", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", build.CSRC, "-I", os.path.join(rocm, "include"),
                    str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("steps", [[-1, 0], [-3, 0], [5, 1], [5, -1], [5], [5, 0, 0]])
def test_counts_that_no_step_left_are_not_loaded(steps):
    opt = object.__new__(optim.AdamW)  # (states themselves are on a GPU)
    opt.groups = [{"lr": 0.1, "state": SimpleNamespace(sizes=[5], m=torch.zeros(128), master=None)}]
    held = {"sizes": [5], "m": torch.zeros(128), "v": torch.zeros(128), "step": torch.tensor(steps, dtype=torch.int32), "ms": None, "vs": None,
            "master": None}
    with pytest.raises(ValueError, match="step must be"):
        opt.load_state_dict({"groups": [{"lr": 0.2, "state": held}]})
    assert opt.groups[0]["lr"] == 0.1


def test_parameters_that_no_gradient_reaches():
    p = torch.nn.Parameter(torch.zeros(3, 4))
    with pytest.raises(TypeError):
        optim.AdamW(p)
    for bad in ([p * 2], [p[0]], list(p), [{"params": [p.t()]}], ["p"], [{"params": "p"}]):
        with pytest.raises(ValueError, match="leaf"):
            optim.AdamW(bad)
