"""The build's check of register spills."""
import os

import pytest

from paper_2309_15812_amd import build

REMARK = "x.h:1:1: remark: Function Name: {} [-Rpass-analysis=kernel-resource-usage]\n" \
         "x.h:1:1: remark:     ScratchSize [bytes/lane]: {} [-Rpass-analysis=kernel-resource-usage]\n"


def test_every_unit_with_kernels_is_checked():
    units = {os.path.basename(s) for s in build.sources()}
    assert {u for u in units if not u.startswith(build.CHECKED)} == {"o1d_api.hip", "o1d_rows_api.hip", "o1d_util.hip"}


def test_spills_beyond_the_known_ones_fail_the_build():
    kernel = "_ZN3o1d4rows12_GLOBAL__N_1{}vNS0_8MmParamsE"
    known = dict(build.SCRATCH)
    build._check_no_scratch("a.hip", "".join(REMARK.format(kernel.format(k), n) for k, n in known.items()))
    build._check_no_scratch("a.hip", REMARK.format(kernel.format("2mmItLi0ELi0ELb0EE"), 0))
    with pytest.raises(RuntimeError, match="2mmItLi0ELi0ELb0EE"):
        build._check_no_scratch("a.hip", REMARK.format(kernel.format("2mmItLi0ELi0ELb0EE"), 4))
    for k, n in known.items():
        with pytest.raises(RuntimeError, match=f"{n + 4} bytes"):
            build._check_no_scratch("a.hip", REMARK.format(kernel.format(k), n + 4))
