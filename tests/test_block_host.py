"""The residual block's module on the host: what its casts do to the angles."""
import copy

import pytest
import torch

from paper_2309_15812_amd.block import OrientedBlock


@pytest.mark.parametrize("directions", [2, 7, 8])
@pytest.mark.parametrize("cast", [lambda m: m.bfloat16(), lambda m: m.to(torch.bfloat16), lambda m: m.half().float().bfloat16(),
                                  lambda m: torch.nn.Sequential(m).bfloat16()[0], lambda m: m.double(),
                                  lambda m: copy.deepcopy(m.bfloat16())])
def test_the_angles_stay_float32_when_the_module_is_cast(directions, cast):
    block = OrientedBlock(28, 5, directions=directions)
    want = ((torch.arange(28) * directions // 28) * (180.0 / directions)).float()
    assert torch.equal(block.theta, want)
    block = cast(block)
    assert block.theta.dtype == torch.float32 and torch.equal(block.theta, want)
    assert torch.equal(block.state_dict()["theta"], want)
    assert block.w1.dtype == block.ln_w.dtype == block.w_dw.dtype != torch.float32


def test_the_angles_move_and_load_with_the_module():
    block = OrientedBlock(24, 5).bfloat16()
    with torch.device("meta"):
        empty = OrientedBlock(24, 5)
    empty = empty.bfloat16().to_empty(device="cpu")
    empty.load_state_dict(block.state_dict())
    assert empty.theta.dtype == torch.float32 and torch.equal(empty.theta, block.theta) and empty.w1.dtype == torch.bfloat16
