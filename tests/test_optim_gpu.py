"""AdamW as programs use it: between forward and backward passes, after parameters were written, with states of other programs."""
import pytest
import torch

from paper_2309_15812_amd import ops, optim
from paper_2309_15812_amd.block import OrientedBlock, OrientedBlock8
from test_rows_gpu import BF16, DEV, DTYPES, F32, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", DTYPES)
def test_a_backward_from_before_the_step_is_refused(dt):
    # (its saved weights are no longer those of the forward)
    for kind in (OrientedBlock, OrientedBlock8):
        torch.manual_seed(1)
        block = kind(24, 3).to(DEV).to(dt)
        opt = optim.AdamW(block.parameters(), lr=1e-2)
        loss = block(randn(2, 6, 5, 24, seed=1, dt=dt)).float().square().mean()
        loss.backward(retain_graph=True)
        opt.step()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        opt.zero_grad()
        block(randn(2, 6, 5, 24, seed=1, dt=dt)).float().square().mean().backward()  # the next one is not


def test_a_step_counts_in_the_versions_of_what_it_writes():
    ws = torch.empty(int(ops._lib.lib().o1d_adamw_workspace_bytes(1.0)), dtype=torch.uint8, device=DEV)
    for kw in ({}, {"workspace": ws}, {"max_norm": 1.0}, {"max_norm": 1.0, "workspace": ws}):
        ps = [randn(40, seed=1), randn(30, seed=2), randn(0, seed=3)]
        gs = [randn(40, seed=4), None, randn(0, seed=5)]
        state = ops.AdamState.zeros(ps)
        before = [t._version for t in (*ps, gs[0])]
        ops.adamw(ps, gs, state, **kw)
        assert [t._version for t in (*ps, gs[0])] == [before[0] + 1, *before[1:]]
        with pytest.raises(RuntimeError):
            ops.adamw(ps, gs, state, lr=-1.0, **kw)
        assert ps[0]._version == before[0] + 1


def test_inference_tensors_have_no_version():
    for kw in ({}, {"workspace": torch.empty(512, dtype=torch.uint8, device=DEV)}):
        with torch.inference_mode():
            p, g = randn(40, seed=1).clone(), randn(40, seed=2).clone()
        state = ops.AdamState.zeros([p])
        was = p.clone()
        ops.adamw([p], [g], state, lr=1e-2, weight_decay=0.0, **kw)
        assert bool(((was - p - 1e-2 * g.sign()).abs() <= 1e-5).all())
