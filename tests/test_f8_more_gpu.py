"""Products of 8-bit operands: weights of another type than the input, calls with odd arguments.  Bounds as in test_f8_gpu.py."""
import math

import pytest
import torch

from paper_2309_15812_amd import ops
from test_f8_gpu import E, value
from test_rows_gpu import ACTS, BF16, DEV, DTYPES, F32, near, randn, u

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "silu"])
def test_a_float32_weight_of_bfloat16_inputs_keeps_its_gradient(act):
    x, w = randn(150, 70, seed=1, dt=BF16), randn(45, 70, seed=2, std=0.1).requires_grad_(True)
    dy = randn(150, 45, seed=3, dt=BF16)
    ops.F8LinearFunction.apply(x, w, None, act).backward(dy)
    assert w.grad.dtype is F32
    pre = ops.f8_linear_fwd(ops.pack_f8(x), ops.pack_f8(w.detach()), act=act, save="pre")[1]
    dh = dy if act == "none" else ops.act_bwd(pre, dy, act)
    D, X = value(ops.pack_f8(dh, "e5m2", along="rows")), value(ops.pack_f8(x, along="rows"))
    want, mag = D @ X.t(), D.abs() @ X.abs().t()
    e = (150 + 16) * E * mag
    near(w.grad, want, e + u(F32) * (want.abs() + e), "dw")
    w.grad = None
    ops.F8LinearFunction.apply(x[:0], w).sum().backward()
    assert w.grad.dtype is F32 and not w.grad.any()


def test_numbers_that_are_none_of_cs():
    x, w = randn(2, 9, 24, seed=10), randn(24, seed=11)
    for groups in (2 ** 31, 2 ** 40, 2 ** 63, 2 ** 70, -2 ** 70):
        with pytest.raises(ValueError):
            ops.gn_fwd(x, w, w, groups)
    p = ops.pack_f8(randn(6, 40, seed=12))
    for cols in (40.0, "40", None):
        with pytest.raises(TypeError):
            ops.F8(p.q, p.e, cols)
    for cols in (2 ** 40, 2 ** 70, 0, -40):
        with pytest.raises(ValueError):
            ops.F8(p.q, p.e, cols)
    assert torch.equal(ops.f8_linear_fwd(ops.F8(p.q, p.e, torch.tensor(40)), p), ops.f8_linear_fwd(p, p))


def test_sums_asked_for_by_any_true_value():
    x = randn(200, 40, seed=13)
    for along, parts in (("rows", 2), ("both", 3)):
        want = ops.pack_f8(x, along=along, sums=True)
        for sums in (1, "yes", torch.tensor(True)):
            got = ops.pack_f8(x, along=along, sums=sums)
            assert len(got) == parts and torch.equal(got[-1], want[-1])
        for sums in (0, None, torch.tensor(False)):
            got = ops.pack_f8(x, along=along, sums=sums)
            assert isinstance(got, ops.F8) if along == "rows" else len(got) == 2


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_what_an_operand_stands_for(fmt):
    # every exponent, 0 and 255 among them
    p = ops.pack_f8(randn(256, 200, seed=14), fmt)
    p.e[0], p.e[1] = torch.arange(256, device=DEV), torch.arange(255, -1, -1, device=DEV)
    q = p.q[:, :200].double()
    scale = (2.0 ** (p.e[:, :256].double() - 127)).t().repeat_interleave(128, 1)[:, :200]
    want = torch.where(p.e[:, :256].t().repeat_interleave(128, 1)[:, :200] == 255, math.nan, q * scale)
    near(p.float(), want.float().double(), 0 * want.nan_to_num(0), fmt)  # (powers of two: rounded only below 2^-126)
    y = ops.f8_linear_fwd(p, ops.pack_f8(randn(9, 200, seed=15)), dtype=F32)
    top = p.e[:, :256].amax(0)
    assert torch.isnan(y[top == 255]).all()
    # (200 products of at most 57344 and 8 times 2^(228 - 127) stay in float32; larger scales may leave it)
    assert torch.isfinite(y[top <= 228]).all()
