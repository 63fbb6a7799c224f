"""Packing of 8-bit operands against its definition, bit by bit, and their products against 64 bits.

Tolerances are bounds, element by element.  u = 2^-24 for float32 and 2^-8 for bfloat16 results, one rounding.  Products for
float32 results are exact and summed in float32: (K + 8) 2^-24 sum |a b|.  Those for bfloat16 results are summed eight at a time,
each to 2^-13 of the power of two below the largest of the eight: eight times that of every group of eight consecutive
k, besides.  An activation adds at most its slope (below 1.2; below 2 for its derivative's) times its argument's error and
2e-6 (1 + |h|) for its own evaluation.
"""
import math

import pytest
import torch

from paper_2309_15812_amd import ops
from test_rows_gpu import ACTS, BF16, DEV, DTYPES, F32, gate, near, randn, sliced, u

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
FORMATS = {"e4m3": (torch.float8_e4m3fn, 448.0, 3, -6), "e5m2": (torch.float8_e5m2, 57344.0, 2, -14)}


def packed(x, fmt):
    """(values of q, e) by the definition, in 64 bits on the CPU."""
    _, top, digits, low = FORMATS[fmt]
    x = x.double().cpu()
    R, K = x.shape
    groups = -(-K // 128)
    g = torch.zeros(R, groups * 128, dtype=torch.float64)
    g[:, :K] = x
    g = g.view(R, groups, 128)
    fine = torch.isfinite(g)
    amax = torch.where(fine, g, 0 * g.nan_to_num(0, 0, 0)).abs().amax(-1)
    e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -300) / top))
    e = torch.where(amax * 2.0 ** -e > top, e + 1, e)  # (a logarithm next to a whole number)
    e = torch.where(amax * 2.0 ** -(e - 1) <= top, e - 1, e).clamp(min=-127)
    e = torch.where(amax > 0, e, 0 * e)
    v = g * (2.0 ** -e)[..., None]
    spacing = 2.0 ** (torch.floor(torch.log2(v.abs().nan_to_num(1, 1, 1).clamp(min=2.0 ** low))) - digits)
    q = torch.where(fine, torch.round(v / spacing) * spacing, torch.full_like(v, math.nan)).view(R, -1)
    exponents = torch.full((groups, -(-R // 16) * 16), 127, dtype=torch.uint8)
    exponents[:, :R] = (e + 127).to(torch.uint8).t()
    return q, exponents


def value(p):
    scale = 2.0 ** (p.e[:, :p.rows].double() - 127)
    return p.q[:, :p.cols].double() * scale.t().repeat_interleave(128, 1)[:, :p.cols]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,C", [(1, 1), (3, 8), (5, 127), (7, 128), (129, 129), (33, 300), (128, 16), (257, 96), (2, 1500), (700, 3)])
def test_packing_is_its_definition(M, C, dt, fmt):
    x = sliced(M, C, 7, 1, dt, 3).clone() if C % 2 else sliced(M, C, 7, 1, dt, 3)
    x *= torch.exp2(torch.arange(M, device=DEV) % 60 - 30.0).to(dt)[:, None]
    x[0] = 0
    if M > 6:
        x[1] *= 1e30
        x[2] = 3e38  # the types' ends
        x[3] = 1e-39
        x[4, C // 2], x[5, 0], x[6, C - 1] = math.nan, -math.inf, math.inf
    r, t, s = ops.pack_f8(x, fmt, along="both", sums=True)
    for got, src in ((r, x), (t, x.t())):
        q, e = packed(src, fmt)
        assert got.q.dtype is FORMATS[fmt][0] and torch.equal(got.e.cpu(), e)
        near(got.q.cpu(), q, 0 * q.nan_to_num(0), fmt)
    for got, want in ((ops.pack_f8(x, fmt), r), (ops.pack_f8(x, fmt, along="rows"), t)):
        assert torch.equal(got.q.view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(got.e, want.e)
    total = x.double().sum(0)
    e = (min(M, 128 + M // 128) + 16) * E * x.double().abs().sum(0)
    near(s, total, e + u(dt) * (total.abs() + e), "sums")


def test_scales_at_powers_of_two():
    # the least power of two that keeps the largest value in range, and ties to even
    for fmt, (_, top, digits, _) in FORMATS.items():
        for big in (top, top * (1 + 2.0 ** -10), top / 2, 1.0, 2.0 - 2.0 ** -20):
            x = torch.full((1, 128), big, device=DEV)
            x[0, 1:] = (1 + 2.0 ** -(digits + 1)) * 2.0 ** torch.arange(127, device=DEV).remainder(9).float()
            x[0, 1:] = torch.minimum(x[0, 1:], x[0, 0])
            p = ops.pack_f8(x, fmt)
            q, e = packed(x, fmt)
            assert torch.equal(p.e.cpu(), e) and torch.equal(p.q.cpu().double(), q)


def lost(A, B):
    """What sums of eight products in fixed point may lose, (M, N)."""
    K = A.shape[1]
    pad = -K % 8
    a, b = (torch.nn.functional.pad(t.abs(), (0, pad)).view(t.shape[0], -1, 8) for t in (A, B))
    got = torch.zeros(A.shape[0], B.shape[0], dtype=torch.float64, device=A.device)
    for g in range(a.shape[1]):
        got += (a[:, None, g] * b[None, :, g]).amax(-1)
    return got * 8 * 2.0 ** -13


MM = [(1, 1, 1), (1, 8, 8), (16, 768, 100), (3, 5, 2), (64, 128, 64), (65, 129, 130), (200, 384, 96), (333, 203, 309), (130, 1000, 61),
      (700, 40, 1), (129, 256, 257)]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,I,O", MM)
def test_forward(M, I, O, dt, fmt):
    for k, act in enumerate(ACTS):
        x = randn(M, I, seed=20) * torch.exp2(torch.arange(M, device=DEV) % 7 - 3.0)[:, None]
        w = randn(O, I, seed=21, std=I ** -0.5)
        px, pw = ops.pack_f8(x, fmt), ops.pack_f8(w)
        pad, lead = ((0, 0), (9, 1))[k % 2]
        b = randn(O, seed=22, dt=dt) if k != 1 else None
        res = sliced(M, O, pad, 23, dt, lead) if k != 2 else None
        y, pre = ops.f8_linear_fwd(px, pw, b, act=act, residual=res, save="pre", dtype=dt)
        X, W = value(px), value(pw)
        h, mag = X @ W.t(), X.abs() @ W.abs().t()
        eh = (I + 8) * E * mag + (lost(X, W) if dt == BF16 else 0)
        if b is not None:
            h = h + b.double()
            eh = eh + 2 * E * (mag + b.double().abs())
        near(pre, h, eh + u(dt) * (h.abs() + eh), "pre")
        want = gate(h, act)[0]
        ey = 1.2 * eh + (0 if act in ("none", "relu") else 2e-6 * (1 + h.abs()))
        if res is not None:
            want = want + res.double()
        near(y, want, ey + u(dt) * (want.abs() + ey) + 2 * E * h.abs(), act)
        assert torch.equal(ops.f8_linear_fwd(px, pw, b, act=act, residual=res, dtype=dt), y)


@pytest.mark.parametrize("dt", DTYPES)
def test_norms_of_the_errors(dt):
    """Where nothing cancels in the bounds above: a rounding of bfloat16 is 2^-8 / sqrt(3) of the values at most in the 2-norm,
    that of the sums of eight far less; float32 sums add a few 2^-24."""
    x, w = randn(512, 2048, seed=30), randn(384, 2048, seed=31)
    px, pw = ops.pack_f8(x), ops.pack_f8(w)
    want = value(px) @ value(pw).t()
    got = ops.f8_linear_fwd(px, pw, dtype=dt).double()
    assert float((got - want).norm() / want.norm()) <= (2.0 ** -8 / 3 ** 0.5 + 1e-4 if dt == BF16 else 5e-7)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,I,O", MM)
def test_input_gradient(M, I, O, dt, fmt):
    for k, act in enumerate(ACTS):
        pad, lead = ((0, 0), (7, 3))[k % 2]
        dy, wt = randn(M, O, seed=40, dt=dt), randn(I, O, seed=41, std=O ** -0.5)
        pre = None if act == "none" else sliced(M, I, pad, 42, dt, lead)
        pd, pw = ops.pack_f8(dy, fmt), ops.pack_f8(wt)
        dx = ops.f8_linear_bwd_input(pd, pw, pre=pre, act=act, dtype=dt)
        D, W = value(pd), value(pw)
        g, mag = D @ W.t(), D.abs() @ W.abs().t()
        e = (O + 8) * E * mag + (lost(D, W) if dt == BF16 else 0)
        H = torch.zeros_like(g) if pre is None else pre.double()
        want = g * gate(H, act)[1]
        near(dx, want, 1.2 * e + 4e-6 * (1 + H.abs()) * (g.abs() + e) * (act not in ("none", "relu")) + u(dt) * (want.abs() + 1.2 * e), act)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,I,O", MM + [(20000, 96, 130), (9001, 33, 17)])
def test_weight_gradient(M, I, O, dt, fmt):
    dy, x = randn(M, O, seed=50, dt=dt), randn(M, I, seed=51, dt=dt)
    dyt, db = ops.pack_f8(dy, fmt, along="rows", sums=True)
    xt = ops.pack_f8(x, along="rows")
    dw = ops.f8_linear_bwd_weight(dyt, xt, dtype=dt)
    D, X = value(dyt), value(xt)
    want, mag = D @ X.t(), D.abs() @ X.abs().t()
    e = (M + 16) * E * mag + (lost(D, X) if dt == BF16 else 0)
    near(dw, want, e + u(dt) * (want.abs() + e), "dw")
    total = dy.double().sum(0)
    es = (min(M, 128 + M // 128) + 16) * E * dy.double().abs().sum(0)
    near(db, total, es + u(dt) * (total.abs() + es), "db")


@pytest.mark.parametrize("dt", DTYPES)
def test_products_keep_non_finite_values_to_their_rows(dt):
    for M, I, O in ((65, 33, 129), (300, 300, 200)):
        x, w = randn(M, I, seed=60), randn(O, I, seed=61)
        bad = torch.zeros(M, dtype=torch.bool, device=DEV)
        bad[[0, M // 2, M - 1]] = True
        xb = x.clone()
        xb[0, 0], xb[M // 2, I - 1], xb[M - 1, 0] = math.nan, math.inf, -math.inf
        y, clean = (ops.f8_linear_fwd(ops.pack_f8(t), ops.pack_f8(w), dtype=dt) for t in (xb, x))
        assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[~bad])


def test_rows_behind_the_last_are_left_alone():
    x, w = ops.pack_f8(randn(70, 130, seed=62)), ops.pack_f8(randn(50, 130, seed=63))
    for dt in DTYPES:
        wide = torch.full((90, 80), 3.0, device=DEV, dtype=dt)
        ops.f8_linear_fwd(x, w, dtype=dt, out=wide[:70, 5:55])
        assert bool((wide[70:] == 3).all()) and bool((wide[:, :5] == 3).all()) and bool((wide[:, 55:] == 3).all())
        assert torch.equal(wide[:70, 5:55], ops.f8_linear_fwd(x, w, dtype=dt))


def test_no_rows_and_refusals():
    x, w = randn(6, 40, seed=64), randn(9, 40, seed=65)
    px, pw, p5 = ops.pack_f8(x), ops.pack_f8(w), ops.pack_f8(w, "e5m2")
    none = ops.pack_f8(x[:0])
    assert none.rows == 0 and ops.f8_linear_fwd(none, pw).shape == (0, 9)
    wrong = ops.pack_f8(randn(9, 41, seed=66))
    for bad in (lambda: ops.pack_f8(x, "e3m4"), lambda: ops.pack_f8(x, along="columns"), lambda: ops.pack_f8(x, sums=True),
                lambda: ops.pack_f8(x[:0], along="rows"), lambda: ops.pack_f8(x.half()), lambda: ops.f8_linear_fwd(px, wrong),
                lambda: ops.f8_linear_fwd(px, p5), lambda: ops.f8_linear_fwd(px, w), lambda: ops.f8_linear_fwd(px, pw, act="tanh"),
                lambda: ops.f8_linear_fwd(px, pw, dtype=torch.float16), lambda: ops.f8_linear_fwd(px, pw, save="pack8"),
                lambda: ops.f8_linear_fwd(px, pw, randn(9, seed=1)), lambda: ops.f8_linear_fwd(px, pw, out=randn(6, 9, seed=1)),
                lambda: ops.f8_linear_bwd_input(px, pw, act="relu"), lambda: ops.f8_linear_bwd_input(px, pw, pre=randn(6, 9, seed=1)),
                lambda: ops.f8_linear_bwd_weight(px, wrong), lambda: ops.F8(px.q, px.e[:, :8], 40),
                lambda: ops.F8(px.q.view(torch.uint8), px.e, 40), lambda: ops.F8(px.q, px.e, 200), lambda: ops.F8(px.q.cpu(), px.e.cpu(), 40)):
        with pytest.raises((ValueError, TypeError)):
            bad()


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("dt", DTYPES)
def test_autograd(act, dt):
    """The function's results against the operators called one by one, and near the products without rounding to 8 bits."""
    x = randn(3, 50, 70, seed=70, dt=dt).requires_grad_(True)
    w, b = randn(45, 70, seed=71, dt=dt, std=0.1).requires_grad_(True), randn(45, seed=72, dt=dt).requires_grad_(True)
    r = randn(150, 45, seed=73, dt=dt).requires_grad_(True)
    dy = randn(3, 50, 45, seed=74, dt=dt)
    y = ops.F8LinearFunction.apply(x, w, b, act, r)
    gx, gw, gb, gr = torch.autograd.grad(y, (x, w, b, r), dy.transpose(1, 2).contiguous().transpose(1, 2))
    X, flat = x.detach().reshape(-1, 70), dy.reshape(-1, 45)
    want, pre = ops.f8_linear_fwd(ops.pack_f8(X), ops.pack_f8(w.detach()), b.detach(), act, r.detach(), "pre", dt)
    assert torch.equal(y.detach().reshape(-1, 45), want)
    dh = flat if act == "none" else ops.act_bwd(pre, flat, act)
    dyt, db = ops.pack_f8(dh, "e5m2", along="rows", sums=True)
    assert torch.equal(gx.reshape(-1, 70), ops.f8_linear_bwd_input(ops.pack_f8(dh, "e5m2"), ops.pack_f8(w.detach().t().contiguous()), dtype=dt))
    assert torch.equal(gw, ops.f8_linear_bwd_weight(dyt, ops.pack_f8(X, along="rows"), dtype=dt)) and torch.equal(gb, db)
    assert torch.equal(gr, flat)
    # an operand's rounding is at most 2^-4 (e4m3) or 2^-3 (e5m2) of its value: the products' norms are within their sum
    h = X.double() @ w.detach().double().t() + b.detach().double()
    D = flat.double() * gate(h, act)[1]
    assert float((gx.reshape(-1, 70).double() - D @ w.detach().double()).norm() / (D @ w.detach().double()).norm()) < 0.25
    assert float((gw.double() - D.t() @ X.double()).norm() / (D.t() @ X.double()).norm()) < 0.25
    y = ops.F8LinearFunction.apply(x, w.detach())
    y.sum().backward()
    assert x.grad.shape == x.shape and w.grad is None
    y = ops.F8LinearFunction.apply(x.detach()[:0], w, b)
    y.sum().backward()
    assert not w.grad.any() and not b.grad.any()
