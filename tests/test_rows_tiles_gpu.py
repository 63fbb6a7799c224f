"""The row operators' kernels that only certain sizes take (rows_cases.py), against their formulas in 64 bits.  Bounds as in
test_rows_gpu.py."""
import pytest
import torch

import rows_cases as cases
from paper_2309_15812_amd import ops
from test_rows_gpu import BF16, EPS, F32, gate, held_of, near, randn, sliced, u, value64

pytestmark = pytest.mark.gpu


def matrix(M, C, whole, seed, dt):
    return randn(M, C, seed=seed, dt=dt) if whole else sliced(M, C, 3, seed, dt, 1)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("M,C", cases.LAYER_NORM)
def test_layer_norm(M, C, dt):
    x, dy = randn(M, C, seed=1, dt=dt), randn(M, C, seed=2, dt=dt)
    w, b = randn(C, seed=3, dt=dt), randn(C, seed=4, dt=dt)
    y, mean, rstd = ops.ln_fwd(x, w, b, eps=EPS)
    X, W = x.double(), w.double()
    mu, rs = X.mean(1, keepdim=True), (X.var(1, keepdim=True, unbiased=False) + EPS).rsqrt()
    eps = 2.0 ** -24
    em = (C + 8) * eps * X.abs().mean(1, keepdim=True)
    ers = rs * ((C + 16) * eps + em * em * rs * rs)
    xh = (X - mu) * rs
    near(mean, mu[:, 0], em[:, 0], "mean")
    near(rstd, rs[:, 0], (ers + 2 * eps * rs)[:, 0], "rstd")
    want = xh * W + b.double()
    near(y, want, W.abs() * (xh.abs() * ers / rs + em * rs + 8 * eps * (xh.abs() + X.abs() * rs)) + u(dt) * want.abs()
         + 4 * eps * b.double().abs(), "y")
    for src in (x, held_of(x)):
        V = X if src is x else value64(src)
        G, m, r = dy.double(), mean.double()[:, None], rstd.double()[:, None]
        xh, g = (V - m) * r, G * W
        mgx = (g * xh).abs().mean(1, keepdim=True)
        n, exh = (C + 16) * eps, 4 * eps * (V.abs() + m.abs()) * r
        dx, dw, db = ops.ln_bwd(src, dy, mean, rstd, w)
        want = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        near(dx, want, r * (8 * eps * g.abs() + n * g.abs().mean(1, keepdim=True)
                            + xh.abs() * (n * mgx + (g.abs() * exh).mean(1, keepdim=True)) + exh * mgx) + u(dt) * want.abs(), "dx")
        nm = (M + 16) * eps
        near(dw, (G * xh).sum(0), nm * (G * xh).abs().sum(0) + (G.abs() * exh).sum(0) + u(dt) * (G * xh).sum(0).abs(), "dw")
        near(db, G.sum(0), nm * G.abs().sum(0) + u(dt) * G.sum(0).abs(), "db")


@pytest.mark.parametrize("M,I,O,dt,whole", cases.FORWARD)
def test_forward(M, I, O, dt, whole):
    x, res = matrix(M, I, whole, 5, dt), matrix(M, O, whole, 6, dt)
    w, b = randn(O, I, seed=7, dt=dt, std=I ** -0.5), randn(O, seed=8, dt=dt)
    X, W, B = x.double(), w.double(), b.double()
    h, mag = X @ W.t() + B, X.abs() @ W.abs().t() + B.abs()
    eh = (I + 8) * 2.0 ** -24 * mag
    y, pre = ops.linear_fwd(x, w, b, act="gelu", residual=res, save="pre")
    near(pre, h, eh + u(dt) * h.abs(), "pre")
    want = gate(h, "gelu")[0] + res.double()
    ey = 1.2 * eh + 2e-6 * (1 + h.abs())
    near(y, want, ey + u(dt) * (want.abs() + ey) + 2.0 ** -23 * h.abs(), "y")
    y, held = ops.linear_fwd(x, w, b, act="gelu", residual=res, save="pack8")
    near(y, want, ey + u(dt) * (want.abs() + ey) + 2.0 ** -23 * h.abs(), "y of a checkpointed call")
    near(value64(held), h, eh + (0.5 + 1e-4) * held.scale.double().repeat_interleave(64, 1)[:, :O], "checkpoint")
    assert not held.q[:, O:].any()


@pytest.mark.parametrize("M,I,O,dt,whole", cases.INPUT_GRADIENT)
def test_input_gradient(M, I, O, dt, whole):
    dy, pre, w = matrix(M, O, whole, 9, dt), matrix(M, I, whole, 10, dt), randn(O, I, seed=11, dt=dt, std=O ** -0.5)
    g, mag = dy.double() @ w.double(), dy.double().abs() @ w.double().abs()
    e = (O + 8) * 2.0 ** -24 * mag
    for src, act in ((None, "none"), (pre, "silu"), (held_of(pre), "gelu")):
        H = value64(src) if act == "gelu" else pre.double()
        want = g * gate(H, act)[1]
        near(ops.linear_bwd_input(dy, w, pre=src, act=act), want,
             1.2 * e + (act != "none") * 4e-6 * (1 + H.abs()) * (g.abs() + e) + u(dt) * (want.abs() + 1.2 * e), act)


@pytest.mark.parametrize("M,I,O,dt,whole", cases.WEIGHT_GRADIENT)
def test_weight_gradient(M, I, O, dt, whole):
    dy, x = matrix(M, O, whole, 12, dt), matrix(M, I, whole, 13, dt)
    D = dy.double()
    edb = (M + 16) * 2.0 ** -24 * D.abs().sum(0)
    for src, act in ((x, "none"), (held_of(x), "gelu")):
        V = x.double() if src is x else value64(src)
        a = gate(V, act)[0]
        want, mag = D.t() @ a, D.abs().t() @ a.abs()
        e = (M + 16) * 2.0 ** -24 * mag + (act != "none") * (u(dt) * mag + 2e-6 * (D.abs().t() @ (1 + V.abs())))
        dw, db = ops.linear_bwd_weight(src, dy, act=act)
        near(dw, want, e + u(dt) * (want.abs() + e), act)
        near(db, D.sum(0), edb + u(dt) * (D.sum(0).abs() + edb), "db")
