"""Group norm at the largest numbers of samples and pixels, against its formulas in 64 bits.  Bounds as in test_gn_gpu.py, but a
gradient's sum over the samples adds a 32nd of them one after the other, then 32."""
import pytest
import torch

import test_gn_gpu as gn
from paper_2309_15812_amd import ops
from test_gn_gpu import E, EPS, parts, per_channel, run_forward, whole
from test_rows_gpu import BF16, DEV, DTYPES, F32, near, randn, u

pytestmark = pytest.mark.gpu


def test_more_groups_than_a_grid_has_waves_forward():
    # 2^26 groups of all samples, in two passes
    run_forward(65536, 1, 7168, 1024, F32, "none", 0, 0)


def test_more_groups_than_a_grid_has_waves_backward():
    N, P, C, G = 65536, 1, 2048, 1024
    x, dy = randn(N, P, C, seed=4), randn(N, P, C, seed=5)
    w, b = randn(C, seed=6), randn(C, seed=7)
    X, DY = parts(x.double(), G), parts(dy.double(), G)
    mean, rstd = X.mean(2).float(), (X.var(2, unbiased=False) + EPS).rsqrt().float()
    dx, dw, db = ops.gn_bwd(x, dy, mean, rstd, w, b)
    chain, long = X.shape[2] + 8, N // 32 + 40
    rs, mu = rstd.double()[..., None], mean.double()[..., None]
    xh, exh = (X - mu) * rs, 4 * E * (X.abs() + mu.abs()) * rs
    g = DY * per_channel(w, N, P, C, G)
    s, sx = g.mean(2, keepdim=True), (g * xh).mean(2, keepdim=True)
    eg = 2 * E * g.abs()
    es = chain * E * g.abs().mean(2, keepdim=True) + eg.mean(2, keepdim=True)
    esx = chain * E * (g * xh).abs().mean(2, keepdim=True) + (eg * xh.abs() + g.abs() * exh).mean(2, keepdim=True)
    want = rs * (g - s - xh * sx)
    tol = rs * (eg + es + xh.abs() * esx + exh * sx.abs() + 8 * E * (g.abs() + s.abs() + (xh * sx).abs())) + u(F32) * want.abs()
    near(dx, whole(want, P), whole(tol * (1 + u(F32)), P), "dx")
    for got, terms, et, what in ((dw, DY * xh, DY.abs() * exh, "dw"), (db, DY, 0 * DY, "db")):
        total = whole(terms, P).sum((0, 1))
        e = long * E * whole(terms.abs(), P).sum((0, 1)) + whole(et, P).sum((0, 1))
        near(got, total, e + u(F32) * (total.abs() + e), what)


def test_the_longest_sample():
    # one channel of 2^31 - 1025 pixels: their sums in pieces, and results all over
    P = 0x7fffffff - 1024
    x = torch.empty(1, P, 1, device=DEV, dtype=BF16)
    part = 1 << 26
    gen = torch.Generator(device=DEV).manual_seed(1)
    for at in range(0, P, part):
        n = min(part, P - at)
        x[0, at:at + n, 0] = torch.randn(n, generator=gen, device=DEV) + at / P  # (the mean moves along the sample)
    w, b = randn(1, seed=2, dt=BF16), randn(1, seed=3, dt=BF16)
    y, mean, rstd = ops.gn_fwd(x, w, b, 1, eps=EPS)
    total = size = square = 0.0
    for at in range(0, P, part):
        v = x[0, at:at + part, 0].double()
        total, size = total + float(v.sum()), size + float(v.abs().sum())
    mu = total / P
    for at in range(0, P, part):
        square += float((x[0, at:at + part, 0].double() - mu).square().sum())
    rs = (square / P + EPS) ** -0.5
    # a thread adds 8 rows at a time and joins 2048 such means (three roundings each), then 256 threads, 512 chunks
    chain = 8 + 3 * 2048 + 256 / 64 + 64 + 8 + 16
    em = chain * E * size / P
    assert abs(float(mean) - mu) <= em
    assert abs(float(rstd) - rs) <= rs * ((chain + 8) * E + em * em * rs * rs)
    W, B = float(w), float(b)
    for at in (0, part, P // 2, P - part, P - 3):
        v = x[0, at:at + part, 0].double()
        h = (v - mu) * rs * W + B
        eh = abs(W) * rs * (em + (chain + 16) * E * ((v - mu).abs() + abs(mu) + v.abs())) + 4 * E * (h.abs() + abs(B))
        near(y[0, at:at + part, 0], h, eh + u(BF16) * (h.abs() + eh), f"pixels from {at}")


@pytest.mark.parametrize("dt", DTYPES)
def test_rows_wider_than_a_workgroup_in_pieces(dt):
    N, P, C, G = 1, 9529, 1224, 51
    for act, pad in (("none", 0), ("silu", 13)):
        run_forward(N, P, C, G, dt, act, pad, pad % 4)
    gn.test_backward(N, P, C, G, dt)
