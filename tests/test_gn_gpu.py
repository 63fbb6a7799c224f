"""Group norm with an activation against its formulas in 64 bits.

Tolerances are bounds, element by element.  u = 2^-24 for float32 and 2^-8 for bfloat16 results, one rounding.  A sum's
error is at most its longest chain of additions times 2^-24 sum |terms|: a thread adds its rows, at most 256 of these
sizes, then at most eight threads' sums, a lane's share of the group's channels and the wave's: below 300 (or the number of
terms, where that is less); over samples and pixels twice that.  An activation adds at most its slope (below 1.2; below 2 for
its derivative's) times its argument's error and 2e-6 (1 + |h|) for its own evaluation.
"""
import math

import pytest
import torch

from paper_2309_15812_amd import ops
from test_rows_gpu import ACTS, BF16, DEV, DTYPES, F32, gate, near, randn, u

pytestmark = pytest.mark.gpu
EPS = 1e-5
E = 2.0 ** -24

# (samples, pixels, channels, groups): a value a group, few channels, odd ones, whole rows in a group, samples that a
# workgroup holds and samples in pieces
SIZES = [(1, 1, 1, 1), (2, 3, 5, 5), (1, 16, 7, 1), (3, 49, 96, 32), (1, 49, 768, 32), (2, 784, 192, 32), (5, 33, 203, 7),
         (64, 49, 24, 3), (3, 1000, 6, 2), (1, 50, 2, 1), (2, 9, 1030, 1030), (2, 20, 1024, 1), (300, 4, 64, 2),
         (1, 3136, 96, 32), (1, 12707, 203, 7), (1, 30000, 64, 8), (4, 5000, 33, 33), (1, 20000, 3, 1), (2, 700, 1100, 11)]


def sliced(N, P, C, pad, seed, dt, lead=0):
    return randn(N, P, C + pad, seed=seed, dt=dt)[..., lead:lead + C]


def parts(t, G):  # (N, G, P D) of (N, P, C)
    N, P, C = t.shape
    return t.view(N, P, G, C // G).permute(0, 2, 1, 3).reshape(N, G, -1)


def whole(t, P):  # and back
    N, G, n = t.shape
    return t.view(N, G, P, n // P).permute(0, 2, 1, 3).reshape(N, P, -1)


def per_channel(t, N, P, C, G):  # a vector of the channels as (N, G, P D)
    return parts(t.double().expand(N, P, C), G)


def run_forward(N, P, C, G, dt, act, pad, lead, shift=0.0):
    x = sliced(N, P, C, pad, 1, dt, lead)
    if shift:
        x = x + shift
    w, b = randn(C, seed=2, dt=dt), randn(C, seed=3, dt=dt)
    y, mean, rstd = ops.gn_fwd(x, w, b, G, eps=EPS, act=act)
    X = parts(x.double(), G)
    n = X.shape[2]
    chain = min(n, 300) + 8
    mu, var = X.mean(2), X.var(2, unbiased=False)
    rs = (var + EPS).rsqrt()
    em = chain * E * X.abs().mean(2) + E * mu.abs()
    near(mean, mu, em, "mean")
    ers = rs * ((chain + 8) * E + em * em * rs * rs)
    near(rstd, rs, ers + 2 * E * rs, "rstd")
    xh = (X - mu[..., None]) * rs[..., None]
    W, B = per_channel(w, N, P, C, G), per_channel(b, N, P, C, G)
    h = xh * W + B
    eh = W.abs() * (xh.abs() * (ers / rs)[..., None] + (em * rs)[..., None] + 8 * E * (xh.abs() + X.abs() * rs[..., None])) \
        + 4 * E * (B.abs() + h.abs())
    want = gate(h, act)[0]
    ey = 1.2 * eh + (0 if act in ("none", "relu") else 2e-6 * (1 + h.abs()))
    near(y, whole(want, P), whole(ey + u(dt) * (want.abs() + ey), P), act)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("N,P,C,G", SIZES)
def test_forward(N, P, C, G, dt):
    for k, act in enumerate(ACTS if N * P * C < 300000 else ["none", "silu"]):
        pad, lead = ((0, 0), (13, 3))[k % 2]
        run_forward(N, P, C, G, dt, act, pad, lead)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("N,P,C,G", [(3, 49, 96, 32), (1, 12707, 203, 7), (1, 3136, 96, 32)])
def test_a_mean_far_above_the_spread(N, P, C, G, dt):
    run_forward(N, P, C, G, dt, "silu", 0, 0, shift=40.0)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("N,P,C,G", SIZES)
def test_backward(N, P, C, G, dt):
    for k, act in enumerate(ACTS if N * P * C < 300000 else ["none", "silu"]):
        pad, lead = ((0, 0), (9, 1))[k % 2]
        x, dy = sliced(N, P, C, pad, 4, dt, lead), sliced(N, P, C, pad, 5, dt, lead)
        w, b = randn(C, seed=6, dt=dt), randn(C, seed=7, dt=dt)
        X, DY = parts(x.double(), G), parts(dy.double(), G)
        mean, rstd = X.mean(2).float(), (X.var(2, unbiased=False) + EPS).rsqrt().float()
        dx, dw, db = ops.gn_bwd(x, dy, mean, rstd, w, b, act=act)
        n = X.shape[2]
        chain = min(n, 300) + 8
        rs, mu = rstd.double()[..., None], mean.double()[..., None]
        W, B = per_channel(w, N, P, C, G), per_channel(b, N, P, C, G)
        xh = (X - mu) * rs
        h = xh * W + B
        slope = gate(h, act)[1]
        dh = DY * slope
        g = dh * W
        s, sx = g.mean(2, keepdim=True), (g * xh).mean(2, keepdim=True)
        want = rs * (g - s - xh * sx)
        exh = 4 * E * (X.abs() + mu.abs()) * rs
        eh = W.abs() * exh + 4 * E * (h.abs() + B.abs())
        if act == "relu":  # (next to 0 the slope is either)
            edh = torch.where(h.abs() <= eh, DY.abs(), 0 * DY)
        else:
            edh = DY.abs() * (2 * eh * (act != "none") + (act != "none") * 4e-6 * (1 + h.abs())) + 2 * E * dh.abs()
        eg = W.abs() * edh + 2 * E * g.abs()
        es = chain * E * g.abs().mean(2, keepdim=True) + eg.mean(2, keepdim=True)
        esx = chain * E * (g * xh).abs().mean(2, keepdim=True) + (eg * xh.abs() + g.abs() * exh).mean(2, keepdim=True)
        tol = rs * (eg + es + xh.abs() * esx + exh * sx.abs() + 8 * E * (g.abs() + s.abs() + (xh * sx).abs())) + u(dt) * want.abs()
        near(dx, whole(want, P), whole(tol * (1 + u(dt)), P), act)
        long = min(N * P, 600) + 8
        for got, terms, et, what in ((dw, dh * xh, edh * xh.abs() + dh.abs() * exh, "dw"), (db, dh, edh, "db")):
            flat, ef = whole(terms, P), whole(et, P)
            total = flat.sum((0, 1))
            e = long * E * flat.abs().sum((0, 1)) + ef.sum((0, 1))
            near(got, total, e + u(dt) * (total.abs() + e), what)


def test_non_finite_values_stay_in_their_group():
    for dt in DTYPES:
        for N, P, C, G in ((3, 40, 33, 11), (2, 20000, 24, 3)):
            D = C // G
            x, dy = randn(N, P, C, seed=8, dt=dt), randn(N, P, C, seed=9, dt=dt)
            w, b = randn(C, seed=10, dt=dt), randn(C, seed=11, dt=dt)
            clean = ops.gn_fwd(x, w, b, G, act="silu")
            cb = ops.gn_bwd(x, dy, clean[1], clean[2], w, b, act="silu")
            bad = x.clone()
            bad[1, P - 1, D] = math.inf  # the second group's first channel
            bad[0, 0, C - 1] = math.nan
            y, mean, rstd = ops.gn_fwd(bad, w, b, G, act="silu")
            hit = torch.zeros(N, G, dtype=torch.bool, device=DEV)
            hit[1, 1] = hit[0, G - 1] = True
            assert torch.isnan(rstd[hit]).all() and torch.equal(rstd[~hit], clean[2][~hit]) and torch.equal(mean[~hit], clean[1][~hit])
            wide = hit.repeat_interleave(D, 1)[:, None].expand(N, P, C)
            assert torch.isnan(y[wide]).all() and torch.equal(y[~wide], clean[0][~wide])
            dx, dw, db = ops.gn_bwd(bad, dy, mean, rstd, w, b, act="silu")
            assert torch.isnan(dx[wide]).all() and torch.equal(dx[~wide], cb[0][~wide])
            cols = hit.any(0).repeat_interleave(D)
            assert torch.isnan(dw[cols]).all() and torch.equal(dw[~cols], cb[1][~cols]) and torch.equal(db[~cols], cb[2][~cols])


def test_constant_groups_and_no_samples():
    x = torch.full((2, 30, 12), 7.25, device=DEV)
    w, b = randn(12, seed=1), randn(12, seed=2)
    y, mean, rstd = ops.gn_fwd(x, w, b, 3, eps=1e-6)
    assert torch.equal(mean, torch.full_like(mean, 7.25)) and torch.allclose(rstd, torch.full_like(rstd, 1e3), rtol=1e-6)
    assert torch.equal(y, b.expand(2, 30, 12))
    y, mean, rstd = ops.gn_fwd(x[:0], w, b, 3)
    assert y.shape == (0, 30, 12) and mean.shape == (0, 3)
    dx, dw, db = ops.gn_bwd(x[:0], x[:0], mean, rstd, w, b)
    assert dx.shape == (0, 30, 12) and not dw.any() and not db.any()


def test_gradients_against_differences():
    """The derivative of sum(y dy) along a direction in x, w and b against the change of the float64 formula."""
    N, P, C, G = 2, 60, 24, 4
    x, dy = randn(N, P, C, seed=20), randn(N, P, C, seed=21)
    w, b = randn(C, seed=22), randn(C, seed=23)
    for act in ("none", "gelu", "gelu_tanh", "silu"):
        xs = [t.clone().requires_grad_(True) for t in (x, w, b)]
        ops.GroupNormFunction.apply(*xs, G, EPS, act).backward(dy)

        def value(x, w, b):
            X = parts(x, G)
            xh = whole((X - X.mean(2, keepdim=True)) * (X.var(2, unbiased=False, keepdim=True) + EPS).rsqrt(), P)
            return float((gate(xh * w + b, act)[0] * dy.double()).sum())

        for k in range(3):
            at = [t.double() for t in (x, w, b)]
            d = torch.randn(at[k].shape, generator=torch.Generator(device=DEV).manual_seed(30 + k), device=DEV).double()
            step = 1e-4
            up, down = ([t + s * step * d if i == k else t for i, t in enumerate(at)] for s in (1, -1))
            want, got = (value(*up) - value(*down)) / (2 * step), float((xs[k].grad.double() * d).sum())
            # (third derivatives are of the order of the terms: step^2 = 1e-8; float32 gradients 1e-6 of their size)
            assert abs(got - want) <= 1e-5 * float((xs[k].grad.double() * d).abs().sum()) + 1e-5 * abs(want)


def test_given_outputs_and_images():
    x = randn(2, 5, 6, 16, seed=12)
    w, b = randn(16, seed=13), randn(16, seed=14)
    out = torch.empty_like(x)
    y, mean, rstd = ops.gn_fwd(x, w, b, 4, out=out)
    assert y is out and torch.equal(y, ops.gn_fwd(x.view(2, 30, 16), w, b, 4)[0].view_as(x))
    outs = (torch.empty_like(x), torch.empty_like(w), torch.empty_like(b))
    got = ops.gn_bwd(x, y, mean, rstd, w, b, act="relu", out=outs)
    assert all(a is b for a, b in zip(got, outs))
    for bad in (lambda: ops.gn_fwd(x, w, b, 5), lambda: ops.gn_fwd(x, w, b, 0), lambda: ops.gn_fwd(x, w[:8], b, 4),
                lambda: ops.gn_fwd(x, w, b, 4, act="tanh"), lambda: ops.gn_fwd(x.transpose(1, 3), w, b, 4),
                lambda: ops.gn_fwd(x[:, :0], w, b, 4), lambda: ops.gn_bwd(x, y, mean[:, :3].contiguous(), rstd, w, b),
                lambda: ops.gn_bwd(x, y, mean[:1], rstd[:1], w, b), lambda: ops.gn_bwd(x.double(), y, mean, rstd, w, b)):
        with pytest.raises((ValueError, TypeError)):
            bad()
    for groups in (4.0, "4", None):
        with pytest.raises(TypeError):
            ops.gn_fwd(x, w, b, groups)
