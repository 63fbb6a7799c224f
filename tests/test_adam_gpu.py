"""The AdamW step over many tensors against its formulas in 64 bits, step by step from the states that it left.

Tolerances are bounds.  Every operation is rounded once, 2^-24: m and v are within 4 and the update within 16 of those of
the terms' sizes.  A value in 8 bits (e4m3) is within 2^-4 of itself, or 2^-10 of its group's unit (the scale) where it
is smaller than 2^-6 units; a positive root is raised to at least 2^-9 units.
"""
import math

import pytest
import torch

from paper_2309_15812_amd import ops
from test_rows_gpu import BF16, DEV, F32, near, u
from test_rows_gpu import randn as normal

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
SHAPES = [(33, 7), (33,), (132, 33), (1,), (), (5, 0), (127,), (128,), (129,), (70, 100), (2049,), (3, 5, 7)]


def randn(*shape, seed, dt=F32):
    return normal(math.prod(shape), seed=seed, dt=dt).view(shape)


def values(state):
    """(m, v) in 64 bits."""
    if state.ms is None:
        return state.m.double(), state.v.double()
    m, r = (t.double().view(-1, 128) * s.double()[:, None] for t, s in ((state.m, state.ms), (state.v, state.vs)))
    return m.view(-1), r.view(-1) ** 2


def make(shapes, dt, gdt, bits, master, seed=1, flat=False):
    if flat:  # one behind the other, whatever their alignment
        n = [math.prod(s) for s in shapes]
        p, g = randn(sum(n), seed=seed, dt=dt), randn(sum(n), seed=seed + 1, dt=gdt)
        ps, gs = ([t.view(s) for t, s in zip(f.split(n), shapes)] for f in (p, g))
    else:
        ps = [randn(*s, seed=seed + i, dt=dt) for i, s in enumerate(shapes)]
        gs = [randn(*s, seed=seed + 50 + i, dt=gdt) * 10.0 ** (i % 5 - 3) for i, s in enumerate(shapes)]
    return ps, gs, ops.AdamState.zeros(ps, bits=bits, master=master)


def check_step(ps, gs, state, lr=1e-2, betas=(0.9, 0.99), eps=1e-8, wd=0.1, max_norm=None, **kw):
    m0, v0 = (t.clone() for t in values(state))
    p0 = [p.double().clone() for p in ps]
    master0 = None if state.master is None else state.master.double().clone()
    t = int(state.step[0]) + 1
    norm = ops.adamw(ps, gs, state, lr=kw.pop("lr_given", lr), betas=betas, eps=eps, weight_decay=wd, max_norm=max_norm)
    assert state.step.tolist() == [t, 0]
    factor, fe = 1.0, 0.0
    if max_norm is not None:
        want = math.sqrt(sum(float(g.double().square().sum()) for g in gs if g is not None))
        assert abs(float(norm) - want) <= 4 * E * want
        factor, fe = min(1.0, max_norm / want) if want else 1.0, 8 * E
    m1, v1 = values(state)
    c1, c2 = 1 / (1 - betas[0] ** t), 1 / math.sqrt(1 - betas[1] ** t)
    inside = torch.zeros(m0.numel(), dtype=torch.bool, device=DEV)
    for i, (p, g, n, at) in enumerate(zip(ps, gs, state.sizes, state.starts)):
        at_ = slice(at, at + n)
        inside[at_] = True
        if g is None:
            assert torch.equal(p.double(), p0[i]) and torch.equal(m1[at_], m0[at_]) and torch.equal(v1[at_], v0[at_])
            continue
        G = g.double().reshape(-1) * factor
        m, v = betas[0] * m0[at_] + (1 - betas[0]) * G, betas[1] * v0[at_] + (1 - betas[1]) * G * G
        em = (4 * E + fe) * (betas[0] * m0[at_].abs() + G.abs())
        ev = (6 * E + 2 * fe) * v
        w = p0[i].reshape(-1) if master0 is None else master0[at_]
        den = v.sqrt() * c2 + eps
        want = w * (1 - lr * wd) - lr * (m * c1) / den
        ew = 4 * E * w.abs() + lr * ((em * c1 + 16 * E * m.abs() * c1) / den + (m.abs() * c1) / den * (ev / v.clamp(min=1e-300)))
        if state.master is not None:
            near(state.master[at_], want, ew, f"master {i}")
        dt = p.dtype
        near(p.reshape(-1), want, ew + (u(dt) * (want.abs() + ew) if dt == BF16 else 0), f"parameter {i}")
        if state.ms is None:
            near(m1[at_].float(), m, em, "m")
            near(v1[at_].float(), v, ev, "v")
        else:
            for got, want8, e, least in ((m1[at_], m, em, False), (v1[at_].sqrt(), v.sqrt(), ev / v.sqrt().clamp(min=1e-300), True)):
                groups = torch.nn.functional.pad(want8.abs(), (0, -n % 128)).view(-1, 128)
                unit = (groups.amax(1) / 448).repeat_interleave(128)[:n]
                size = torch.maximum(want8.abs() * 2.0 ** -4, unit * 2.0 ** -10)
                if least:
                    size = torch.maximum(size, torch.where(want8 < unit * 2.0 ** -9, unit * 2.0 ** -9, 0 * unit))
                    assert bool((got[want8 > 0] > 0).all())
                tol = size * (1 + 1e-5) + 2 * e + 4 * E * want8.abs()
                assert bool(((got - want8).abs() <= tol).all()), float(((got - want8).abs() - tol).max())
    for t_ in (m1, v1, state.master):
        assert t_ is None or not t_[~inside].any()
    return norm


@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dt,gdt,master", [(F32, F32, False), (BF16, BF16, True), (BF16, BF16, False), (BF16, F32, True), (F32, BF16, True)])
def test_steps(dt, gdt, master, bits, flat):
    ps, gs, state = make(SHAPES, dt, gdt, bits, master, flat=flat)
    for k in range(3):
        check_step(ps, gs, state, max_norm=(None, 0.5, 1e6)[k])
        for i, g in enumerate(gs):
            g.copy_(randn(*g.shape, seed=200 + 20 * k + i, dt=gdt))


def test_more_tensors_than_a_launch_takes():
    for count in (96, 97, 250):
        ps, gs, state = make([(1 + 37 * (i % 60),) for i in range(count)], F32, F32, 8, False)
        gs[5] = gs[count - 1] = None
        check_step(ps, gs, state, max_norm=1.0)
        check_step(ps, gs, state, lr=1e-2, lr_given=torch.tensor(1e-2, device=DEV))


def test_large_tensor_in_both_states():
    for bits in (32, 8):
        ps, gs, state = make([(2100, 4099)], F32, F32, bits, False)
        check_step(ps, gs, state, max_norm=1.0)


def test_a_norm_that_is_not_finite_changes_nothing():
    for bits in (32, 8):
        for bad in (math.nan, math.inf, -math.inf):
            ps, gs, state = make(SHAPES, BF16, F32, bits, True)
            check_step(ps, gs, state)
            before = [t.clone().view(torch.uint8) for t in (*ps[:4], state.m, state.v, state.master, state.step)]
            gs[2][3, 4] = bad
            norm = ops.adamw(ps, gs, state, max_norm=1.0)
            assert not math.isfinite(float(norm))
            after = [t.view(torch.uint8) for t in (*ps[:4], state.m, state.v, state.master, state.step)]
            assert all(torch.equal(a, b) for a, b in zip(before, after))
            gs[2][3, 4] = 1e25  # its square leaves float32, the norm does not
            check_step(ps, gs, state, max_norm=1.0)


def test_states_of_the_smallest_gradients():
    # e4m3's steps of a scale of 2^-126: 2^-4 of a value, or 2^-10 of the scale; a root is at least 2^-9 of it
    sizes = (1e-30, 1e-36, 1e-37, 1e-38, 1e-40)
    ps, gs, state = make([(256,)] * len(sizes), F32, F32, 8, False)
    for g, size in zip(gs, sizes):
        g.copy_(torch.linspace(-1, 1, 256, device=DEV) * size)
        g[::3] = 0
    before = [p.clone() for p in ps]
    ops.adamw(ps, gs, state, lr=1e-2, weight_decay=0.0)
    m = state.m.float().double() * state.ms.double().repeat_interleave(128)
    r = state.v.float().double() * state.vs.double().repeat_interleave(128)
    for i, g in enumerate(gs):
        at_ = slice(256 * i, 256 * i + 256)
        want = 0.1 * g.double()
        unit = state.ms[2 * i:2 * i + 2].double().repeat_interleave(128)
        assert bool(((m[at_] - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, unit * 2.0 ** -10) * (1 + 1e-5) + 2.0 ** -148).all())
        assert bool((state.ms[2 * i:2 * i + 2] >= 2.0 ** -126).all()) and not r[at_].any()  # (squares below 1e-60)
        assert bool((ps[i] - before[i]).abs().max() <= 2.0 ** -20)  # eps is far above them


def test_tensors_may_share_a_gradient():
    for bits in (32, 8):
        ps, gs, state = make([(300,), (300,)], F32, F32, bits, False)
        check_step(ps, [gs[0], gs[0]], state, max_norm=1.0)


def test_an_update_counts_where_a_small_one_would_be_lost():
    # bfloat16 parameters with their float32 values: steps below bfloat16's spacing add up
    ps, gs, state = make([(256,)], BF16, BF16, 8, True)
    ps[0].fill_(1.0)
    state.master.fill_(1.0)
    gs[0].fill_(0.5)
    for _ in range(20):
        ops.adamw(ps, gs, state, lr=1e-3, weight_decay=0.0)
    assert bool(((state.master - 0.98).abs() < 1e-4).all()) and bool((ps[0].float() - 0.98).abs().max() <= 2.0 ** -8)


def test_captured_steps_count_on_every_replay():
    ps, gs, state = make(SHAPES, F32, F32, 8, False)
    other, _, twin = make(SHAPES, F32, F32, 8, False)
    lr = torch.tensor(1e-2, device=DEV)
    ws = torch.empty(int(ops._lib.lib().o1d_adamw_workspace_bytes(1.0)), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ops.adamw(ps, gs, state, lr=lr, max_norm=1.0, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    ops.adamw(other, gs, twin, lr=1e-2, max_norm=1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.adamw(ps, gs, state, lr=lr, max_norm=1.0, workspace=ws)
    for k in range(4):
        rate = 1e-2 / (1 + k)
        lr.fill_(rate)
        for i, g in enumerate(gs):
            g.copy_(randn(*g.shape, seed=300 + 20 * k + i))
        graph.replay()
        ops.adamw(other, gs, twin, lr=torch.tensor(rate, device=DEV), max_norm=1.0)
        torch.cuda.synchronize()
        assert state.step.tolist() == twin.step.tolist() == [k + 2, 0]
        for a, b in zip((*ps, state.m.view(torch.uint8), state.vs), (*other, twin.m.view(torch.uint8), twin.vs)):
            assert torch.equal(a, b)


def test_refusals():
    ps, gs, state = make([(40,), (30,)], F32, F32, 8, False)
    for bad in (lambda: ops.adamw(ps[:1], gs, state), lambda: ops.adamw(ps, gs[:1], state), lambda: ops.adamw([ps[0], ps[0][:30]], gs, state),
                lambda: ops.adamw(ps, [gs[0], gs[1].bfloat16()], state), lambda: ops.adamw([ps[0].cpu(), ps[1]], gs, state),
                lambda: ops.adamw(ps, [gs[0], ps[1]], state), lambda: ops.adamw(ps, [gs[0], gs[1][:29]], state),
                lambda: ops.adamw(ps, gs, state, lr=-1.0), lambda: ops.adamw(ps, gs, state, betas=(1.0, 0.9)),
                lambda: ops.adamw(ps, gs, state, eps=-1.0), lambda: ops.adamw(ps, gs, state, lr=torch.tensor(1.0)),
                lambda: ops.adamw(ps, gs, state, max_norm=0.0), lambda: ops.adamw(ps, gs, state, weight_decay=math.nan),
                lambda: ops.adamw([p.half() for p in ps], gs, state), lambda: ops.AdamState.zeros([], bits=8),
                lambda: ops.AdamState.zeros(ps, bits=16), lambda: ops.AdamState([40, 30], state.m, state.v, state.step),
                lambda: ops.AdamState([40, 200], state.m, state.v, state.step, state.ms, state.vs)):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            bad()
    assert state.step.tolist() == [0, 0] and not state.ms.any()
