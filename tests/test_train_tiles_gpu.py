"""Group norm's and the 8-bit products' kernels that only certain sizes take, against their formulas in 64 bits.  Bounds as in
test_gn_gpu.py and test_f8_gpu.py."""
import pytest
import torch

import test_f8_gpu as f8
import test_gn_gpu as gn
from paper_2309_15812_amd import ops
from test_rows_gpu import BF16, DEV, DTYPES, F32, near, randn, sliced, u

pytestmark = pytest.mark.gpu

# (samples, pixels, channels, groups): workgroups of 256, 512 and 1024 threads with 2, 4, 6, 8 and 10 runs in a thread, of either
# type and direction, aligned rows and odd ones
HELD = [(1, 196, 24, 3), (1, 1500, 6, 2), (1, 196, 64, 1), (1, 400, 203, 7), (1, 784, 33, 33), (64, 196, 203, 7), (1, 1500, 24, 3),
        (1, 400, 64, 1), (1, 784, 203, 7), (1, 400, 6, 2), (64, 30, 203, 7), (1, 400, 33, 33), (64, 49, 203, 7), (1, 784, 6, 2),
        (1, 196, 203, 7), (1, 1500, 192, 4), (64, 784, 203, 7), (1, 1500, 203, 7), (1, 1500, 33, 33), (1, 49, 1024, 1),
        (1, 784, 24, 3), (1, 784, 192, 4), (64, 400, 203, 7), (1, 14, 560, 1), (1, 21, 720, 1), (1, 3136, 6, 2), (1, 3136, 203, 7),
        (1, 1053, 58, 2), (1, 2161, 1, 1), (1, 1156, 5, 1)]


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("N,P,C,G", HELD)
def test_group_norm(N, P, C, G, dt):
    gn.run_forward(N, P, C, G, dt, "silu", 0 if C % 2 else 5, 0)
    gn.test_backward(N, P, C, G, dt)


# (rows, summed features, features): few tiles of 32 x 32 in each of their kernels, tiles of 64 x 64, 128 x 128 and, for
# bfloat16 results, 256 x 256, of 1, 2, 3 and more steps of 128, whole ones and ones that end inside
PRODUCTS = [(100, 1500, 40), (128, 1500, 128), (128, 2300, 128), (33, 2700, 65), (5, 5671, 568), (300, 16, 1000), (512, 16, 1024),
            (300, 300, 1000), (1001, 768, 777), (640, 700, 1024), (700, 16, 3000), (2048, 128, 2048), (1500, 300, 2000), (2048, 640, 2048), (3001, 100, 5003), (4096, 128, 4096), (4096, 384, 4096),
            (3001, 1500, 5003), (8192, 250, 2048)]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("M,K,N", PRODUCTS)
def test_products(M, K, N, dt, fmt):
    x = randn(M, K, seed=20) * torch.exp2(torch.arange(M, device=DEV) % 7 - 3.0)[:, None]
    w, b = randn(N, K, seed=21, std=K ** -0.5), randn(N, seed=22, dt=dt)
    lead = M % 2
    res = sliced(M, N, 9 * lead, 23, dt, lead)
    px, pw = ops.pack_f8(x, fmt), ops.pack_f8(w)
    y, pre = ops.f8_linear_fwd(px, pw, b, act="silu", residual=res, save="pre", dtype=dt)
    X, W = f8.value(px), f8.value(pw)
    g, mag = X @ W.t(), X.abs() @ W.abs().t()
    e = (K + 8) * f8.E * mag + (f8.lost(X, W) if dt == BF16 else 0)
    h = g + b.double()
    eh = e + 2 * f8.E * (mag + b.double().abs())
    near(pre, h, eh + u(dt) * (h.abs() + eh), "pre")
    want = f8.gate(h, "silu")[0] + res.double()
    ey = 1.2 * eh + 2e-6 * (1 + h.abs())
    near(y, want, ey + u(dt) * (want.abs() + ey) + 2 * f8.E * h.abs(), "y")
    del h, eh, ey
    dx = ops.f8_linear_bwd_input(px, pw, pre=res, act="silu", dtype=dt)
    H = res.double()
    want = g * f8.gate(H, "silu")[1]
    near(dx, want, 1.2 * e + 4e-6 * (1 + H.abs()) * (g.abs() + e) + u(dt) * (want.abs() + 1.2 * e), "dx")
    near(ops.f8_linear_bwd_input(px, pw, dtype=dt), g, e + u(dt) * (g.abs() + e), "dx of none")


# (rows, summed, features): the tiles, in one piece and in several
@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("O,M,I", [(3001, 100, 5003), (2048, 128, 2048), (700, 4100, 1500), (129, 20000, 512), (512, 9000, 1024), (128, 1500, 128),
                                   (1344, 292, 181), (331, 18238, 458), (300, 16, 1000), (512, 16, 1024), (1, 9000, 16), (128, 2300, 128),
                                   (128, 2300, 256), (130, 1500, 70), (400, 2200, 500), (1, 2300, 1)])
def test_weight_gradients(O, M, I, dt):
    dyt, xt = ops.pack_f8(randn(O, M, seed=50), "e5m2"), ops.pack_f8(randn(I, M, seed=51))
    D, X = f8.value(dyt), f8.value(xt)
    want, mag = D @ X.t(), D.abs() @ X.abs().t()
    e = (M + 16) * f8.E * mag + (f8.lost(D, X) if dt == BF16 else 0)
    dw = ops.f8_linear_bwd_weight(dyt, xt, dtype=dt)
    near(dw, want, e + u(dt) * (want.abs() + e), "dw")
    for _ in range(2):
        assert torch.equal(ops.f8_linear_bwd_weight(dyt, xt, dtype=dt), dw)


def test_captured_operators_replay_alike():
    # each in a graph of its own on workspaces that both graphs share, replayed in turn with eager work between them
    cases = []
    for N, P, C, G in ((2, 30, 24, 3), (1, 3136, 96, 32)):
        x, dy = randn(N, P, C, seed=1, dt=BF16), randn(N, P, C, seed=2, dt=BF16)
        w, b = randn(C, seed=3, dt=BF16), randn(C, seed=4, dt=BF16)

        def norm(x=x, dy=dy, w=w, b=b, G=G, C=C, N=N, P=P):
            ws = shared[:max(512, int(ops._lib.lib().o1d_gn_fwd_workspace_bytes(N, P, C, G, 1)))]
            y, mean, rstd = ops.gn_fwd(x, w, b, G, act="gelu", workspace=ws)
            return (y, mean, rstd, *ops.gn_bwd(x, dy, mean, rstd, w, b, "gelu", workspace=shared))

        cases.append((norm, (x, dy)))
    for M, I, O in ((9001, 33, 17), (1344, 181, 292)):
        x, dy = randn(M, I, seed=5, dt=BF16), randn(M, O, seed=6, dt=BF16)

        def weights(x=x, dy=dy):
            dyt, db = ops.pack_f8(dy, "e5m2", along="rows", sums=True, workspace=shared)
            return ops.f8_linear_bwd_weight(dyt, ops.pack_f8(x, along="rows"), workspace=shared), db

        cases.append((weights, (x, dy)))
    shared = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    graphs = []
    for run, _ in cases:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out))
    for k in range(3):
        for (run, ins), (graph, out) in zip(cases, graphs):
            for i, t in enumerate(ins):
                t.copy_(randn(*t.shape, seed=100 + 10 * k + i, dt=BF16))
            graph.replay()
        for (run, _), (_, out) in zip(cases, graphs):
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, run()))


def test_a_stream_that_is_not_the_current_one():
    x, w = randn(500, 300, seed=1, dt=BF16), randn(200, 300, seed=2, dt=BF16)
    img, v = randn(2, 90, 48, seed=3, dt=BF16), randn(48, seed=4, dt=BF16)
    want = ops.f8_linear_fwd(ops.pack_f8(x), ops.pack_f8(w)), ops.gn_fwd(img, v, v, 4)[0]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.randn(1 << 24, device=DEV).square_()
        a, b = x.clone(), img.clone()
        got = ops.f8_linear_fwd(ops.pack_f8(a), ops.pack_f8(w)), ops.gn_fwd(b, v, v, 4)[0]
    side.synchronize()
    assert all(torch.equal(g, t) for g, t in zip(got, want))
