"""The residual block and the autograd functions of the row operators against float64 autograd of their formulas.

Angles 0 and 90 degrees, where the convolution is a horizontal correlation and a vertical one with the kernel reversed.
Errors are 2-norms relative to the reference's.  float32: sums of at most 600 terms behind one another, well below 1e-4.
bfloat16: each stored intermediate adds 2^-9 relative and a gradient passes fewer than ten of them, so at most 2e-2.
8-bit checkpoints: an element is off by amax / 254 at most, uniformly, 0.7% of a normal group's size, once per
checkpointed factor, so at most 3e-2 with bfloat16's own.
"""
import pytest
import torch
import torch.nn.functional as F

from paper_2309_15812_amd import ops
from paper_2309_15812_amd.block import OrientedBlock

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def off(got, want):
    want = want.detach()
    return float((got.detach().double().cpu() - want).norm() / want.norm())


def reference(block, x, dy):
    p = {n: t.detach().double().cpu().requires_grad_(True) for n, t in block.named_parameters()}
    x = x.detach().double().cpu().requires_grad_(True)
    C, K = p["w_dw"].shape
    flat = (block.theta == 0).cpu()
    nchw = x.permute(0, 3, 1, 2)
    rows = F.conv2d(nchw, p["w_dw"].view(C, 1, 1, K), padding=(0, K // 2), groups=C)
    cols = F.conv2d(nchw, p["w_dw"].flip(1).view(C, 1, K, 1), padding=(K // 2, 0), groups=C)
    u = torch.where(flat[:, None, None], rows, cols).permute(0, 2, 3, 1)
    v = F.layer_norm(u, (C,), p["ln_w"], p["ln_b"], block.eps)
    h = v @ p["w1"].t() + p["b1"]
    a = {"gelu": F.gelu, "relu": F.relu, "silu": F.silu, "none": lambda t: t}[block.act](h)
    y = x + a @ p["w2"].t() + p["b2"]
    y.backward(dy.double().cpu())
    return y.detach(), x.grad, {n: t.grad for n, t in p.items()}


@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("dtype,act", [(torch.float32, "gelu"), (torch.float32, "silu"), (torch.bfloat16, "gelu"),
                                       (torch.bfloat16, "none")])
@pytest.mark.parametrize("N,H,W,C,K", [(2, 9, 11, 24, 7), (1, 14, 14, 33, 5)])
def test_block_against_float64(N, H, W, C, K, dtype, act, checkpoint):
    torch.manual_seed(3)
    block = OrientedBlock(C, K, directions=2, act=act, checkpoint=checkpoint).to(DEV).to(dtype)
    with torch.no_grad():
        for t in (block.ln_b, block.b1, block.b2):
            t.normal_(std=0.3)
        block.ln_w.add_(0.2 * torch.randn_like(block.ln_w))
    x = torch.randn(N, H, W, C, device=DEV).to(dtype).requires_grad_(True)
    dy = torch.randn(N, H, W, C, device=DEV).to(dtype)
    y = block(x)
    y.backward(dy)
    want, dx, grads = reference(block, x, dy)
    tol = 3e-2 if checkpoint else 1e-4 if dtype == torch.float32 else 2e-2
    assert off(y, want) <= (1e-5 if dtype == torch.float32 else 2e-2)
    assert off(x.grad, dx) <= tol
    for n, t in block.named_parameters():
        assert off(t.grad, grads[n]) <= tol, n


# (relu from a checkpoint is tested against the checkpoint's own values with the row operators: a pre-activation that rounds
# to zero changes its slope from 1 to 0, which no bound on the rounding covers)
@pytest.mark.parametrize("act,checkpoint", [(a, c) for a in ("none", "relu", "gelu", "silu") for c in (False, True)
                                            if (a, c) != ("relu", True)])
def test_autograd_functions(act, checkpoint):
    torch.manual_seed(4)
    x, w, b, r = (torch.randn(*s, device=DEV).requires_grad_(True) for s in ((50, 37), (45, 37), (45,), (50, 45)))
    lw, lb = (torch.randn(37, device=DEV).requires_grad_(True) for _ in range(2))
    dy = torch.randn(50, 45, device=DEV)
    n = ops.LayerNormFunction.apply(x, lw, lb, 1e-6, checkpoint)
    y = ops.LinearFunction.apply(n, w, b, act, r, checkpoint)
    # an expanded gradient, as a sum gives, and a strided one
    got = torch.autograd.grad(y, (x, lw, lb, w, b, r), dy.t().contiguous().t())
    ref = [t.detach().double().cpu().requires_grad_(True) for t in (x, lw, lb, w, b, r)]
    h = F.layer_norm(ref[0], (37,), ref[1], ref[2], 1e-6) @ ref[3].t() + ref[4]
    a = {"gelu": F.gelu, "relu": F.relu, "silu": F.silu, "none": lambda t: t}[act](h)
    want = torch.autograd.grad(a + ref[5], ref, dy.double().cpu())
    for g, t in zip(got, want):
        assert off(g, t) <= (3e-2 if checkpoint else 1e-5)
    y = ops.LinearFunction.apply(ops.LayerNormFunction.apply(x, lw, lb, 1e-6, checkpoint), w, None, act, None, checkpoint)
    y.sum().backward()
    assert x.grad.shape == x.shape and torch.isfinite(x.grad).all() and b.grad is None


def test_the_example_trains_and_checkpoints_keep_less(capsys):
    from paper_2309_15812_amd import block

    block.main(steps=6)
    lines = [line.split() for line in capsys.readouterr().out.splitlines() if "loss" in line]
    for checkpoint in ("checkpoint=False", "checkpoint=True"):
        mine = [line for line in lines if line[0] == checkpoint]
        losses, kept = [float(line[4].rstrip(",")) for line in mine], [float(line[9]) for line in mine]
        assert losses[-1] < 0.9 * losses[0]
        if checkpoint == "checkpoint=True":
            assert kept[-1] < 0.45 * whole
        whole = kept[-1]
