"""A channels-last residual block around the oriented depthwise convolution, trained on the row operators.

    y = x + W2 act(W1 LN(conv(x)) + b1) + b2

The block the paper puts its convolution into: oriented depthwise 1D convolution, layer norm over the channels, a hidden
layer and the residual.  It runs in the library's kernels: the convolution's channels-last entry points, layer
norm, and the two products, whose epilogues add the biases, the activation and the residual; in the backward the activation's
derivative is applied in the epilogue of the second product's input gradient.  One pass is torch's: the sum of the
convolution's input gradient and the residual's, which in bfloat16 is rounded a second time there.

checkpoint=True keeps what the backward needs of the block's inside (the convolution's output, layer norm's output and the
hidden pre-activation) in 8 bits, 6.4 bytes per pixel and channel with a hidden layer four times as wide, instead of 20 in
bfloat16 and 40 in float32.

    block = OrientedBlock(96, 31).cuda().bfloat16()
    y = block(x)                                  # x: (N, H, W, 96)

`python -m paper_2309_15812_amd.block` fits a small one to a target on the GPU, with and without checkpoints.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import ops


class OrientedBlockFunction(torch.autograd.Function):
    """apply(x, theta, w_dw, ln_w, ln_b, w1, b1, w2, b2, act, eps, checkpoint, keep=True); theta gets no gradient.  keep=False:
    there will be no backward, and nothing is kept for it."""

    @staticmethod
    def forward(ctx, x, theta, w_dw, ln_w, ln_b, w1, b1, w2, b2, act, eps, checkpoint, keep=True):
        x = x.contiguous()
        u = ops.fwd_ex(x, w_dw, theta, layout="nhwc")
        v, mean, rstd = ops.ln_fwd(u, ln_w, ln_b, eps)
        if not (keep and any(ctx.needs_input_grad)):
            return ops.linear_fwd(ops.linear_fwd(v, w1, b1, act=act), w2, b2, residual=x)
        a, pre = ops.linear_fwd(v, w1, b1, act=act, save="pack8" if checkpoint else "pre")
        y = ops.linear_fwd(a, w2, b2, residual=x)
        if checkpoint:
            u, v, a = ops.pack8(u), ops.pack8(v), None
        ctx.act, ctx.cols = act, (w_dw.shape[0], w1.shape[0])
        ctx.save_for_backward(x, theta, w_dw, ln_w, w1, w2, mean, rstd, a,
                              *(t for held in (u, v, pre) for t in ops._parts(held)))
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        x, theta, w_dw, ln_w, w1, w2, mean, rstd, a, u, us, v, vs, pre, ps = ctx.saved_tensors
        C, hidden = ctx.cols
        u, v, pre = ops._whole(u, us, C), ops._whole(v, vs, C), ops._whole(pre, ps, hidden)
        dy, act = gy.contiguous(), ctx.act
        want_x, _, want_dw, want_ln_w, want_ln_b, want_w1, want_b1, want_w2, want_b2 = ctx.needs_input_grad[:9]
        deep = want_x or want_dw or want_ln_w or want_ln_b
        dx = dw_dw = dln_w = dln_b = dw1 = db1 = dw2 = db2 = None
        if want_w2 or want_b2:
            # the second product's input is kept, or made again from the pre-activation
            src, src_act = (pre, act) if a is None else (a, "none")
            dw2, db2 = ops.linear_bwd_weight(src, dy, act=src_act, bias=want_b2)
        if deep or want_w1 or want_b1:
            dh = ops.linear_bwd_input(dy, w2, pre=None if act == "none" else pre, act=act)
            if want_w1 or want_b1:
                dw1, db1 = ops.linear_bwd_weight(v, dh, bias=want_b1)
        if deep:
            du, dln_w, dln_b = ops.ln_bwd(u, ops.linear_bwd_input(dh, w1), mean, rstd, ln_w)
        if want_x:
            dx = ops.bwd_input_ex(du, w_dw, theta, tuple(x.shape[1:3]), layout="nhwc").add_(dy)
        if want_dw:
            dw_dw = ops.bwd_weight_ex(x, du, theta, w_dw.shape[1], layout="nhwc")
        return dx, None, dw_dw, dln_w, dln_b, dw1, db1, dw2, db2, None, None, None, None


class OrientedBlock(torch.nn.Module):
    """channels C, kernel length K, `directions` angles over the channels in equal groups, hidden width expand * C."""

    def __init__(self, C: int, K: int, directions: int = 8, expand: int = 4, act: str = "gelu", eps: float = 1e-6,
                 checkpoint: bool = False):
        super().__init__()
        hidden = expand * C
        self.act, self.eps, self.checkpoint = act, eps, checkpoint
        self.register_buffer("theta", (torch.arange(C) * directions // C) * (180.0 / directions), persistent=True)
        self.w_dw = torch.nn.Parameter(torch.randn(C, K) * K ** -0.5)
        self.ln_w, self.ln_b = torch.nn.Parameter(torch.ones(C)), torch.nn.Parameter(torch.zeros(C))
        self.w1, self.b1 = torch.nn.Parameter(torch.randn(hidden, C) * C ** -0.5), torch.nn.Parameter(torch.zeros(hidden))
        self.w2, self.b2 = torch.nn.Parameter(torch.randn(C, hidden) * hidden ** -0.5), torch.nn.Parameter(torch.zeros(C))

    def _apply(self, fn, *args, **kwargs):
        # a cast of the module is one of its weights: the angles move with it and stay float32 (bfloat16 makes 158 of 157.5)
        theta = self.theta
        super()._apply(fn, *args, **kwargs)
        if self.theta.dtype != torch.float32:
            self.theta = theta.to(self.theta.device)
        return self

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return OrientedBlockFunction.apply(x, self.theta, self.w_dw, self.ln_w, self.ln_b, self.w1, self.b1, self.w2,
                                           self.b2, self.act, self.eps, self.checkpoint, torch.is_grad_enabled())


def main(steps: int = 20) -> None:
    for checkpoint in (False, True):
        torch.manual_seed(1)
        target, block = (OrientedBlock(96, 31, checkpoint=checkpoint).cuda().bfloat16() for _ in range(2))
        x = torch.randn(16, 28, 28, 96, device="cuda", dtype=torch.bfloat16)
        with torch.no_grad():
            want = target(x)
        opt = torch.optim.Adam(block.parameters(), lr=3e-3)
        for step in range(steps):
            before = torch.cuda.memory_allocated()
            y = block(x)
            kept = torch.cuda.memory_allocated() - before - y.numel() * y.element_size()
            loss = (y.float() - want.float()).square().mean()
            opt.zero_grad()
            loss.backward()
            opt.step()
            if step % 5 == 0 or step == steps - 1:
                print(f"checkpoint={checkpoint} step {step}: loss {loss.item():.4f}, kept for the backward {kept / 1e6:.1f} MB",
                      flush=True)


if __name__ == "__main__":
    main()
