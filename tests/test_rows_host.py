"""Argument checks of the row operators' C ABI (no GPU needed: every call fails before any launch, or has no rows)."""
import ctypes

import pytest

from paper_2309_15812_amd import _lib

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16 = 0, 1


def at(k):  # device addresses 256 MiB apart, never used
    return ctypes.c_void_p(0x100000000 + k * 0x10000000)


def ln_fwd(x=at(0), ldx=24, w=at(1), b=at(2), y=at(3), ldy=24, mean=at(4), rstd=at(5), M=8, C=24, eps=1e-6, dt=F32):
    return _lib.call("o1d_ln_fwd", x, ldx, w, b, y, ldy, mean, rstd, M, C, eps, dt, None)


def ln_bwd(x=at(0), ldx=24, q=None, s=None, dy=at(1), lddy=24, mean=at(2), rstd=at(3), w=at(4), dx=at(5), lddx=24, dw=at(6),
           db=at(7), M=8, C=24, dt=F32, ws=at(8), n=1 << 20):
    return _lib.call("o1d_ln_bwd", x, ldx, q, s, dy, lddy, mean, rstd, w, dx, lddx, dw, db, M, C, dt, ws, n, None)


def fwd(x=at(0), ldx=24, w=at(1), b=at(2), act=0, res=at(3), ldres=40, y=at(4), ldy=40, pre=at(5), ldpre=40, q=at(6), s=at(7),
        M=8, I=24, O=40, dt=F32):
    return _lib.call("o1d_linear_fwd", x, ldx, w, b, act, res, ldres, y, ldy, pre, ldpre, q, s, M, I, O, dt, None)


def bwd_input(dy=at(0), lddy=40, w=at(1), act=2, pre=at(2), ldpre=24, q=None, s=None, dx=at(3), lddx=24, M=8, I=24, O=40,
              dt=F32):
    return _lib.call("o1d_linear_bwd_input", dy, lddy, w, act, pre, ldpre, q, s, dx, lddx, M, I, O, dt, None)


def bwd_weight(x=at(0), ldx=24, q=None, s=None, act=0, dy=at(1), lddy=40, dw=at(2), db=at(3), M=8, I=24, O=40, dt=F32,
               ws=at(4), n=1 << 20):
    return _lib.call("o1d_linear_bwd_weight", x, ldx, q, s, act, dy, lddy, dw, db, M, I, O, dt, ws, n, None)


def act_bwd(pre=at(0), ldpre=24, q=None, s=None, act=2, dy=at(1), lddy=24, dh=at(2), lddh=24, M=8, C=24, dt=F32):
    return _lib.call("o1d_act_bwd", pre, ldpre, q, s, act, dy, lddy, dh, lddh, M, C, dt, None)


def pack(x=at(0), ldx=24, q=at(1), s=at(2), M=8, C=24, dt=F32):
    return _lib.call("o1d_pack", x, ldx, q, s, M, C, dt, None)


def unpack(q=at(0), s=at(1), act=0, y=at(2), ldy=24, M=8, C=24, dt=F32):
    return _lib.call("o1d_unpack", q, s, act, y, ldy, M, C, dt, None)


ODD = ctypes.c_void_p(0x100000000 + 2)

REFUSED = [
    (ln_fwd, dict(M=-1), INVALID), (ln_fwd, dict(C=0), INVALID), (ln_fwd, dict(dt=9), INVALID), (ln_fwd, dict(ldx=23), INVALID),
    (ln_fwd, dict(x=None), INVALID), (ln_fwd, dict(w=None), INVALID), (ln_fwd, dict(y=at(0)), INVALID),
    (ln_fwd, dict(mean=None), INVALID), (ln_fwd, dict(eps=-1.0), INVALID), (ln_fwd, dict(eps=float("nan")), INVALID),
    (ln_fwd, dict(ldx=1 << 21), UNSUPPORTED), (ln_fwd, dict(C=(1 << 20) + 1, ldx=1 << 20, ldy=1 << 20), UNSUPPORTED),
    (ln_fwd, dict(M=0x7fffffff), UNSUPPORTED), (ln_fwd, dict(x=ODD), INVALID), (ln_fwd, dict(rstd=at(4)), INVALID),
    (ln_bwd, dict(x=None), INVALID), (ln_bwd, dict(q=at(9), s=at(10)), INVALID), (ln_bwd, dict(x=None, q=at(9)), INVALID),
    (ln_bwd, dict(x=None, q=ODD, s=at(10)), INVALID), (ln_bwd, dict(dw=None), INVALID), (ln_bwd, dict(dx=at(1)), INVALID),
    (ln_bwd, dict(db=at(6)), INVALID), (ln_bwd, dict(ws=None), WORKSPACE), (ln_bwd, dict(n=8), WORKSPACE),
    (ln_bwd, dict(ws=at(5)), INVALID), (ln_bwd, dict(lddy=3), INVALID), (ln_bwd, dict(C=-4), INVALID),
    (fwd, dict(M=-2), INVALID), (fwd, dict(I=0), INVALID), (fwd, dict(O=0), INVALID), (fwd, dict(act=5), INVALID),
    (fwd, dict(act=-1), INVALID), (fwd, dict(ldx=5), INVALID), (fwd, dict(ldres=5), INVALID), (fwd, dict(ldpre=39), INVALID),
    (fwd, dict(x=None), INVALID), (fwd, dict(w=None), INVALID), (fwd, dict(y=None), INVALID), (fwd, dict(q=None), INVALID),
    (fwd, dict(s=None), INVALID), (fwd, dict(q=ODD), INVALID), (fwd, dict(y=at(3)), INVALID), (fwd, dict(y=at(1)), INVALID),
    (fwd, dict(pre=at(4)), INVALID), (fwd, dict(dt=-1), INVALID), (fwd, dict(ldy=1 << 22), UNSUPPORTED),
    (fwd, dict(M=0x7fffff00, O=1 << 16, ldres=1 << 16, ldy=1 << 16, ldpre=1 << 16, res=None, pre=None, q=None, s=None,
               y=ctypes.c_void_p(1 << 62)), UNSUPPORTED),
    (bwd_input, dict(pre=None), INVALID), (bwd_input, dict(q=at(5), s=at(6)), INVALID), (bwd_input, dict(lddx=1), INVALID),
    (bwd_input, dict(pre=None, q=at(5)), INVALID), (bwd_input, dict(dx=at(0)), INVALID), (bwd_input, dict(act=7), INVALID),
    (bwd_input, dict(w=None), INVALID), (bwd_input, dict(O=-1), INVALID), (bwd_input, dict(dx=at(2)), INVALID),
    (bwd_weight, dict(x=None), INVALID), (bwd_weight, dict(q=at(5), s=at(6)), INVALID), (bwd_weight, dict(dw=None), INVALID),
    (bwd_weight, dict(dy=None), INVALID), (bwd_weight, dict(ws=None), WORKSPACE), (bwd_weight, dict(n=100), WORKSPACE),
    (bwd_weight, dict(dw=at(1)), INVALID), (bwd_weight, dict(db=at(2)), INVALID), (bwd_weight, dict(ws=at(0)), INVALID),
    (bwd_weight, dict(ldx=7), INVALID), (bwd_weight, dict(act=9), INVALID),
    (bwd_weight, dict(ws=ctypes.c_void_p(0x200000008)), INVALID),
    (act_bwd, dict(pre=None), INVALID), (act_bwd, dict(dh=at(1)), INVALID), (act_bwd, dict(dy=None), INVALID),
    (act_bwd, dict(act=11), INVALID), (act_bwd, dict(lddh=2), INVALID),
    (pack, dict(x=None), INVALID), (pack, dict(q=None), INVALID), (pack, dict(q=at(0)), INVALID), (pack, dict(s=at(1)), INVALID),
    (pack, dict(q=ODD), INVALID), (pack, dict(ldx=2), INVALID),
    (unpack, dict(y=None), INVALID), (unpack, dict(q=None), INVALID), (unpack, dict(y=at(0)), INVALID),
    (unpack, dict(act=6), INVALID), (unpack, dict(ldy=1), INVALID),
]


@pytest.mark.parametrize("f,kw,status", REFUSED)
def test_refusals(f, kw, status):
    assert f(**kw) == status
    assert _lib.lib().o1d_last_error().decode().startswith("o1d_")


def test_no_rows_launch_nothing():
    assert ln_fwd(M=0, x=None, y=None) == OK
    assert fwd(M=0, x=None, w=None, y=None, res=None, pre=None, q=None, s=None) == OK
    assert bwd_input(M=0, dy=None, dx=None) == OK
    assert act_bwd(M=0, dy=None, dh=None) == OK
    assert pack(M=0, x=None) == OK and unpack(M=0, y=None) == OK


def test_workspace_sizes():
    L = _lib.lib()
    n = L.o1d_ln_bwd_workspace_bytes(200704, 96, F32)
    assert 0 < n <= 16 << 20 and n % (2 * 96 * 4) == 0
    assert L.o1d_ln_bwd_workspace_bytes(0, 96, F32) == 0 and L.o1d_ln_bwd_workspace_bytes(4, 0, F32) == 0
    plain = L.o1d_linear_bwd_weight_workspace_bytes(50176, 768, 192, 0, 0, BF16)
    made = L.o1d_linear_bwd_weight_workspace_bytes(50176, 768, 192, 2, 1, BF16)
    assert 0 < plain <= made
    assert L.o1d_linear_bwd_weight_workspace_bytes(10, 24, 40, 0, 0, 7) == 0


def test_wrappers_refuse_host_tensors():
    import torch

    from paper_2309_15812_amd import ops

    x = torch.zeros(4, 24)
    for call in (lambda: ops.pack8(x), lambda: ops.ln_fwd(x, x[0], x[0]), lambda: ops.linear_fwd(x, torch.zeros(3, 24)),
                 lambda: ops.linear_bwd_weight(x, x), lambda: ops.act_bwd(x, x, "gelu"),
                 lambda: ops.Packed8(torch.zeros(2, 16, dtype=torch.int8), torch.zeros(2, 1), 16)):
        with pytest.raises(ValueError):
            call()
