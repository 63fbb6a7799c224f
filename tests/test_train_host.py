"""Argument checks of group norm's, the 8-bit products' and AdamW's C ABI, and the sizes of their workspaces (no GPU needed: every
call fails before any launch, or has nothing to do)."""
import ctypes
import itertools

import pytest

from paper_2309_15812_amd import _lib, ops

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16 = 0, 1
SILU = 4


def at(k):  # device addresses 256 MiB apart, never used
    return ctypes.c_void_p(0x100000000 + k * 0x10000000)


ODD = ctypes.c_void_p(0x100000000 + 2)


def gn_fwd(x=at(0), ldx=24, w=at(1), b=at(2), act=SILU, y=at(3), ldy=24, mean=at(4), rstd=at(5), N=2, P=9, C=24, G=4, eps=1e-5, dt=F32,
           ws=at(6), n=1 << 20):
    return _lib.call("o1d_gn_fwd", x, ldx, w, b, act, y, ldy, mean, rstd, N, P, C, G, eps, dt, ws, n, None)


def gn_bwd(x=at(0), ldx=24, dy=at(1), lddy=24, mean=at(2), rstd=at(3), w=at(4), b=at(5), act=0, dx=at(6), lddx=24, dw=at(7), db=at(8),
           N=2, P=9, C=24, G=4, dt=BF16, ws=at(9), n=1 << 20):
    return _lib.call("o1d_gn_bwd", x, ldx, dy, lddy, mean, rstd, w, b, act, dx, lddx, dw, db, N, P, C, G, dt, ws, n, None)


def pack(x=at(0), ldx=24, type=0, q=at(1), e=at(2), qt=at(3), et=at(4), sums=at(5), M=8, C=24, dt=F32, ws=at(6), n=1 << 20):
    return _lib.call("o1d_pack_scaled", x, ldx, type, q, e, qt, et, sums, M, C, dt, ws, n, None)


def fwd(xq=at(0), xe=at(1), type=0, wq=at(2), we=at(3), b=at(4), act=2, res=at(5), ldres=40, y=at(6), ldy=40, pre=at(7), ldpre=40,
        M=8, I=24, O=40, dt=BF16):
    return _lib.call("o1d_scaled_linear_fwd", xq, xe, type, wq, we, b, act, res, ldres, y, ldy, pre, ldpre, M, I, O, dt, None)


def bwd_input(dyq=at(0), dye=at(1), type=1, wq=at(2), we=at(3), act=2, pre=at(4), ldpre=24, dx=at(5), lddx=24, M=8, I=24, O=40, dt=BF16):
    return _lib.call("o1d_scaled_linear_bwd_input", dyq, dye, type, wq, we, act, pre, ldpre, dx, lddx, M, I, O, dt, None)


def bwd_weight(dyq=at(0), dye=at(1), type=1, xq=at(2), xe=at(3), dw=at(4), M=9000, I=24, O=40, dt=BF16, ws=at(5), n=1 << 26):
    return _lib.call("o1d_scaled_linear_bwd_weight", dyq, dye, type, xq, xe, dw, M, I, O, dt, ws, n, None)


def adamw(tensors=((at(0), at(1), 300, 0), (at(2), at(3), 5, 384)), count=None, pdt=F32, gdt=F32, bits=8, m=at(4), v=at(5), ms=at(6),
          vs=at(7), master=at(8), step=at(9), norm=at(10), ws=at(11), n=1 << 20, lr_at=None, **options):
    table = (_lib.AdamTensor * max(1, len(tensors)))(*(_lib.AdamTensor(p, g, size, start) for p, g, size, start in tensors))
    s = _lib.AdamState(m, v, ms, vs, master, step, bits)
    h = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, "weight_decay": 0.1, "max_norm": 1.0, **options}
    o = _lib.AdamOptions(*(h[k] for k in ("lr", "beta1", "beta2", "eps", "weight_decay", "max_norm")), lr_at)
    return _lib.call("o1d_adamw", ctypes.addressof(table), len(tensors) if count is None else count, pdt, gdt, ctypes.addressof(s),
                     ctypes.addressof(o), norm, ws, n, None)


INF, NAN = float("inf"), float("nan")
ONE = (at(0), at(1), 300, 0)

REFUSED = [
    (gn_fwd, dict(N=-1), INVALID), (gn_fwd, dict(P=0), INVALID), (gn_fwd, dict(P=-3), INVALID), (gn_fwd, dict(C=0), INVALID),
    (gn_fwd, dict(G=0), INVALID), (gn_fwd, dict(G=5), INVALID), (gn_fwd, dict(G=48), INVALID), (gn_fwd, dict(act=9), INVALID),
    (gn_fwd, dict(dt=7), INVALID), (gn_fwd, dict(ldx=23), INVALID), (gn_fwd, dict(ldy=23), INVALID), (gn_fwd, dict(eps=-1.0), INVALID),
    (gn_fwd, dict(eps=NAN), INVALID), (gn_fwd, dict(eps=INF), INVALID), (gn_fwd, dict(x=None), INVALID), (gn_fwd, dict(w=None), INVALID),
    (gn_fwd, dict(mean=None), INVALID), (gn_fwd, dict(rstd=at(4)), INVALID), (gn_fwd, dict(y=at(0)), INVALID), (gn_fwd, dict(x=ODD), INVALID),
    (gn_fwd, dict(C=1025, G=1, ldx=1025, ldy=1025), UNSUPPORTED), (gn_fwd, dict(N=1 << 16, P=1 << 16), UNSUPPORTED),
    (gn_fwd, dict(ldx=1 << 21), UNSUPPORTED), (gn_fwd, dict(P=3136, C=96, G=32, ldx=96, ldy=96, N=1, ws=None), WORKSPACE),
    (gn_fwd, dict(P=3136, C=96, G=32, ldx=96, ldy=96, N=1, n=100), WORKSPACE),
    (gn_fwd, dict(P=3136, C=96, G=32, ldx=96, ldy=96, N=1, ws=at(5)), INVALID),
    (gn_bwd, dict(dw=None), INVALID), (gn_bwd, dict(db=at(7)), INVALID), (gn_bwd, dict(dx=at(1)), INVALID), (gn_bwd, dict(dx=at(0)), INVALID),
    (gn_bwd, dict(mean=None), INVALID), (gn_bwd, dict(b=None), INVALID), (gn_bwd, dict(lddx=3), INVALID), (gn_bwd, dict(lddy=3), INVALID),
    (gn_bwd, dict(ws=None), WORKSPACE), (gn_bwd, dict(n=8), WORKSPACE), (gn_bwd, dict(G=7), INVALID), (gn_bwd, dict(act=-1), INVALID),
    (gn_bwd, dict(ws=ctypes.c_void_p(0x200000008)), INVALID), (gn_bwd, dict(C=2050, G=2, ldx=2050, lddy=2050, lddx=2050), UNSUPPORTED),
    (pack, dict(M=-1), INVALID), (pack, dict(C=0), INVALID), (pack, dict(type=2), INVALID), (pack, dict(dt=5), INVALID),
    (pack, dict(ldx=2), INVALID), (pack, dict(x=None), INVALID), (pack, dict(e=None), INVALID), (pack, dict(et=None), INVALID),
    (pack, dict(q=None, e=None, qt=None, et=None), INVALID), (pack, dict(qt=None, et=None), INVALID), (pack, dict(q=ODD), INVALID),
    (pack, dict(ws=None), WORKSPACE), (pack, dict(n=10), WORKSPACE), (pack, dict(q=at(0)), INVALID), (pack, dict(qt=at(1)), INVALID),
    (pack, dict(sums=at(4)), INVALID), (pack, dict(sums=ODD), INVALID), (pack, dict(C=(1 << 20) + 1, ldx=1 << 20), UNSUPPORTED),
    (pack, dict(M=1 << 30, C=1, ldx=1), UNSUPPORTED), (gn_fwd, dict(N=1 << 27, P=1, C=8, G=1, ldx=8, ldy=8,
     **{k: ctypes.c_void_p(1 << (42 + i)) for i, k in enumerate(("x", "y", "mean", "rstd", "ws"))}, n=1 << 40), UNSUPPORTED),
    (fwd, dict(M=-1), INVALID), (fwd, dict(I=0), INVALID), (fwd, dict(O=0), INVALID), (fwd, dict(type=-1), INVALID), (fwd, dict(act=5), INVALID),
    (fwd, dict(ldy=39), INVALID), (fwd, dict(ldres=39), INVALID), (fwd, dict(ldpre=39), INVALID), (fwd, dict(xq=None), INVALID),
    (fwd, dict(we=None), INVALID), (fwd, dict(y=None), INVALID), (fwd, dict(wq=ODD), INVALID), (fwd, dict(xe=ODD), INVALID),
    (fwd, dict(y=at(5)), INVALID), (fwd, dict(pre=at(6)), INVALID), (fwd, dict(y=at(0)), INVALID), (fwd, dict(b=ctypes.c_void_p(0x140000001)), INVALID),
    (fwd, dict(ldy=1 << 21), UNSUPPORTED), (fwd, dict(M=0x7fffffff), UNSUPPORTED),
    (fwd, dict(M=0x7fffff00 // 2, O=1 << 16, I=1, ldy=1 << 16, res=None, pre=None, y=ctypes.c_void_p(1 << 62)), UNSUPPORTED),
    (bwd_input, dict(pre=None), INVALID), (bwd_input, dict(ldpre=2), INVALID), (bwd_input, dict(dx=at(4)), INVALID), (bwd_input, dict(dyq=None), INVALID),
    (bwd_input, dict(lddx=2), INVALID), (bwd_input, dict(act=6), INVALID), (bwd_input, dict(type=3), INVALID), (bwd_input, dict(dx=None), INVALID),
    (bwd_weight, dict(dw=None), INVALID), (bwd_weight, dict(ws=None), WORKSPACE), (bwd_weight, dict(n=100), WORKSPACE), (bwd_weight, dict(xe=None), INVALID),
    (bwd_weight, dict(dw=at(2)), INVALID), (bwd_weight, dict(ws=at(0)), INVALID), (bwd_weight, dict(M=1 << 25), UNSUPPORTED),
    (bwd_weight, dict(type=2), INVALID), (bwd_weight, dict(M=-1), INVALID),
    (adamw, dict(count=-1), INVALID), (adamw, dict(pdt=2), INVALID), (adamw, dict(gdt=-1), INVALID), (adamw, dict(bits=16), INVALID),
    (adamw, dict(lr=-1.0), INVALID), (adamw, dict(lr=NAN), INVALID), (adamw, dict(beta1=1.0), INVALID), (adamw, dict(beta2=-0.1), INVALID),
    (adamw, dict(eps=INF), INVALID), (adamw, dict(weight_decay=NAN), INVALID), (adamw, dict(max_norm=-1.0), INVALID), (adamw, dict(max_norm=INF), INVALID),
    (adamw, dict(step=None), INVALID), (adamw, dict(norm=None), INVALID), (adamw, dict(m=None), INVALID), (adamw, dict(ms=None), INVALID),
    (adamw, dict(v=ctypes.c_void_p(0x150000008)), INVALID), (adamw, dict(ws=None), WORKSPACE), (adamw, dict(n=8), WORKSPACE),
    (adamw, dict(master=at(4)), INVALID), (adamw, dict(norm=at(9)), INVALID), (adamw, dict(lr_at=at(9)), INVALID), (adamw, dict(lr_at=ODD), INVALID),
    (adamw, dict(tensors=(ONE, ONE)), INVALID), (adamw, dict(tensors=(ONE, (at(0), at(3), 5, 384))), INVALID),  # the same tensor twice
    (adamw, dict(tensors=(ONE, (at(2), at(3), 5, 256))), INVALID), (adamw, dict(tensors=(ONE, (at(2), at(0), 5, 384))), INVALID),
    (adamw, dict(tensors=((at(0), at(1), 300, 64),)), INVALID), (adamw, dict(tensors=((at(0), at(1), -1, 0),)), INVALID),
    (adamw, dict(tensors=((at(0), at(1), 300, -128),)), INVALID), (adamw, dict(tensors=((None, at(1), 300, 0),)), INVALID),
    (adamw, dict(tensors=((at(0), ODD, 300, 0),)), INVALID), (adamw, dict(tensors=((at(0), at(1), (1 << 37) + 1, 0),)), UNSUPPORTED),
]


@pytest.mark.parametrize("f,kw,status", REFUSED)
def test_refusals(f, kw, status):
    assert f(**kw) == status
    assert _lib.lib().o1d_last_error()


def test_nothing_to_do():
    assert gn_fwd(N=0, P=0) == gn_fwd(N=0, x=None, y=None) == OK
    assert pack(M=0, sums=None) == fwd(M=0) == bwd_input(M=0) == OK
    assert adamw(tensors=(), max_norm=0.0, norm=None) == adamw(tensors=((at(0), at(1), 0, 0),), max_norm=0.0, norm=None, ws=None, n=0) == OK


def test_workspaces_are_nothing_or_larger_than_what_calls_share():
    lib = _lib.lib()
    for N, P, (C, G), dt in itertools.product([1, 2, 7, 300], [1, 3, 49, 1000, 12707], [(1, 1), (6, 3), (24, 3), (96, 32), (203, 7)], [F32, BF16]):
        b = lib.o1d_gn_fwd_workspace_bytes(N, P, C, G, dt)
        assert b == ops._NO_SPACE or b >= 2 * ops._NO_SPACE, (N, P, C, G, dt)
        b = lib.o1d_gn_bwd_workspace_bytes(N, P, C, G, dt)  # (dw and db of each sample at least)
        assert b >= max(2 * ops._NO_SPACE, 8 * N * C)
    for M, I, O, dt in itertools.product([1, 100, 700, 9001, 50176], [1, 24, 192], [1, 17, 768], [F32, BF16]):
        b = lib.o1d_scaled_linear_bwd_weight_workspace_bytes(M, I, O, dt)
        assert b == ops._NO_SPACE or b >= max(2 * ops._NO_SPACE, 8 * I * O)
        assert lib.o1d_pack_scaled_workspace_bytes(M, I, 0) == ops._NO_SPACE
        assert lib.o1d_pack_scaled_workspace_bytes(M, I, 1) >= max(2 * ops._NO_SPACE, -(-M // 128) * I * 4)
    assert lib.o1d_adamw_workspace_bytes(0.0) == ops._NO_SPACE < lib.o1d_adamw_workspace_bytes(1.0)


def test_sizes_that_no_call_takes_ask_for_nothing():
    lib = _lib.lib()
    assert lib.o1d_gn_fwd_workspace_bytes(2, 9, 24, 5, F32) == lib.o1d_gn_bwd_workspace_bytes(0, 9, 24, 4, F32) == 0
    assert lib.o1d_scaled_linear_bwd_weight_workspace_bytes(1 << 25, 24, 40, F32) == lib.o1d_pack_scaled_workspace_bytes(-1, 24, 1) == 0
